"""A cache of 8 bits: read back, copied, committed, all of them exact."""
import pytest
import torch

import plain_cache as pc
from paper_2510_26475_amd import binding
from plain_cache import Cache, ints, offsets

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lens,Hkv,D,page", [([1], 1, 64, 16), ([0, 40, 0, 0, 17, 1, 300], 2, 64, 16), ([5, 1000, 64], 8, 128, 64), ([2500], 3, 128, 1024)])
def test_read_back(dtype, lens, Hkv, D, page):
    c = Cache(lens, Hkv, D, page, torch.float32, pool="e4m3", table_room=1)
    room = [n + 2 for n in lens]                                  # rows of no token between the sequences
    total = sum(room) + 5
    out = [torch.full((total, Hkv, D), 9.0, dtype=dtype, device="cuda") for _ in range(2)]
    want = [x.clone() for x in out]
    kv_indptr = offsets(room, torch.int64) + 3
    binding.respec_read_paged_quantised(*c.args(), *c.tables(), kv_indptr, *out, max(max(lens), 1))
    for w, name in zip(want, "kv"):
        for b, n in enumerate(lens):
            at = kv_indptr[b].item()
            w[at:at + n] = c.tokens(name, b).to(dtype)           # (exact in both types)
    for w, o in zip(want, out):
        assert torch.equal(w, o)


def test_read_back_is_cut_by_what_it_is_given():
    """By max_kv_len, by the rows between two offsets, by the pages a sequence has; a page id that does not exist leaves its rows."""
    c = Cache([100, 40, 60], 2, 64, 16, torch.float32, pool="e4m3")
    c.page_table[c.page_indptr[1] + 1] = 10 ** 6
    c.kv_len[2] = 1000
    kv_indptr = ints([0, 50, 90, 250], torch.int64)
    out = [torch.full((250, 2, 64), 9.0, device="cuda") for _ in range(2)]
    binding.respec_read_paged_quantised(*c.args(), *c.tables(), kv_indptr, *out, 70)
    for o, name in zip(out, "kv"):
        want = torch.full_like(o, 9.0)
        want[:50] = c.tokens(name, 0)[:50].float()
        t = c.tokens(name, 2).float()
        want[90:150] = t
        got = o.clone()
        assert torch.equal(got[:50], want[:50]) and torch.equal(got[90:150], want[90:150]) and (got[154:] == 9.0).all()
        c.page_table[c.page_indptr[1] + 1] = 10 ** 6
        assert (got[66:82] == 9.0).all() and not (got[50:66] == 9.0).any() and not (got[82:90] == 9.0).any()


@pytest.mark.parametrize("Hkv,D,page", [(1, 64, 16), (4, 128, 16), (3, 64, 256), (8, 128, 1024)])
def test_copies(Hkv, D, page):
    n = 9
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = [torch.randint(0, 256, shape, generator=gen, device="cuda", dtype=torch.uint8) for shape in [(n, page, Hkv, D)] * 2 + [(n, Hkv, page)] * 2]
    want = [y.clone() for y in x]
    src, dst = [0, 3, -1, 5, 4, 99, 2], [8, 7, 1, 5, -2, 6, 10 ** 6]
    for a, b in ((0, 8), (3, 7)):
        for w in want:
            w[b] = w[a]
    binding.respec_pages_copy_quantised(*x, ints(src), ints(dst))
    for w, y in zip(want, x):
        assert torch.equal(w, y)


@pytest.mark.parametrize("Hkv,D,page", [(1, 64, 16), (4, 128, 32)])
def test_commit_does_what_it_does_in_bf16(Hkv, D, page):
    """Chains, paths, paths that are none, sequences without rows or shorter than their rows: the moves and lengths of respec_commit_accepted_paged."""
    R, L = [4, 7, 5, 1, 3, 6, 0], [30, 17, 64, 1, 2, 40, 9]
    path = [[1, 2, 3], [2, 4, 6], [1, 3, 4], [0, 0, 0], [1, 2, -1], [3, 2, 5], [1, 2, 3]]
    accepted = [2, 3, 3, 0, 1, 3, 1]
    for paths in (None, path):
        c = Cache(L, Hkv, D, page, torch.float32, pool="e4m3")
        codes = [x.view(torch.uint8) for x in (c.k, c.v)]
        # the same moves on bf16 pools that hold codes and scales as numbers
        wide = [x.to(torch.bfloat16) for x in codes]
        marks = [s.transpose(1, 2)[..., None].expand(-1, -1, -1, D).to(torch.bfloat16).contiguous() for s in (c.k_scale, c.v_scale)]
        lens, lens2, lens3 = c.kv_len.clone(), c.kv_len.clone(), c.kv_len.clone()
        p = None if paths is None else ints(paths)
        tables = offsets(R), c.page_indptr, c.page_table
        binding.respec_commit_accepted_paged(*wide, *tables, lens, ints(accepted), sum(R), max(R), path=p)
        binding.respec_commit_accepted_paged(*marks, *tables, lens2, ints(accepted), sum(R), max(R), path=p)
        binding.respec_commit_accepted_paged_quantised(*codes, c.k_scale, c.v_scale, *tables, lens3, ints(accepted), sum(R), max(R), path=p)
        assert torch.equal(lens, lens3)
        for w, m, x, s in zip(wide, marks, codes, (c.k_scale, c.v_scale)):
            assert torch.equal(w, x.to(torch.bfloat16)) and torch.equal(m[..., 0], s.transpose(1, 2).to(torch.bfloat16))
