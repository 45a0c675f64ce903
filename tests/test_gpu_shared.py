"""Verify attention over pages that groups of sequences share, and over a cache of 8 bits, against float64."""
import math

import pytest
import torch

import plain
import plain_cache as pc
from paper_2510_26475_amd import binding
from plain_cache import Cache, ints, offsets, scratch

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def workspace(B, total_q, groups, max_q, max_kv, Hq, Hkv, D, dtype, fill=0xa5):
    ws = scratch(binding.respec_verify_attention_shared_workspace_bytes(B, total_q, groups, max_q, max_kv, Hq, Hkv, D, int(dtype == BF16)))
    return ws.fill_(fill)


def run(c, R, Hq, dtype, groups=(), shared=(), masks=None, scale=None, seed=5, entry="respec_verify_attention_shared", max_q=None, max_kv=None, ws=None, q=None,
        lse=True):
    """One call over the cache; returns q, out and lse."""
    D = c.D
    if q is None:
        q = torch.randn((sum(R), Hq, D), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)
    out, z = torch.full((sum(R) + 2, Hq, D), 5.0, dtype=dtype, device="cuda"), torch.full((sum(R) + 2, Hq), 5.0, device="cuda")
    max_q, max_kv = max_q or max(R), max_kv or max(max(c.lens), 1)
    g = (ints([a[0] for a in groups] + [groups[-1][-1] + 1]), ints(shared)) if groups else (None, None)
    if ws is None:
        ws = workspace(len(R), sum(R), len(groups), max_q, max_kv, Hq, c.Hkv, D, dtype)
    mask = None if masks is None else ints(masks, torch.int64)
    scale = 1 / math.sqrt(D) if scale is None else scale
    getattr(binding, entry)(q, *c.args(), offsets(R), *c.tables(), *g, mask, out[:sum(R)], z[:sum(R)] if lse else None, max_q, max_kv, scale, ws)
    torch.cuda.synchronize()
    assert (out[sum(R):] == 5.0).all() and (z[sum(R):] == 5.0).all()
    return q, out[:sum(R)], z[:sum(R)]


def check(c, R, Hq, dtype, groups=(), shared=(), masks=None, **kw):
    q, out, z = run(c, R, Hq, dtype, groups, shared, masks, **kw)
    ref = pc.attention(q, *c.both(), R, c.lens, kw.get("scale") if kw.get("scale") is not None else 1 / math.sqrt(c.D), masks)
    plain.check_prompt(out, z, ref)


POOLS = [(F32, "same"), (BF16, "same"), (BF16, "e4m3")]
HEADS = [(4, 1, 64), (8, 2, 128), (28, 4, 128), (6, 3, 64), (5, 5, 128)]


@pytest.mark.parametrize("dtype,pool", POOLS)
@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("page", [16, 64])
def test_sequences_by_themselves(dtype, pool, Hq, Hkv, D, page):
    """Lengths around tiles and pages, no rows, no tokens, fewer tokens than rows, one row."""
    R = [1, 4, 0, 3, 5, 2, 1, 4, 3]
    lens = [1, 4, 20, 2, 0, 31, 32, 33, 700]
    check(Cache(lens, Hkv, D, page, dtype, pool=pool, seed=1), R, Hq, dtype)


@pytest.mark.parametrize("dtype,pool", POOLS)
@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("page,prompt", [(16, 48), (16, 256), (64, 64), (64, 640), (16, 16)])
def test_groups(dtype, pool, Hq, Hkv, D, page, prompt):
    """A group, sequences by themselves before and behind it, and one more group."""
    groups, shared = [[1, 2, 3, 4], [5, 6]], [prompt, 2 * page]
    lens = [90] + [prompt + n for n in (1, 7, 33, 100)] + [2 * page + 5, 2 * page + 40, 17]
    R = [2, 1, 4, 3, 4, 1, 2, 4]
    check(Cache(lens, Hkv, D, page, dtype, groups, shared, pool, seed=2), R, Hq, dtype, groups, shared)


@pytest.mark.parametrize("dtype,pool", POOLS)
def test_any_number_of_shared_tokens(dtype, pool):
    """Not whole pages or tiles; more than a member holds before its new tokens, none, a negative number; a group of one; members without rows or tokens."""
    Hq, Hkv, D, page = 8, 2, 64, 16
    groups = [[0, 1, 2], [3], [4, 5], [6, 7, 8], [9, 10], [11, 12]]
    lens = [100, 140, 128, 50, 80, 81, 70, 64, 90, 64, 0, 70, 75]
    R = [4, 3, 1, 2, 4, 4, 1, 0, 2, 1, 2, 6, 3]
    c = Cache(lens, Hkv, D, page, dtype, groups, [96, 0, 80, 64, 0, 64], pool, seed=3)
    for shared in ([77, 50, 80, 63, 10, 1000], [96, 10, -5, 64, 64, 33], [1, 0, 31, 32, 0, 64], [64, 2 ** 31 - 1, 65, 2 ** 31 - 1, 2 ** 31 - 1, 69]):
        same = [min(s, k) for s, k in zip(shared, [96, 50, 80, 64, 0, 64])]   # (tokens that are the same: whole pages of the first member)
        check(c, R, Hq, dtype, groups, same)


@pytest.mark.parametrize("dtype,pool", POOLS)
def test_more_shared_than_a_member_holds(dtype, pool):
    groups, lens, R = [[0, 1, 2]], [70, 50, 60], [3, 5, 2]
    c = Cache(lens, 2, 64, 16, dtype, groups, [64], pool, seed=4)
    # (the second holds 45 tokens before its rows: the rest is its own, and the pages say the same)
    check(c, R, 8, dtype, groups, [64])


@pytest.mark.parametrize("dtype,pool", POOLS)
@pytest.mark.parametrize("Hq,Hkv,D,R", [(28, 4, 128, 9), (40, 8, 128, 13), (4, 1, 64, 64), (16, 2, 64, 32), (8, 8, 64, 64), (3, 1, 64, 50)])
def test_many_columns(dtype, pool, Hq, Hkv, D, R):
    """Rows and heads for two and four waves, and for two blocks of columns."""
    groups, shared = [[0, 1, 2]], [128]
    c = Cache([128 + R + 5, 128 + R, 128 + R + 70, R + 3], Hkv, D, 16, dtype, groups, shared, pool, seed=6)
    check(c, [R, R - 1, R, 2], Hq, dtype, groups, shared)
    check(c, [R, R - 1, R, 2], Hq, dtype)


@pytest.mark.parametrize("dtype,pool", POOLS)
@pytest.mark.parametrize("shape", ["wide", "chains", "holes", "full"])
def test_trees(dtype, pool, shape):
    n = 64 if shape == "full" else 7
    parent = {"wide": [-1, 0, 0, 0, 0, 0, 0], "chains": [-1, 0, 0, 1, 2, 3, 4], "holes": [-1] * 7, "full": [-1] + [(i - 1) // 2 for i in range(1, 64)]}[shape]
    masks = []
    for i, p in enumerate(parent):
        masks.append((masks[p] if p >= 0 else 0) | 1 << i)
    if shape == "holes":
        masks = [0, 1, 2, 0, 0x55, 0x7f, 0x40]                    # (rows that do not see themselves, or no new token at all)
    to_signed = [m - (1 << 64) if m >> 63 else m for m in masks]
    groups, shared = [[0, 1, 2]], [48]
    lens = [48 + n, 48 + n + 3, 48 + n + 40, n, n + 31, 400]
    c = Cache(lens, 2, 64, 16, dtype, groups, shared, pool, seed=7)
    q, out, z = run(c, [n] * 6, 6, dtype, groups, shared, to_signed * 6)
    plain.check_prompt(out, z, pc.attention(q, *c.both(), [n] * 6, lens, 1 / 8, masks * 6))
    if pool == "e4m3":
        out2, z2 = torch.empty_like(out), torch.empty_like(z)
        binding.respec_verify_attention_paged_quantised(q, *c.args(), offsets([n] * 6), *c.tables(), out2, z2, n, 400, 1 / 8,
                                                        workspace(6, 6 * n, 0, n, 400, 6, 2, 64, dtype), tree_mask=ints(to_signed * 6, torch.int64))
        plain.check_prompt(out2, z2, pc.attention(q, *c.both(), [n] * 6, lens, 1 / 8, masks * 6))


@pytest.mark.parametrize("dtype,pool", POOLS)
@pytest.mark.parametrize("scale", [0.0, -0.125, 3.0])
def test_scales(dtype, pool, scale):
    groups, shared = [[0, 1]], [64]
    check(Cache([70, 99, 40], 2, 64, 16, dtype, groups, shared, pool, seed=8), [2, 4, 3], 4, dtype, groups, shared, scale=scale)


@pytest.mark.parametrize("dtype,pool", POOLS)
def test_ranges_that_end_anywhere(dtype, pool):
    """Long sequences and prompts in many parts, and many short ones in a range."""
    check(Cache([9000], 1, 64, 16, dtype, pool=pool, seed=9), [3], 4, dtype)
    groups, shared = [[0, 1, 2, 3]], [6000 // 64 * 64]
    check(Cache([6100, 6005, 6400, 7000], 2, 64, 64, dtype, groups, shared, pool, seed=10), [4, 4, 2, 1], 4, dtype, groups, shared)
    lens = [(37 * i) % 90 + 5 for i in range(1500)]
    groups = [list(range(i, i + 5)) for i in range(0, 1000, 5)]
    shared = [min(lens[g[0]:g[-1] + 1]) // 16 * 16 - (16 if min(lens[g[0]:g[-1] + 1]) % 16 < 3 else 0) for g in groups]
    shared = [max(0, s) for s in shared]
    check(Cache(lens, 2, 64, 16, dtype, groups, shared, pool, seed=11), [i % 3 + 1 for i in range(1500)], 4, dtype, groups, shared)


@pytest.mark.parametrize("dtype,pool", [(F32, "same"), (BF16, "same"), (BF16, "e4m3")])
def test_values_that_are_not_finite(dtype, pool):
    """NaN and infinities in V reach the rows that see their key and no others: among the new tokens, among those before, among shared ones, and behind the last
    token (where the caches of these tests hold NaN)."""
    Hkv, D, page = 2, 64, 16
    groups, shared = [[0, 1]], [75]
    for where in (75, 71, 40, 100, 101, 102, 64, 72, 73):
        c = Cache([103, 110, 200], Hkv, D, page, dtype, groups, [80], pool, seed=12)
        bad = math.inf if pool == "same" and where % 2 else math.nan
        for b in (0, 1, 2):
            page_id, slot = c.pages[b][where // page], where % page
            if pool == "e4m3":
                c.v.view(torch.uint8)[page_id, slot, 1, 5] = 0x7f
            else:
                c.v[page_id, slot, 1, 5] = bad
        R = [4, 4, 4]
        q, out, z = run(c, R, 4, dtype, groups, shared)
        k, v = c.both()
        clean = [x.clone() for x in v]
        for x in clean:
            x[where, 1, 5] = 0.0
        ref = pc.attention(q, k, clean, R, c.lens, 1 / 8)
        hit = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
        for b in range(3):
            for i in range(4):
                if where <= c.lens[b] - 4 + i:
                    hit[4 * b + i, 2:, 5] = True
        assert not torch.isfinite(out[hit]).any(), where
        if math.isinf(bad):
            assert (out[hit] == math.inf).all(), where
        got = torch.where(hit, ref[0], out.double())
        plain.check_prompt(got, z, ref)


@pytest.mark.parametrize("dtype,pool", POOLS)
def test_next_layers_and_repeats_give_the_same_bits(dtype, pool):
    groups, shared = [[0, 1, 2], [3, 4]], [320, 64]
    lens, R, Hq = [330, 400, 350, 90, 300, 500], [4, 2, 4, 1, 4, 3], 8
    c, c2 = (Cache(lens, 2, 128, 64, dtype, groups, shared, pool, seed=s) for s in (13, 13))
    ws = workspace(6, sum(R), 2, 4, 500, Hq, 2, 128, dtype)
    q, out, z = run(c, R, Hq, dtype, groups, shared, ws=ws)
    for seed in (20, 21):
        q2, out2, z2 = run(c2, R, Hq, dtype, groups, shared, ws=ws, seed=seed, entry="respec_verify_attention_shared_next_layer")
        q3, out3, z3 = run(c2, R, Hq, dtype, groups, shared, seed=seed)
        assert torch.equal(out2, out3) and torch.equal(z2, z3)
    for _ in range(3):
        assert torch.equal(run(c, R, Hq, dtype, groups, shared, ws=ws)[1], out)


def test_next_layer_without_a_plan_of_its_sizes_does_nothing():
    c, R = Cache([40, 50], 2, 64, 16, BF16, seed=14), [2, 3]
    for ws in (workspace(2, 5, 0, 3, 50, 4, 2, 64, BF16, fill=0), workspace(2, 5, 0, 3, 50, 4, 2, 64, BF16, fill=0xff)):
        assert (run(c, R, 4, BF16, ws=ws, entry="respec_verify_attention_shared_next_layer")[1] == 5.0).all()
    ws = workspace(2, 5, 0, 3, 64, 4, 2, 64, BF16)
    run(c, R, 4, BF16, ws=ws)
    assert (run(c, R, 4, BF16, ws=ws, max_kv=64, entry="respec_verify_attention_shared_next_layer")[1] == 5.0).all()


@pytest.mark.parametrize("dtype,pool", POOLS)
def test_rows_and_keys_past_the_bounds(dtype, pool):
    """A sequence of more rows or tokens than the bounds say counts as one of so many."""
    c = Cache([100, 100], 2, 64, 16, dtype, pool=pool, seed=15)
    q, out, z = run(c, [5, 2], 4, dtype, max_q=3, max_kv=60)
    k, v = ([x[:60] for x in y] for y in c.both())
    q_kept = torch.cat([q[:3], q[5:]])
    ref = pc.attention(q_kept, k, v, [3, 2], [60, 60], 1 / 8)
    plain.check_prompt(torch.cat([out[:3], out[5:]]), torch.cat([z[:3], z[5:]]), ref)
    assert (out[3:5] == 5.0).all()


@pytest.mark.parametrize("dtype,pool", POOLS)
def test_data_errors_stay_inside_the_buffers(dtype, pool):
    """Offsets, page ids, lengths and groups that mean nothing: the call returns, and what belongs to sound sequences is right."""
    lens, R, Hq = [60, 70, 80, 50], [2, 2, 2, 2], 4
    c = Cache(lens, 2, 64, 16, dtype, pool=pool, seed=16)
    q, out, z = run(c, R, Hq, dtype)
    k_len, table = c.kv_len.clone(), c.page_table.clone()
    c.kv_len[1], c.kv_len[3] = 10 ** 9, -7
    c.page_table[c.page_indptr[2]] = 2 ** 31 - 1
    _, out2, _ = run(c, R, Hq, dtype, max_kv=80)
    assert torch.equal(out2[:2], out[:2])
    c.kv_len.copy_(k_len)
    c.page_table.copy_(table)
    ws = workspace(4, 8, 3, 2, 80, Hq, 2, 64, dtype)
    for gi, sl in (([0, 2, 1, 4], [10, 20, 30]), ([-5, 90, 2, 3], [50, 50, 50]), ([3, 2, 1, 0], [5, 5, 5]), ([0, 4, 4, 4], [-1, 9, 9])):
        o = torch.empty_like(out)
        binding.respec_verify_attention_shared(q, *c.args(), offsets(R), *c.tables(), ints(gi), ints(sl), None, o, None, 2, 80, 1 / 8, ws)
        torch.cuda.synchronize()
    bad = [ints([0, 5, 3, 9, 8]), ints([0, 2, 4, 6, 10 ** 6]), ints([-9, -2, 4, 6, 8])]
    for qi in bad:
        o = torch.empty_like(out)
        binding.respec_verify_attention_shared(q, *c.args(), qi, *c.tables(), ints([0, 2, 4, 4]), ints([40, 40, 40]), None, o, None, 2, 80, 1 / 8, ws)
        torch.cuda.synchronize()


@pytest.mark.parametrize("dtype,pool", POOLS)
def test_two_calls_at_once_and_captured(dtype, pool):
    """Two streams with a workspace each; a graph of a call and its next layer replayed on changed inputs with eager calls between."""
    groups, shared = [[0, 1, 2, 3]], [256]
    lens, R, Hq = [300, 270, 400, 258, 90], [4, 4, 4, 2, 3], 8
    c = Cache(lens, 2, 64, 16, dtype, groups, shared, pool, seed=17)
    g = ints([0, 4]), ints(shared)
    q = [torch.randn((sum(R), Hq, 64), device="cuda").to(dtype) for _ in range(2)]
    out, z = [torch.empty_like(x) for x in q], [torch.empty((sum(R), Hq), device="cuda") for _ in q]
    ws = [workspace(5, sum(R), 1, 4, 400, Hq, 2, 64, dtype) for _ in range(2)]

    state = offsets(R), *c.tables(), *g

    def call(i, o, lse, w, entry=binding.respec_verify_attention_shared, stream=None):
        entry(q[i], *c.args(), *state, None, o, lse, 4, 400, 1 / 8, w, stream=stream)

    def check_both():
        for x, o, lse in zip(q, out, z):
            plain.check_prompt(o, lse, pc.attention(x, *c.both(), R, lens, 1 / 8))

    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for i in (0, 1):
            call(i, out[i], z[i], ws[i], stream=streams[i])
    torch.cuda.synchronize()
    check_both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(0, out[0], z[0], ws[0])
        call(1, out[1], z[1], ws[0], binding.respec_verify_attention_shared_next_layer)
    for i in range(4):
        for x in q:
            x.copy_(torch.randn(x.shape, device="cuda"))
        for o in out:
            o.zero_()
        graph.replay()
        eager = torch.empty_like(out[0])
        torch.cuda.synchronize()
        call(0, eager, None, ws[1])
        torch.cuda.synchronize()
        assert torch.equal(eager, out[0]), i
        check_both()


def test_offsets_past_32_bits():
    """Pools of more than 2^32 elements: the sequence lies at their end."""
    Hkv, D, page, dtype = 8, 128, 16, BF16
    num = (1 << 32) // (page * Hkv * D) + 40
    k, v = (torch.empty((num, page, Hkv, D), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.full((num, Hkv, page), 120, dtype=torch.uint8, device="cuda") for _ in range(2))
    n, first = 300, num - 25
    new = [torch.randn((n, Hkv, D), device="cuda").to(dtype) for _ in range(2)]
    tables = ints([0, 19]), ints(list(range(first, first + 19))), ints([n])
    binding.respec_norm_rope_append_paged(None, *new, None, None, None, None, None, k, v, ks, vs, ints([0, n]), *tables, n, 0.0)
    back = [torch.empty_like(x) for x in new]
    binding.respec_read_paged_quantised(k, v, ks, vs, *tables, ints([0, n], torch.int64), *back, n)
    for x, y in zip(new, back):
        code, byte = pc.quantise(x)
        assert torch.equal(pc.values(code, byte), y.double())
    q = torch.randn((3, 16, D), device="cuda").to(dtype)
    out, z = torch.empty_like(q), torch.empty((3, 16), device="cuda")
    binding.respec_verify_attention_paged_quantised(q, k, v, ks, vs, ints([0, 3]), *tables, out, z, 3, n, 0.1, workspace(1, 3, 0, 3, n, 16, Hkv, D, dtype))
    plain.check_prompt(out, z, pc.attention(q, [back[0]], [back[1]], [3], [n], 0.1))
