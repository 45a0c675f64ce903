"""Offsets, groups and lengths of the attention over shared pages that mean nothing: the call stays inside its buffers, and what does not depend on them is as it was.
And shared lengths far past what the members hold."""
import math

import pytest
import torch

import plain
import plain_cache as pc
from paper_2510_26475_amd import binding
from plain_cache import Cache, ints, offsets
from test_gpu_shared import POOLS, run, workspace

pytestmark = pytest.mark.gpu
GUARD = 4  # rows before and behind, and bytes of the workspace in units of 256


def guarded(c, q, q_indptr, group_indptr, shared_len, total, tables=None):
    """A call whose outputs and workspace lie between guard rows; returns out and lse, 5 where nothing was written."""
    Hq, D = q.shape[1:]
    out = torch.full((total + 2 * GUARD, Hq, D), 5.0, dtype=q.dtype, device="cuda")
    lse = torch.full((total + 2 * GUARD, Hq), 5.0, device="cuda")
    n = workspace(len(c.lens), total, len(shared_len), 2, 80, Hq, c.Hkv, D, q.dtype).numel()
    ws = torch.full((n + 512 * GUARD,), 0xa5, dtype=torch.uint8, device="cuda")
    inner = ws[256 * GUARD:256 * GUARD + n]
    assert inner.data_ptr() % 256 == 0
    binding.respec_verify_attention_shared(q, *c.args(), q_indptr, *(tables or c.tables()), ints(group_indptr) if shared_len else None,
                                           ints(shared_len) if shared_len else None, None, out[GUARD:-GUARD], lse[GUARD:-GUARD], 2, 80, 1 / 8, inner)
    torch.cuda.synchronize()
    for x in (out, lse):
        assert (x[:GUARD] == 5.0).all() and (x[-GUARD:] == 5.0).all()
    assert (ws[:256 * GUARD] == 0xa5).all() and (ws[256 * GUARD + n:] == 0xa5).all()
    return out[GUARD:-GUARD], lse[GUARD:-GUARD]


@pytest.mark.parametrize("dtype,pool", POOLS)
def test_groups_that_mean_nothing(dtype, pool):
    """Offsets of groups past the batch, below zero, decreasing.  The members of what could be read as a group hold the same tokens, so that whatever the call takes
    for a group every row has one right result."""
    R, Hq, page = [2, 2, 2, 2], 4, 16
    everyone = [[0, 1, 2, 3]]
    c = Cache([66, 70, 80, 75], 2, 64, page, dtype, everyone, [64], pool, seed=16)
    q = torch.randn((8, Hq, 64), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(dtype)
    ref = pc.attention(q, *c.both(), R, c.lens, 1 / 8)
    for gi, sl in (([0, 4], [64]), ([0, 2, 1, 4], [10, 20, 30]), ([-5, 90, 2, 3], [50, 50, 50]), ([3, 2, 1, 0], [5, 5, 5]), ([0, 4, 4, 4], [-1, 9, 9]),
                   ([-2 ** 31, 2 ** 31 - 1], [64]), ([2 ** 31 - 1, -2 ** 31, 7], [64, 64]), ([1, 1, 1], [64, 64])):
        plain.check_prompt(*guarded(c, q, offsets(R), gi, sl, 8), ref)


@pytest.mark.parametrize("dtype,pool", POOLS)
@pytest.mark.parametrize("grouped", [False, True])
def test_rows_that_mean_nothing(dtype, pool, grouped):
    """Offsets of rows past the end, below zero, decreasing: rows of sequences whose offsets are sound are right, and rows of no sequence are left as they were."""
    Hq = 4
    groups, shared = ([[0, 1, 2]], [48]) if grouped else ((), ())
    c = Cache([60, 70, 80, 50], 2, 64, 16, dtype, groups, shared, pool, seed=16)
    q = torch.randn((8, Hq, 64), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").to(dtype)
    k, v = c.both()
    cases = [([0, 2, 4, 6, 10 ** 6], {0, 1, 2, 3}, {}),             # (the last sequence: two rows are there)
             ([-9, -2, 4, 6, 8], {2, 3}, {}),                      # (the first: no rows; the second: of rows below zero)
             ([0, 5, 3, 7, 8], {3}, {}),
             ([2, 4, 4, 6, 6], {0, 1, 2, 3}, {0, 1, 6, 7})]
    for indptr, sound, nobody in cases:
        # (a group's rows are those between its first and its last member's: groups only where these are sound)
        g = grouped and {0, 1, 2} <= sound
        out, lse = guarded(c, q, ints(indptr), [0, 3] if g else [], shared if g else [], 8)
        for b in sound:
            a, z = indptr[b], min(indptr[b + 1], 8)
            if z > a:
                ref = pc.attention(q[a:z], [k[b]], [v[b]], [z - a], [c.lens[b]], 1 / 8)
                plain.check_prompt(out[a:z], lse[a:z], ref)
        for i in nobody:
            assert (out[i] == 5.0).all() and (lse[i] == 5.0).all()
    for indptr in ([0, 5, 3, 9, 8], [-9, -2, 4, 6, 8], [8, 6, 4, 2, 0], [-2 ** 31, 2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1, 0]):
        guarded(c, q, ints(indptr), [0, 2, 4, 4], [40, 40, 40], 8)


@pytest.mark.parametrize("dtype,pool", POOLS)
def test_lengths_and_pages_that_mean_nothing(dtype, pool):
    """A length past the pages, below zero, page ids that do not exist: the other sequences' rows are right."""
    R, Hq = [2, 2, 2, 2], 4
    c = Cache([60, 70, 80, 50], 2, 64, 16, dtype, pool=pool, seed=16)
    q = torch.randn((8, Hq, 64), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(dtype)
    ref = pc.attention(q, *c.both(), R, c.lens, 1 / 8)
    out, lse = guarded(c, q, offsets(R), [], [], 8)
    plain.check_prompt(out, lse, ref)
    for i, (length, page_id) in enumerate(((10 ** 9, 2 ** 31 - 1), (-7, -1), (2 ** 31 - 1, -2 ** 31), (-2 ** 31, 10 ** 6))):
        b = i % 4
        kv_len, table = c.kv_len.clone(), c.page_table.clone()
        kv_len[b] = length
        other = (b + 1) % 4
        table[c.page_indptr[other]] = page_id
        got, z = guarded(c, q, offsets(R), [], [], 8, (c.page_indptr, table, kv_len))
        keep = [r for s in range(4) if s not in (b, other) for r in (2 * s, 2 * s + 1)]
        o, zr, tol, z_tol = (x[keep] for x in ref)
        plain.check_prompt(got[keep], z[keep], (o, zr, tol, z_tol))


@pytest.mark.parametrize("dtype,pool", POOLS)
@pytest.mark.parametrize("page", [16, 64])
def test_shared_lengths_past_what_the_members_hold(dtype, pool, page):
    """The members hold the same tokens up to where the first of their rows begins, in pages of their own behind the whole shared ones: any length from there on, to
    the end of 31 bits, counts as that."""
    Hq, Hkv, D = 8, 2, 64
    groups, R = [[0, 1, 2], [3, 4]], [3, 2, 4, 1, 2, 3]
    lens = [101, 160, 131, 70, 66, 90]
    same = [min(lens[b] - R[b] for b in g) for g in groups]       # 98 and 64
    c = Cache(lens, Hkv, D, page, dtype, groups, same, pool, seed=18)
    for g, n in zip(groups, same):
        for b in g[1:]:
            for i in range(n // page, -(-n // page)):
                src, dst, many = c.pages[g[0]][i], c.pages[b][i], n - i * page
                for x in (c.k, c.v):
                    x.view(torch.uint8)[dst, :many] = x.view(torch.uint8)[src, :many].clone()
                if c.k_scale is not None:
                    for s in (c.k_scale, c.v_scale):
                        s[dst, :, :many] = s[src, :, :many].clone()
    k, v = c.both()
    for g, n in zip(groups, same):
        for b in g[1:]:
            assert torch.equal(k[b][:n], k[g[0]][:n]) and torch.equal(v[b][:n], v[g[0]][:n])
            assert not torch.equal(v[b][n:n + 1], v[g[0]][n:n + 1])
    want = None
    for shared in (same, [n + 1 for n in same], [1000, 200], [2 ** 31 - 1, 2 ** 31 - 1]):
        q, out, z = run(c, R, Hq, dtype, groups, shared)
        plain.check_prompt(out, z, pc.attention(q, k, v, R, lens, 1 / math.sqrt(D)))
        want = want if want is not None else out
        assert torch.equal(out, want)                             # (the same limit, the same cut)
