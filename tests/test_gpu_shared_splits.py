"""The attention over shared pages under every cut of its work: few ranges and many, all work-groups on one kind of work, waves that share the tiles of many
columns.  Against float64; what one cut gives again and again has the same bits."""
import math
from contextlib import ExitStack, contextmanager

import pytest
import torch

import plain
import plain_cache as pc
from helpers import env_setting
from plain_cache import Cache
from test_gpu_shared import BF16, POOLS, check, run

pytestmark = pytest.mark.gpu


@contextmanager
def knobs(**values):
    with ExitStack() as stack:
        for name, value in values.items():
            stack.enter_context(env_setting(f"RESPEC_SHARED_{name}", value))
        yield


@pytest.mark.parametrize("dtype,pool", POOLS)
@pytest.mark.parametrize("cut", [dict(RANGES=1), dict(RANGES=2), dict(RANGES=7), dict(RANGES=100), dict(TILES=1), dict(TILES=40), dict(COST=1), dict(COST=100000)],
                         ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
@pytest.mark.parametrize("R", [3, 11])
def test_cuts(dtype, pool, cut, R):
    """Eight columns to a KV head and, of 44, two waves of them: sequences of a group, by themselves, without rows, without tokens."""
    groups, shared = [[0, 1, 2], [3], [4, 5]], [640, 0, 64]         # (what lies between two groups is a group too: of one)
    lens = [640 + R, 700 + R, 1100, 300 + R, 70 + R, 200, 0, R, 90]
    rows = [R, R, R - 1, R, R, 1, 2, R, 0]
    c = Cache(lens, 2, 64, 16, dtype, groups, shared, pool, seed=31)
    with knobs(**cut):
        q, out, z = run(c, rows, 8, dtype, groups, shared)
        again = run(c, rows, 8, dtype, groups, shared, q=q)
    plain.check_prompt(out, z, pc.attention(q, *c.both(), rows, lens, 1 / 8))
    assert torch.equal(again[1], out) and torch.equal(again[2], z)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,R", [(8, 2, 9), (8, 2, 16), (8, 2, 17), (4, 1, 12), (6, 3, 20), (4, 1, 60)])
def test_waves_that_share_tiles(D, Hq, Hkv, R):
    """8 bits: two and four waves to a KV head, ranges that go through many sequences and through parts of a long one."""
    lens = [(53 * i) % 170 + R for i in range(60)] + [5000, R, R + 31, R + 32]
    rows = [(R - i % 3) for i in range(60)] + [R] * 4
    check(Cache(lens, Hkv, D, 16, BF16, pool="e4m3", seed=32), rows, Hq, BF16)
    with knobs(RANGES=3):
        check(Cache(lens[:20] + lens[60:], Hkv, D, 32, BF16, pool="e4m3", seed=33), rows[:20] + rows[60:], Hq, BF16)


@pytest.mark.parametrize("dtype,pool", POOLS)
@pytest.mark.parametrize("ranges", [1, 64])
def test_values_that_are_not_finite_where_waves_share_tiles(dtype, pool, ranges):
    """NaN in V reaches the rows that see its key, of every column wave, and no others; the sequences around it are whole."""
    R, Hq, Hkv, D, page = 10, 8, 2, 64, 16
    groups, shared = [[0, 1]], [75]
    for where in (64, 74, 75, 90, 99, 108, 109):
        c = Cache([110, 120, 150, 40], Hkv, D, page, dtype, groups, [80], pool, seed=34)
        for b in (0, 2):
            place = c.pages[b][where // page], where % page
            if pool == "e4m3":
                c.v.view(torch.uint8)[place[0], place[1], 1, 5] = 0xff
            else:
                c.v[place[0], place[1], 1, 5] = math.nan
        with knobs(RANGES=ranges):
            q, out, z = run(c, [R] * 4, Hq, dtype, groups, shared)
        k, v = c.both()
        hit = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
        for b in range(3):
            seen = torch.isnan(v[b][:, 1, 5]).nonzero().flatten().tolist()
            for n in seen:
                for i in range(R):
                    if n <= c.lens[b] - R + i:
                        hit[R * b + i, 4:, 5] = True
        assert hit.any()
        assert torch.isnan(out[hit]).all(), where
        ref = pc.attention(q, k, [torch.nan_to_num(x, nan=0.0) for x in v], [R] * 4, c.lens, 1 / 8)
        plain.check_prompt(torch.where(hit, ref[0], out.double()), z, ref)


def test_groups_of_many_and_many_groups():
    """A group of 300 sequences, and 300 groups of two: a plan in LDS and one in memory."""
    lens = [64 + 5 + i % 40 for i in range(300)] + [20 + i % 7 for i in range(700)]
    for groups, shared in (([list(range(300))], [64]), ([[2 * i, 2 * i + 1] for i in range(300)], [48] * 150 + [16] * 150)):
        c = Cache(lens, 1, 64, 16, BF16, groups, shared, seed=35)
        check(c, [1 + i % 4 for i in range(1000)], 4, BF16, groups, shared)


@pytest.mark.parametrize("dtype,pool", POOLS)
@pytest.mark.parametrize("power", [110, 60, -60])
@pytest.mark.parametrize("grouped", [False, True])
def test_parts_of_very_different_sizes(dtype, pool, power, grouped):
    """Values of V of 2^110 (2^60, 2^-60) in one half of the keys and of 1 in the other: each part's sum counts for all."""
    groups, shared = ([[0, 1]], [1024]) if grouped else ((), ())
    c = Cache([2100, 1500, 700], 2, 64, 16, dtype, groups, shared, pool, seed=36)
    for b, first, end in ((0, 0, 64), (1, 0, 64), (2, 20, 40)):
        for page in set(c.pages[b][first:end]) - (set(c.pages[0][:64]) if grouped and b == 1 else set()):
            if pool == "e4m3":
                c.v_scale[page] = (c.v_scale[page].int() + power).clamp(1, 247).to(torch.uint8)
            else:
                c.v[page] = torch.where(torch.isnan(c.v[page]), c.v[page], c.v[page] * 2.0 ** power)
    check(c, [4, 3, 4], 8, dtype, groups, shared)
