"""Attention that is cut into parts where the channels of V differ widely: every channel of the output is as near as it is without a cut."""
import pytest
import torch

import plain
import plain_cache as pc
from plain_cache import Cache
from test_gpu_shared import BF16, F32, run
from test_gpu_shared_splits import knobs

pytestmark = pytest.mark.gpu


def spread_channels(c, pool, powers):
    """Channel d of V becomes |V| + 1/2 times 2^-powers[d] (positive: nothing cancels); 8 bits: of what the codes can hold."""
    factor = torch.ldexp(torch.ones(len(powers), dtype=torch.float64), -torch.tensor(powers)).cuda()
    if pool == "e4m3":
        v = pc.values(c.v.view(torch.uint8), c.v_scale.transpose(1, 2).contiguous())
        code, byte = pc.quantise((v.abs() + 0.5) * factor)
        keep = torch.isnan(v)
        c.v.view(torch.uint8).copy_(torch.where(keep, 0x7f, code))
        c.v_scale.copy_(byte.transpose(1, 2))
    else:
        c.v.copy_(((c.v.double().abs() + 0.5) * factor).to(c.v.dtype))


@pytest.mark.parametrize("dtype,pool,spread", [(BF16, "same", n) for n in (12, 16, 20, 24, 28, 30, 33, 60, 90)] + [(BF16, "e4m3", n) for n in (8, 12, 16, 17)]
                         + [(F32, "same", 60)])
@pytest.mark.parametrize("grouped", [False, True])
@pytest.mark.parametrize("D,R", [(64, [4, 3, 4]), (128, [2, 9, 1])])
def test_channels_of_very_different_sizes(dtype, pool, spread, grouped, D, R):
    """Powers from 0 to `spread` along the channels, and one channel of 1 among those of 2^-spread.  A part rounds each of its numbers once more than the bound of
    the uncut attention counts: by 2^-11 of it, or, where a row's numbers lie 2^29 apart, by 2^-8."""
    groups, shared = ([[0, 1]], [1024]) if grouped else ((), ())
    for powers in ([spread * d // (D - 1) for d in range(D)], [0 if d == 5 else spread for d in range(D)]):
        c = Cache([2100, 1500, 700], 2, D, 16, dtype, groups, shared, pool, seed=41)
        spread_channels(c, pool, powers)
        for cut in ({}, {"RANGES": 5}):
            with knobs(**cut):
                q, out, z = run(c, R, 8, dtype, groups, shared)
            k, v = c.both()
            o, lse, tol, lse_tol = pc.attention(q, k, v, R, c.lens, D ** -0.5)
            size = pc.attention(q, k, [x.abs() for x in v], R, c.lens, D ** -0.5)[0]
            part = 0.0 if dtype == F32 else 2.0 ** -8 if spread > 24 else 2.0 ** -11
            plain.check_prompt(out, z, (o, lse, tol + part * 1.01 * size, lse_tol))


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("grouped", [False, True])
@pytest.mark.parametrize("D,R", [(64, [4, 3, 4]), (128, [2, 9, 1])])
def test_values_that_are_not_finite_among_such_channels(bad, grouped, D, R):
    """In a tile that some row does not see whole: they reach the rows that see their key, in their channel alone."""
    groups, shared = ([[0, 1]], [1024]) if grouped else ((), ())
    powers = [60 * d // (D - 1) for d in range(D)]
    for channel in (0, 31, D - 1):
        c = Cache([2100, 1500, 700], 2, D, 16, BF16, groups, shared, seed=42)
        spread_channels(c, "same", powers)
        clean = c.both()[1]
        for b, n in enumerate(c.lens):
            c.v[c.pages[b][(n - 2) // 16], (n - 2) % 16, 1, channel] = bad
            clean[b][n - 2, 1, channel] = 0.0
        q, out, z = run(c, R, 8, BF16, groups, shared)
        k = c.both()[0]
        o, lse, tol, lse_tol = pc.attention(q, k, clean, R, c.lens, D ** -0.5)
        size = pc.attention(q, k, [x.abs() for x in clean], R, c.lens, D ** -0.5)[0]
        at, hit = 0, torch.zeros(out.shape, dtype=torch.bool, device="cuda")
        for r in R:
            hit[max(at, at + r - 2):at + r, 4:, channel] = True   # (the last two rows see the last key but one)
            at += r
        got = out[hit].float()
        assert torch.isnan(got).all() if bad != bad else (got == bad).all()
        plain.check_prompt(torch.where(hit, o, out.double()), z, (o, lse, tol + 2.0 ** -8 * 1.01 * size, lse_tol))
