"""Sines and cosines of the rotation: accurate to a rounding of themselves, also next to their zeros."""
import math

import pytest
import torch

from paper_2510_26475_amd import binding
from plain_cache import ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("furthest", [1000, 1 << 20])
def test_next_to_the_zeros(interleaved, furthest):
    """Pairs (1, 0) become (cos t, sin t).  Bounds: two units of the function of the angle's leading part (2^-22 of the value), a rounding where the rest of the
    angle is added (2^-24), the square of that rest (below 2^-46) and the roundings of the angle in 64 bits (three of 2^-53 of it).  An angle rounded to 32 bits
    would be off by up to pi 2^-25, far more than that wherever a value is small."""
    n, D, rotary = 4096, 64, 64
    gen = torch.Generator(device="cuda").manual_seed(4)
    inv = torch.rand(rotary // 2, generator=gen, device="cuda") + 2.0 ** -10
    pos = torch.randint(0, furthest, (n,), generator=gen, device="cuda", dtype=torch.int32)
    k = torch.zeros((n, 1, D), device="cuda")
    a = slice(0, rotary, 2) if interleaved else slice(0, rotary // 2)
    b = slice(1, rotary, 2) if interleaved else slice(rotary // 2, rotary)
    k[:, 0, a] = 1.0
    pools = [torch.zeros((n // 16, 16, 1, D), device="cuda") for _ in range(2)]
    binding.respec_norm_rope_append_paged(None, k, k, None, None, inv, pos, None, *pools, None, None, ints([0, n]), ints([0, n // 16]), ints(list(range(n // 16))),
                                          ints([n]), n, 0.0, interleaved=interleaved)
    got = pools[0].view(n, D).cpu().double()
    t = pos.cpu().double()[:, None] * inv.cpu().double()
    near = 0
    for x, ref in ((got[:, a], t.cos()), (got[:, b], t.sin())):
        tol = ref.abs() * (2.0 ** -22 + 2.0 ** -24) + 2.0 ** -46 + 3 * 2.0 ** -53 * (t + 2 * math.pi)
        over = (x - ref).abs() - tol
        assert over.max() <= 0, f"{over.max():.3e} over its bound"
        near += (ref.abs() < 2.0 ** -6).sum().item()
    assert near > 1000
