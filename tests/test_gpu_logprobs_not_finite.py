"""The gradient of token log-probabilities in rows that are not finite."""
import math

import pytest
import torch

from paper_2510_26475_amd import binding
from test_gpu_logprobs import DT, make, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [5, 1000, 20011])
@pytest.mark.parametrize("shift", [0, 1])   # gradients that lie like their logits, and otherwise
def test_gradient_of_rows_that_are_not_finite_is_nan(dtype, V, shift):
    rows, T = 9, 0.6
    logits, tokens = make(rows, V, dtype, seed=V)
    tokens[6] = -1
    gen = torch.Generator(device="cuda").manual_seed(2)
    g, h = (torch.randn(rows, generator=gen, device="cuda") for _ in range(2))
    g[5] = 0.0

    def grads(x):
        _, lse, ent, _, _ = run(x, tokens, T)
        out = []
        for a, b in ((g, None), (None, h), (g, h)):
            wide = torch.full((rows, V + 16), 7.0, dtype=DT[dtype], device="cuda")
            binding.respec_token_logprobs_grad(x, tokens, lse, ent, a, b, wide[:, shift:shift + V], T)
            out.append(wide[:, shift:shift + V])
        return out

    clean = grads(logits)
    logits[1, V // 2], logits[3, V - 1], logits[4], logits[5, 0], logits[6, 0] = math.nan, math.inf, -math.inf, math.nan, math.nan
    bad = torch.zeros(rows, dtype=torch.bool, device="cuda")
    bad[[1, 3, 4, 5]] = True
    for got, want in zip(grads(logits), clean):
        assert torch.isnan(got[bad]).all() and torch.equal(got[~bad], want[~bad])
        assert (got[6] == 0).all()
