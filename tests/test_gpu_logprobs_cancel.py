"""Token log-probabilities at low temperatures and in nearly certain rows, where large numbers cancel."""
import math

import pytest
import torch

import plain
from test_gpu_logprobs import DT, check, make, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(3, 50257), (1100, 1500)])
@pytest.mark.parametrize("T", [0.4, 0.05, 1e-2, 1e-3, 1e-6, 1e-12])
def test_low_temperatures(dtype, rows, V, T):
    """The bounds of `check` hold whatever T is: differences of logits are exact or rounded once, and everything comes from them."""
    T = torch.tensor(T, dtype=torch.float32).item()
    logits, tokens = make(rows, V, dtype, seed=V)
    logits.clamp_(max=9.0)
    lead = (47.3 + 0.37 * torch.arange(rows, device="cuda") % 13).to(DT[dtype])
    at = torch.arange(rows, device="cuda") * 7919 % V
    logits[torch.arange(rows, device="cuda"), at] = lead
    tokens[::2] = at[::2].to(torch.int32)
    got = run(logits, tokens, T, 3)
    check(got, plain.token_logprobs(logits, tokens, T, 3), T)
    # the leading token: everybody else's share is below e^-95 or so, nothing in 32 bits
    assert (got[0][::2] == 0).all() and (got[4][:, 0] == 0).all() and (got[2].abs() <= 1e-30).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1.0, 0.6, 1e-2, 1e-4])
def test_close_logits_far_from_zero(dtype, T):
    """A few tokens share the probability, all of them at the same large logit: what differs is small beside what cancels."""
    T = torch.tensor(T, dtype=torch.float32).item()
    rows, V = 200, 3001
    logits, tokens = make(rows, V, dtype, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    base = (53.0 + 8 * torch.rand((rows, 1), generator=gen, device="cuda")).to(DT[dtype]).float()
    step = torch.maximum(T * torch.rand((rows, 12), generator=gen, device="cuda"), torch.tensor(0.0, device="cuda"))
    at = torch.randint(0, V, (rows, 12), generator=gen, device="cuda")
    logits.scatter_(1, at, (base - step * 3).to(DT[dtype]))
    tokens.copy_(at[:, 0])
    got = run(logits, tokens, T, 6)
    check(got, plain.token_logprobs(logits, tokens, T, 6), T)
    assert (got[0] <= 0).all() and (got[2] >= 0).all()


@pytest.mark.parametrize("V", [3, 40, 2000])
def test_entropy_of_nearly_certain_rows(V):
    """One token far ahead of a few: its lead grows over the range in which the reference may lie below the maximum."""
    rows = 640
    lead = torch.linspace(0.5, 30.0, rows, device="cuda")
    logits = torch.full((rows, V), -math.inf, device="cuda")
    logits[:, ::7] = torch.randn((rows, len(range(0, V, 7))), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda") * 0.1 + 3.3
    top = torch.arange(rows, device="cuda") * 31 % V
    logits[torch.arange(rows, device="cuda"), top] = 3.7 + lead
    tokens = top.to(torch.int32)
    got, ref = run(logits, tokens), plain.token_logprobs(logits, tokens, 1.0)
    check(got, ref, 1.0)
    assert (got[2] >= 0).all() and (got[0] <= 0).all()
