"""Token log-probabilities, entropies, alternatives and their gradient on the GPU against a plain implementation in 64 bits."""
import math

import pytest
import torch

import plain
from paper_2510_26475_amd import binding

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def make(rows, V, dtype, seed=1, sigma=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    logits = (sigma * torch.randn((rows, V), generator=g, device="cuda")).to(DT[dtype])
    tokens = torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=torch.int32)
    return logits, tokens


def run(logits, tokens, T=1.0, top=0, entropy=True, row_T=None):
    rows, V = logits.shape
    f = dict(dtype=torch.float32, device="cuda")
    lp, lse, ent = (torch.full((rows,), 77.0, **f) for _ in range(3))
    ids = torch.full((rows, top), -7, dtype=torch.int32, device="cuda") if top else None
    best = torch.full((rows, top), 77.0, **f) if top else None
    ws = torch.full((binding.respec_token_logprobs_workspace_bytes(rows, V, top, int(logits.dtype == torch.bfloat16)),), 0xff,
                    dtype=torch.uint8, device="cuda")
    binding.respec_token_logprobs(logits, tokens, lp, lse, ent if entropy else None, ids, best, T, ws, row_temperature=row_T)
    torch.cuda.synchronize()
    return lp, lse, ent, ids, best


def check(got, ref, T):
    """Per element an exponent (x - m)/T has two roundings of its size, e^... one step more; sums of up to 600 terms per thread add
    half a step per term at most (their errors are of both signs: far less), a dozen joins one each.  So 1e-5 of e.g. ln s
    absolutely, and the roundings of lse and logprob themselves."""
    for a, b in zip(got[:3], ref[:3]):
        nan = torch.isnan(b)
        assert torch.equal(torch.isnan(a), nan)
        inf = torch.isinf(b)
        assert torch.equal(a[inf].double(), b[inf])
        ok = ~(nan | inf)
        err = (a.double() - b).abs()[ok] - (2e-5 + 2.0 ** -22 * b.abs()[ok])
        assert err.numel() == 0 or err.max() <= 0, err.max()
    if got[3] is not None:
        assert torch.equal(got[3].long(), ref[3])
        a, b = got[4].double(), ref[4]
        inf = torch.isinf(b)
        assert torch.equal(a[inf], b[inf])
        err = (a - b).abs()[~inf] - (2e-5 + 2.0 ** -22 * b.abs()[~inf])
        assert err.numel() == 0 or err.max() <= 0, err.max()


@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 63, 1000, 2048, 2049, 32000, 50257, 151936])
@pytest.mark.parametrize("rows", [1, 3, 70])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_all_sizes(dtype, rows, V):
    logits, tokens = make(rows, V, dtype, seed=V + rows)
    tokens[rows // 2] = V - 1
    for T, top in ((1.0, 5), (0.4, 0)):
        check(run(logits, tokens, T, top), plain.token_logprobs(logits, tokens, T, top), T)


@pytest.mark.parametrize("rows,V", [(2, 151936), (600, 4000), (1500, 997)])
@pytest.mark.parametrize("top", [1, 20, 33, 64])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_alternatives(dtype, rows, V, top):
    logits, tokens = make(rows, V, dtype, seed=top)
    check(run(logits, tokens, 0.6, top), plain.token_logprobs(logits, tokens, 0.6, top), 0.6)


@pytest.mark.parametrize("rows,V", [(1, 20000), (1200, 1500)])
@pytest.mark.parametrize("kind", ["ascending", "descending", "constant", "few values", "signed zeros"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_orders_and_ties(dtype, rows, V, kind):
    """Ties go to the lowest token id, whatever order the row comes in."""
    x = torch.arange(V, device="cuda").float()
    row = {"ascending": x / 1000, "descending": -x / 1000, "constant": torch.full_like(x, 2.5), "few values": x * 7 % 5,
           "signed zeros": torch.where(x % 2 == 0, -0.0, 0.0)}[kind]
    logits = row.to(DT[dtype]).expand(rows, V).contiguous()
    tokens = torch.arange(rows, device="cuda", dtype=torch.int32) % V
    for top in (3, 64):
        check(run(logits, tokens, 1.0, top), plain.token_logprobs(logits, tokens, 1.0, top), 1.0)


def test_fewer_logits_than_alternatives():
    logits, tokens = make(4, 5, "f32")
    got = run(logits, tokens, 1.0, 12)
    check(got, plain.token_logprobs(logits, tokens, 1.0, 12), 1.0)
    assert (got[3][:, 5:] == -1).all() and (got[4][:, 5:] == -math.inf).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(3, 40000), (1100, 3000)])
@pytest.mark.parametrize("fill", ["-inf", "lowest"])
def test_masked_logits(dtype, rows, V, fill):
    """-inf or the type's lowest value in most places, in whole stretches, everywhere but one, everywhere (row 1)."""
    x, tokens = make(rows, V, dtype, seed=4)
    fill = -math.inf if fill == "-inf" else torch.finfo(DT[dtype]).min
    g = torch.Generator(device="cuda").manual_seed(5)
    x[torch.rand((rows, V), generator=g, device="cuda") < 0.999] = fill
    x[:, 17] = 1.0
    x[0], x[0, V - 1] = fill, 0.5
    x[1] = fill
    x[2, 100:] = fill
    tokens[2] = 17
    rest = torch.arange(rows, device="cuda") != 1
    for top in (0, 30):
        got, ref = run(x, tokens, 0.6, top), plain.token_logprobs(x, tokens, 0.6, top)
        if top:
            assert torch.equal(got[3].long(), ref[3])
        if math.isinf(fill):
            assert math.isnan(got[0][1].item()) and math.isnan(got[2][1].item()) and got[1][1].item() == -math.inf
        else:  # all equal, whatever they are
            assert abs(got[0][1].item() + math.log(V)) < 2e-5 and abs(got[2][1].item() - math.log(V)) < 2e-5
        # (a lowest value over T is past the range of float32: -inf)
        check([None if t is None else t[rest] for t in got], [t[rest].float().double() if t.is_floating_point() else t[rest] for t in ref], 0.6)


def test_nan_and_infinity_in_a_row_are_nan_of_that_row_only():
    logits, tokens = make(5, 30000, "f32")
    clean = run(logits, tokens, 1.0, 4)
    logits[1, 777], logits[3, 29999] = math.nan, math.inf
    got = run(logits, tokens, 1.0, 4)
    for a, b in zip(got[:3], clean[:3]):
        assert torch.isnan(a[[1, 3]]).all() and torch.equal(a[[0, 2, 4]], b[[0, 2, 4]])


def test_unused_rows_are_not_read():
    for rows in (6, 1200):
        logits, tokens = make(rows, 9000, "bf16")
        want = run(logits, tokens, 1.0, 3)
        tokens[1], tokens[4] = -1, 9000
        logits[1] = logits[4] = math.nan
        got = run(logits, tokens, 1.0, 3)
        for a, b in zip(got, want):
            keep = torch.ones(rows, dtype=torch.bool, device="cuda")
            keep[1] = keep[4] = False
            assert torch.equal(a[keep], b[keep])
            assert (a[~keep] == (-1 if a.dtype == torch.int32 else 0)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [1, 3, 5])
def test_rows_that_start_anywhere(dtype, shift):
    """Slices of a wider tensor: every row begins at another place of a 16-byte piece, and what lies around it is NaN."""
    for rows, V in ((9, 5003), (1100, 513)):
        wide = torch.full((rows, V + 17), math.nan, dtype=DT[dtype], device="cuda")
        logits, tokens = make(rows, V, dtype, seed=shift)
        wide[:, shift:shift + V] = logits
        got, want = run(wide[:, shift:shift + V], tokens, 0.6, 6), plain.token_logprobs(logits, tokens, 0.6, 6)
        check(got, want, 0.6)
        _, lse, ent, _, _ = got
        g, h = torch.randn(rows, device="cuda"), torch.randn(rows, device="cuda")
        out = torch.full((rows, V + 9), 7.0, dtype=DT[dtype], device="cuda")
        for at in (shift % 4, 2):
            out.fill_(7.0)
            binding.respec_token_logprobs_grad(wide[:, shift:shift + V], tokens, lse, ent, g, h, out[:, at:at + V], 0.6)
            check_grad(out[:, at:at + V], logits, tokens, g, h, 0.6)
            assert (out[:, :at] == 7).all() and (out[:, at + V:] == 7).all()


def test_temperatures_per_row():
    logits, tokens = make(40, 3000, "f32")
    T = torch.linspace(0.3, 2.0, 40, device="cuda")
    check(run(logits, tokens, 0.0, 4, row_T=T), plain.token_logprobs(logits, tokens, T.double(), 4), T)
    for bad in (0.0, -1.0, math.nan, math.inf):
        T2 = T.clone()
        T2[7] = bad
        got, want = run(logits, tokens, 1.0, 4, row_T=T2), run(logits, tokens, 1.0, 4, row_T=T)
        for a, b in zip(got[:3], want[:3]):
            assert torch.isnan(a[7]) and torch.equal(a[:7], b[:7]) and torch.equal(a[8:], b[8:])


def check_grad(got, logits, tokens, g, h, T):
    """The result is a difference of terms, so its error is that of the terms and not of what is left of them (with V = 1 nothing is).
    p = e^(z - lse): lse carries two roundings and its sums' 2e-6, |lse| <= 50 here, so z - lse is off by 2 * 50 * 2^-24 + 2e-6
    < 1e-5, and p by that share; log p + H by 1e-5 for either part.  With a step for each further product:
    p (1e-5 (|g| + |h| |log p + H|) + 2e-5 |h|) / T, four roundings of the terms, and the rounding of the result."""
    ref = plain.logprob_grad(logits, tokens, T, g, h)
    z = logits.double() / T
    log_p = z - torch.logsumexp(z, dim=1, keepdim=True)
    p = log_p.exp()
    log_p = torch.where(p > 0, log_p, 0.0)
    part = (log_p - (p * log_p).sum(dim=1, keepdim=True)).abs()
    g, h = g.abs()[:, None].double(), h.abs()[:, None].double()
    term = g + h * part
    hit = torch.zeros_like(p).scatter_(1, tokens.long().clamp(0, logits.shape[1] - 1)[:, None], 1.0)
    tol = (p * (1e-5 * term + 2e-5 * h) + 4 * 2.0 ** -24 * (p * term + hit * g)) / T + plain.HALF_STEP[got.dtype] * 1.01 * ref.abs() + 1e-37
    assert torch.isfinite(got).all()
    over = (got.double() - ref).abs() - tol
    assert over.max() <= 0, over.max()


@pytest.mark.parametrize("V", [1, 7, 8, 1000, 50257])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradient(dtype, V):
    rows = 37
    logits, tokens = make(rows, V, dtype, seed=V)
    tokens[5] = -1
    gen = torch.Generator(device="cuda").manual_seed(3)
    g, h = (torch.randn(rows, generator=gen, device="cuda") for _ in range(2))
    for T in (1.0, 0.4):
        _, lse, ent, _, _ = run(logits, tokens, T)
        for use_g, use_h in ((g, h), (g, None), (None, h)):
            grad = torch.full_like(logits, 7.0)
            binding.respec_token_logprobs_grad(logits, tokens, lse, ent, use_g, use_h, grad, T)
            zero = torch.zeros_like(g)
            a, b = use_g if use_g is not None else zero, use_h if use_h is not None else zero
            check_grad(grad, logits, tokens, a, b, T)
            assert (grad[5] == 0).all()
        over = logits.clone()   # over its own logits
        binding.respec_token_logprobs_grad(over, tokens, lse, ent, g, h, over, T)
        full = torch.empty_like(logits)
        binding.respec_token_logprobs_grad(logits, tokens, lse, ent, g, h, full, T)
        assert torch.equal(over, full)


def test_gradient_against_differences():
    """Central differences of the loss in 64 bits: their error is h^2/6 of its third derivative (below 1 here)."""
    rows, V, T, step = 4, 23, 0.7, 1e-4
    logits, tokens = make(rows, V, "f32", sigma=1.0)
    g, h = torch.randn(rows, device="cuda").double(), torch.randn(rows, device="cuda").double()

    def loss(z):
        lp, _, ent, _, _ = plain.token_logprobs(z, tokens, T)
        return g * lp + h * ent

    z = logits.double()
    diff = torch.empty_like(z)
    for x in range(V):
        e = torch.zeros_like(z)
        e[:, x] = step
        diff[:, x] = (loss(z + e) - loss(z - e)) / (2 * step)
    _, lse, ent, _, _ = run(logits, tokens, T)
    grad = torch.empty_like(logits)
    binding.respec_token_logprobs_grad(logits, tokens, lse, ent, g.float(), h.float(), grad, T)
    assert (grad.double() - diff).abs().max() <= 2e-5


def test_gradient_of_masked_tokens_is_zero():
    logits, tokens = make(8, 4000, "bf16")
    logits[:, 1000:] = -math.inf
    tokens %= 1000
    _, lse, ent, _, _ = run(logits, tokens, 1.0)
    g, h = torch.ones(8, device="cuda"), torch.ones(8, device="cuda")
    grad = torch.empty_like(logits)
    binding.respec_token_logprobs_grad(logits, tokens, lse, ent, g, h, grad, 1.0)
    assert (grad[:, 1000:] == 0).all()
    check_grad(grad, logits, tokens, g, h, 1.0)


def test_repeats_and_captured_calls_give_the_same_bits():
    for rows in (4, 1500):
        logits, tokens = make(rows, 20011, "bf16")
        want = run(logits, tokens, 0.6, 8)
        lp, lse, ent = (torch.empty(rows, device="cuda") for _ in range(3))
        ids, best = torch.empty((rows, 8), dtype=torch.int32, device="cuda"), torch.empty((rows, 8), device="cuda")
        grad = torch.empty_like(logits)
        ws = torch.empty(binding.respec_token_logprobs_workspace_bytes(rows, 20011, 8, 1), dtype=torch.uint8, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            binding.respec_token_logprobs(logits, tokens, lp, lse, ent, ids, best, 0.6, ws)
            binding.respec_token_logprobs_grad(logits, tokens, lse, ent, lp, ent, grad, 0.6)
        first = None
        for _ in range(3):
            for t in (lp, lse, ent, ids, best, grad):
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip((lp, lse, ent, ids, best), want):
                assert torch.equal(a, b)
            first = grad.clone() if first is None else first
            assert torch.equal(grad, first)
            run(logits, tokens, 0.6, 8)


def test_offsets_past_32_bits():
    rows, V = 2, 40001
    ld = (1 << 31) + 8
    base = torch.empty(ld + V, dtype=torch.bfloat16, device="cuda")
    logits = base.as_strided((rows, V), (ld, 1))
    x, tokens = make(rows, V, "bf16")
    logits.copy_(x)
    got = run(logits, tokens, 1.0, 4)
    check(got, plain.token_logprobs(x, tokens, 1.0, 4), 1.0)
    g = torch.ones(rows, device="cuda")
    binding.respec_token_logprobs_grad(logits, tokens, got[1], got[2], g, g, logits, 1.0)
    check_grad(logits, x, tokens, g, g, 1.0)
