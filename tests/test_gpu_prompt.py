"""Attention over whole prompts on the GPU against a plain implementation in 64 bits: packed and paged, chunks, odd lengths, rows that
see nothing, strides, values that are not finite, splits, captured calls, offsets past 32 bits."""
import math

import pytest
import torch

import plain
from helpers import env_setting
from paper_2510_26475_amd import binding

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
RAGGED = [(1, 1), (33, 33), (0, 0), (64, 64), (65, 130), (17, 300), (128, 128), (5, 2), (0, 40), (3, 0), (129, 129), (31, 1000), (200, 200)]


def randn(*shape, dt, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dt)


def offsets(n, dt):
    return torch.tensor([0] + list(n), device="cuda").cumsum(0).to(dt)


def workspace(B, total_q, total_kv, max_q, max_kv, heads, dt):
    n = binding.respec_prompt_attention_workspace_bytes(B, total_q, total_kv, max_q, max_kv, *heads, int(dt == torch.bfloat16))
    assert n > 0
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def run(q, k, v, R, L, scale, lse=True, spare_rows=0):
    """k, v [sum L (+ more), Hkv, D] packed.  Rows of out behind the last sequence have to stay."""
    Hq, D = q.shape[1:]
    out = torch.full((q.shape[0], Hq, D), 7.0, dtype=q.dtype, device="cuda")
    z = torch.full((q.shape[0], Hq), 7.0, device="cuda") if lse else None
    ws = workspace(len(R), q.shape[0], k.shape[0], max(max(R), 1), max(max(L), 1), (Hq, k.shape[1], D), q.dtype)
    ws.fill_(0xff)  # (NaN: nothing that was not written may be read)
    binding.respec_prompt_attention(q, k, v, offsets(R, torch.int32), offsets(L, torch.int64), out, z, max(max(R), 1), max(max(L), 1),
                                    scale, ws)
    torch.cuda.synchronize()
    n = sum(R)
    assert (out[n:] == 7).all() and (z is None or (z[n:] == 7).all())
    return out[:n], None if z is None else z[:n]


def split_keys(k, L):
    return list(torch.split(k[:sum(L)], L))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads", [(4, 1, 64), (28, 4, 128), (8, 8, 64), (6, 2, 128)], ids=str)
def test_ragged_batch(dtype, heads):
    Hq, Hkv, D = heads
    R, L = [r for r, _ in RAGGED], [n for _, n in RAGGED]
    q = randn(sum(R) + 5, Hq, D, dt=DT[dtype], seed=1)
    kv = randn(sum(L) + 3, 2 * Hkv, D, dt=DT[dtype], seed=2)
    kv[sum(L):] = math.nan
    k, v = kv[:, :Hkv], kv[:, Hkv:]
    out, lse = run(q, k, v, R, L, D ** -0.5)
    plain.check_prompt(out, lse, plain.prompt_attention(q[:sum(R)], split_keys(k, L), split_keys(v, L), R, L, D ** -0.5))


@pytest.mark.parametrize("n", [1, 2, 31, 32, 63, 64, 65, 96, 127, 128, 129, 255, 257])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_lengths_around_the_tiles(dtype, n):
    q, k, v = (randn(n, h, 64, dt=DT[dtype], seed=n + h) for h in (3, 1, 1))
    v = randn(n, 1, 64, dt=DT[dtype], seed=n + 9)
    out, lse = run(q, k, v, [n], [n], 0.125)
    plain.check_prompt(out, lse, plain.prompt_attention(q, [k], [v], [n], [n], 0.125))


@pytest.mark.parametrize("scale", [-0.2, 0.0, 1.0, 3.0])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scales(dtype, scale):
    q, k, v = (randn(150, h, 64, dt=DT[dtype], seed=h) for h in (4, 2, 2))
    out, lse = run(q, k, v, [150], [150], scale)
    plain.check_prompt(out, lse, plain.prompt_attention(q, [k], [v], [150], [150], scale))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rising_scores_move_the_reference(dtype):
    """Every key scores higher than the one before it, over a range that an exponential from the first one would overflow."""
    n = 700
    q = torch.ones((n, 2, 64), dtype=DT[dtype], device="cuda")
    k = (torch.arange(n, device="cuda") * (240.0 / n / 64))[:, None, None].expand(n, 1, 64).to(DT[dtype]).contiguous()
    v = randn(n, 1, 64, dt=DT[dtype], seed=3)
    out, lse = run(q, k, v, [n], [n], 1.0)
    plain.check_prompt(out, lse, plain.prompt_attention(q, [k], [v], [n], [n], 1.0))


@pytest.mark.parametrize("dtype,R,L,heads", [("bf16", [40], [9001], (28, 4, 128)), ("bf16", [1], [5000], (4, 1, 64)),
                                             ("f32", [3, 50], [4097, 2100], (4, 1, 64)), ("bf16", [100, 0, 20], [100, 70, 6000], (16, 2, 128)),
                                             ("bf16", [700, 10], [700, 5], (16, 2, 128)), ("f32", [9], [3000], (4, 2, 128))], ids=str)
def test_few_rows_split_the_keys(dtype, R, L, heads):
    Hq, Hkv, D = heads
    q, k, v = (randn(n, h, D, dt=DT[dtype], seed=h + n) for n, h in ((sum(R), Hq), (sum(L), Hkv), (sum(L), Hkv)))
    v = randn(sum(L), Hkv, D, dt=DT[dtype], seed=77)
    out, lse = run(q, k, v, R, L, D ** -0.5)
    plain.check_prompt(out, lse, plain.prompt_attention(q, split_keys(k, L), split_keys(v, L), R, L, D ** -0.5))
    again, lse2 = run(q, k, v, R, L, D ** -0.5)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("splits", [1, 2, 3, 16])
@pytest.mark.parametrize("dtype,waves,heads", [("bf16", 4, (28, 4, 128)), ("bf16", 8, (28, 4, 128)), ("bf16", 4, (3, 1, 64)),
                                               ("bf16", 8, (6, 2, 64)), ("f32", 4, (6, 2, 128)), ("f32", 4, (5, 1, 64)),
                                               ("f32", 1, (6, 2, 128)), ("f32", 1, (5, 1, 64))], ids=str)
def test_every_form_and_number_of_parts(dtype, waves, heads, splits):
    """What the rule would choose by size, forced: parts without a key, tiles that end inside a sequence, more sequences than lanes."""
    Hq, Hkv, D = heads
    R, L = [r for r, _ in RAGGED], [n for _, n in RAGGED]
    if splits == 2:
        R, L = R + [1] * 60, L + [3, 150, 0] * 20
    q, k, v = (randn(n, h, D, dt=DT[dtype], seed=n + h) for n, h in ((sum(R), Hq), (sum(L), Hkv), (sum(L), Hkv)))
    v = randn(sum(L), Hkv, D, dt=DT[dtype], seed=78)
    v[5, 0, 1] = math.inf if splits == 3 else 0.0     # (seen by the second sequence alone)
    with env_setting("RESPEC_PROMPT_WAVES", waves), env_setting("RESPEC_PROMPT_SPLITS", splits):
        out, lse = run(q, k, v, R, L, D ** -0.5)
    if splits == 3:
        hit = torch.zeros_like(out, dtype=torch.bool)
        hit[R[0] + 4:R[0] + R[1], :Hq // Hkv, 1] = True
        assert torch.isinf(out[hit]).all()
        out, v[5, 0, 1] = torch.where(hit, 0.0, out), 0.0
        o, z, tol, z_tol = plain.prompt_attention(q, split_keys(k, L), split_keys(v, L), R, L, D ** -0.5)
        plain.check_prompt(out, lse, (torch.where(hit, 0.0, o), z, tol, z_tol))
    else:
        plain.check_prompt(out, lse, plain.prompt_attention(q, split_keys(k, L), split_keys(v, L), R, L, D ** -0.5))


def paginate(x, L, ps, table, num_pages):
    pages = torch.full((num_pages, ps, *x.shape[1:]), math.nan, dtype=x.dtype, device="cuda")
    at = e = 0
    for n in L:
        for i in range(0, n, ps):
            m = min(ps, n - i)
            pages[table[e], :m] = x[at + i:at + i + m]
            e += 1
        at += n
    return pages


@pytest.mark.parametrize("ps", [16, 64, 1024])
@pytest.mark.parametrize("dtype,heads", [("f32", (4, 1, 64)), ("bf16", (28, 4, 128)), ("bf16", (2, 2, 64))], ids=str)
def test_paged_equals_packed(dtype, heads, ps):
    """Through pages in scattered order, bit for bit what the tokens in one piece give; unused slots hold NaN."""
    Hq, Hkv, D = heads
    R, L = [r for r, _ in RAGGED], [n for _, n in RAGGED]
    q = randn(sum(R), Hq, D, dt=DT[dtype], seed=5)
    k, v = randn(sum(L), Hkv, D, dt=DT[dtype], seed=6), randn(sum(L), Hkv, D, dt=DT[dtype], seed=7)
    flat, flat_lse = run(q, k, v, R, L, 0.1)
    plain.check_prompt(flat, flat_lse, plain.prompt_attention(q, split_keys(k, L), split_keys(v, L), R, L, 0.1))
    held = [-(-n // ps) for n in L]
    num = sum(held) + 3
    order = torch.randperm(num, generator=torch.Generator().manual_seed(1))[:sum(held)].tolist()
    kp, vp = paginate(k, L, ps, order, num), paginate(v, L, ps, order, num)
    # every sequence's part of the table has room for one page more
    table, at = [], 0
    for h in held:
        table += order[at:at + h] + [-1]
        at += h
    out, lse = torch.empty_like(q), torch.empty((sum(R), Hq), device="cuda")
    ws = workspace(len(R), sum(R), num * ps, max(R), max(L), heads, q.dtype)
    binding.respec_prompt_attention_paged(q, kp, vp, offsets(R, torch.int32), offsets([h + 1 for h in held], torch.int32),
                                          torch.tensor(table, dtype=torch.int32, device="cuda"),
                                          torch.tensor(L, dtype=torch.int32, device="cuda"), out, lse, max(R), max(L), 0.1, ws)
    assert torch.equal(out, flat) and torch.equal(lse, flat_lse)


def test_appended_tokens_are_what_the_paged_call_reads():
    Hq, Hkv, D, ps = 8, 2, 64, 16
    R, L = [20, 0, 1, 50], [20, 9, 33, 70]
    k, v = randn(sum(L), Hkv, D, dt=torch.bfloat16, seed=1), randn(sum(L), Hkv, D, dt=torch.bfloat16, seed=2)
    held = [-(-n // ps) for n in L]
    order = torch.randperm(sum(held), generator=torch.Generator().manual_seed(2)).tolist()
    kp, vp = paginate(k, L, ps, order, sum(held)), paginate(v, L, ps, order, sum(held))
    kq, vq = kp.clone(), vp.clone()
    new = torch.cat([torch.arange(s + n - r, s + n) for s, r, n in zip([0] + offsets(L, torch.int64).tolist()[1:], R, L)])
    at = e = 0
    for r, n in zip(R, L):  # what the call has to fill in
        for i in range(n - r, n):
            kq[order[e + i // ps], i % ps] = vq[order[e + i // ps], i % ps] = math.nan
        e += -(-n // ps)
    fused = torch.cat([k[new.cuda()], v[new.cuda()]], dim=1)
    binding.respec_append_paged(fused[:, :Hkv], fused[:, Hkv:], kq, vq, offsets(R, torch.int32), offsets(held, torch.int32),
                                torch.tensor(order, dtype=torch.int32, device="cuda"), torch.tensor(L, dtype=torch.int32, device="cuda"), max(R))
    assert torch.equal(kq.view(torch.int16), kp.view(torch.int16)) and torch.equal(vq.view(torch.int16), vp.view(torch.int16))


def test_append_writes_nothing_outside_its_pages():
    """Bad page ids, a length past the table and one below the rows: those rows are left out, the others arrive."""
    Hkv, D, ps = 1, 64, 16
    R = [4, 4, 4]
    k = randn(12, Hkv, D, dt=torch.float32, seed=1)
    kp, vp = torch.zeros((3, ps, Hkv, D), device="cuda"), torch.zeros((3, ps, Hkv, D), device="cuda")
    table = torch.tensor([1, 99, -5, 2], dtype=torch.int32, device="cuda")
    kv_len = torch.tensor([18, 2, 40], dtype=torch.int32, device="cuda")   # rows at 14..17, -2..1, (cut to 16) 12..15
    binding.respec_append_paged(k, k, kp, vp, offsets(R, torch.int32), offsets([2, 1, 1], torch.int32), table, kv_len, 4)
    want = torch.zeros_like(kp)
    want[1, 14:16] = k[0:2]
    want[2, 12:16] = k[8:12]
    assert torch.equal(kp, want) and torch.equal(vp, want)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_that_are_not_finite_stay_with_the_rows_that_see_them(dtype, bad):
    n, at = 200, 137
    q, k = randn(n, 4, 64, dt=DT[dtype], seed=1), randn(n, 2, 64, dt=DT[dtype], seed=2)
    v = randn(n, 2, 64, dt=DT[dtype], seed=3)
    clean, _ = run(q, k, v, [n], [n], 0.125)
    v[at, 0, 5] = bad                       # one element of one KV head
    out, _ = run(q, k, v, [n], [n], 0.125)
    hit = torch.zeros_like(out, dtype=torch.bool)
    hit[at:, :2, 5] = True
    assert torch.equal(out[~hit], clean[~hit])
    assert (torch.isnan(out[hit]) if math.isnan(bad) else torch.isinf(out[hit])).all()
    k[at, 1] = math.nan                     # and a key of the other
    out, _ = run(q, k, v, [n], [n], 0.125)
    assert torch.equal(out[:at, 2:], clean[:at, 2:]) and torch.isnan(out[at:, 2:]).all()


def test_hints_below_the_batch_leave_rows_and_keys_out():
    q, k = randn(60, 2, 64, dt=torch.float32, seed=1), randn(60, 1, 64, dt=torch.float32, seed=2)
    out = torch.full_like(q, 7.0)
    ws = workspace(1, 60, 60, 40, 50, (2, 1, 64), torch.float32)
    binding.respec_prompt_attention(q, k, k, offsets([60], torch.int32), offsets([60], torch.int64), out, None, 40, 50, 0.1, ws)
    ref = plain.prompt_attention(q[:40], [k[:50]], [k[:50]], [40], [50], 0.1)
    plain.check_prompt(out[:40], None, ref)
    assert (out[40:] == 7).all()


def test_captured_calls_replay():
    R, L = [70, 3], [70, 2500]
    q, k = randn(73, 8, 64, dt=torch.bfloat16, seed=1), randn(2570, 2, 64, dt=torch.bfloat16, seed=2)
    v = randn(2570, 2, 64, dt=torch.bfloat16, seed=3)
    want, want_lse = run(q, k, v, R, L, 0.125)
    out, lse = torch.zeros_like(q), torch.zeros((73, 8), device="cuda")
    ws = workspace(2, 73, 2570, 70, 2500, (8, 2, 64), torch.bfloat16)
    a, b = offsets(R, torch.int32), offsets(L, torch.int64)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.respec_prompt_attention(q, k, v, a, b, out, lse, 70, 2500, 0.125, ws)
    for _ in range(3):
        out.zero_()
        lse.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
        run(q, k, v, R, L, 0.125)


def test_another_stream():
    q, k = randn(300, 4, 64, dt=torch.bfloat16, seed=1), randn(300, 4, 64, dt=torch.bfloat16, seed=2)
    want, _ = run(q, k, k, [300], [300], 0.125)
    out = torch.zeros_like(q)
    ws = workspace(1, 300, 300, 300, 300, (4, 4, 64), torch.bfloat16)
    a, b = offsets([300], torch.int32), offsets([300], torch.int64)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    binding.respec_prompt_attention(q, k, k, a, b, out, None, 300, 300, 0.125, ws, stream=stream)
    stream.synchronize()
    assert torch.equal(out, want)


def test_offsets_past_32_bits():
    """A cache of more than 2^32 bytes (and 2^31 elements): the sequence at its end."""
    n, Hkv, D = 300, 8, 128
    total = (1 << 31) // (Hkv * D) + 5000
    k, v = (torch.empty((total, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = randn(n, 16, D, dt=torch.bfloat16, seed=1)
    k[-n:], v[-n:] = randn(n, Hkv, D, dt=torch.bfloat16, seed=2), randn(n, Hkv, D, dt=torch.bfloat16, seed=3)
    out = torch.empty_like(q)
    a = torch.tensor([0, 0, n], dtype=torch.int32, device="cuda")
    b = torch.tensor([0, total - n, total], dtype=torch.int64, device="cuda")
    ws = workspace(2, n, total, n, n, (16, Hkv, D), torch.bfloat16)
    binding.respec_prompt_attention(q, k, v, a, b, out, None, n, n, D ** -0.5, ws)
    plain.check_prompt(out, None, plain.prompt_attention(q, [k[-n:]], [v[-n:]], [n], [n], D ** -0.5))
    pages = total // 64                     # the same memory as pages
    kp, vp = (x[-pages * 64:].view(pages, 64, Hkv, D) for x in (k, v))
    table = torch.arange(pages - 5, pages, dtype=torch.int32, device="cuda")   # the last 320 tokens
    kv_len = torch.tensor([320], dtype=torch.int32, device="cuda")
    k[-320:-n], v[-320:-n] = 0.0, 1.0
    out2 = torch.empty_like(q)
    binding.respec_prompt_attention_paged(q, kp, vp, torch.tensor([0, n], dtype=torch.int32, device="cuda"), offsets([5], torch.int32), table,
                                          kv_len, out2, None, n, 320, D ** -0.5, ws)
    plain.check_prompt(out2, None, plain.prompt_attention(q, [k[-320:]], [v[-320:]], [n], [320], D ** -0.5))


def test_many_sequences_of_one_token():
    B = 3000
    q, k = randn(B, 4, 64, dt=torch.bfloat16, seed=1), randn(B, 2, 64, dt=torch.bfloat16, seed=2)
    v = randn(B, 2, 64, dt=torch.bfloat16, seed=3)
    out, _ = run(q, k, v, [1] * B, [1] * B, 0.125)
    assert torch.equal(out, v.repeat_interleave(2, dim=1))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_loose_hints(dtype):
    """Bounds far above the batch change how the work is cut, not what comes out."""
    R, L = [40, 1, 0, 130], [40, 600, 9, 131]
    q, k = randn(sum(R), 6, 128, dt=DT[dtype], seed=1), randn(sum(L), 2, 128, dt=DT[dtype], seed=2)
    v = randn(sum(L), 2, 128, dt=DT[dtype], seed=3)
    ref = plain.prompt_attention(q, split_keys(k, L), split_keys(v, L), R, L, 0.1)
    for max_q, max_kv in ((130, 600), (sum(R), sum(L)), (1 << 20, 1 << 30), (1 << 20, 2 ** 31 - 257)):
        out, lse = torch.full_like(q, 7.0), torch.full((sum(R), 6), 7.0, device="cuda")
        ws = workspace(4, sum(R), sum(L), max_q, max_kv, (6, 2, 128), DT[dtype])
        binding.respec_prompt_attention(q, k, v, offsets(R, torch.int32), offsets(L, torch.int64), out, lse, max_q, max_kv, 0.1, ws)
        plain.check_prompt(out, lse, ref)


def test_two_calls_at_once():
    """On two streams, each with its workspace; both cut their keys into parts."""
    calls = []
    for seed, (R, L) in enumerate((([30, 2], [3000, 4100]), ([5, 50, 1], [700, 2000, 5000]))):
        q, k = randn(sum(R), 8, 128, dt=torch.bfloat16, seed=seed), randn(sum(L), 2, 128, dt=torch.bfloat16, seed=seed + 9)
        want, _ = run(q, k, k, R, L, 0.1)
        ws = workspace(len(R), sum(R), sum(L), max(R), max(L), (8, 2, 128), torch.bfloat16)
        calls.append((torch.cuda.Stream(), q, k, offsets(R, torch.int32), offsets(L, torch.int64), torch.zeros_like(q), max(R), max(L), ws, want))
    torch.cuda.synchronize()
    for _ in range(20):
        for stream, q, k, a, b, out, max_q, max_kv, ws, _ in calls:
            binding.respec_prompt_attention(q, k, k, a, b, out, None, max_q, max_kv, 0.1, ws, stream=stream)
    torch.cuda.synchronize()
    for *_, out, _, _, _, want in calls:
        assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads", [(1, 1, 128), (130, 1, 64), (300, 2, 64), (64, 1, 128)], ids=str)
def test_one_head_and_more_heads_than_a_tile_has_rows(dtype, heads):
    Hq, Hkv, D = heads
    R, L = [3, 40, 1], [3, 140, 70]
    q, k = randn(sum(R), Hq, D, dt=DT[dtype], seed=1), randn(sum(L), Hkv, D, dt=DT[dtype], seed=2)
    v = randn(sum(L), Hkv, D, dt=DT[dtype], seed=3)
    out, lse = run(q, k, v, R, L, D ** -0.5)
    plain.check_prompt(out, lse, plain.prompt_attention(q, split_keys(k, L), split_keys(v, L), R, L, D ** -0.5))
