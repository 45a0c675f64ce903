"""Which rows the write of the paged cache belongs to: many sequences, most of them without rows, offsets that begin late or end early, more rows than the
bound; and offsets that mean nothing, which stay inside the buffers."""
import pytest
import torch

from paper_2510_26475_amd import binding
from plain_cache import ints
from test_gpu_cache_write import check, write

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.mark.parametrize("R", [[0] * 200 + [3] + [0] * 300 + [1, 2] + [0] * 50, [i % 3 for i in range(1500)], [0] * 63 + [1], [0] * 64 + [1], [1] + [0] * 64, [1] * 65,
                               [0] * 4095 + [2, 1], [0, 5, 0, 0, 2]], ids=lambda R: f"{len(R)}-{sum(R)}")
@pytest.mark.parametrize("pool", ["same", "e4m3"])
def test_rows_among_many_sequences(R, pool):
    check(write(R, [(7 * b) % 40 if b % 5 else 0 for b in range(len(R))], 4, 2, 64, 16, BF16, pool, rotary=64))


def call(q_indptr, total_q, max_q, before, held=2, D=64, page=16):
    """K and V only, each sequence with pages of its own; returns K, V and the pools."""
    B = len(q_indptr) - 1
    k, v = (torch.randn((total_q, 1, D), device="cuda") for _ in range(2))
    pools = [torch.full((B * held, page, 1, D), 7.0, device="cuda") for _ in range(2)]
    lens = ints([n + (q_indptr[b + 1] - q_indptr[b]) for b, n in enumerate(before)])
    binding.respec_norm_rope_append_paged(None, k, v, None, None, None, None, None, *pools, None, None, ints(q_indptr), ints([b * held for b in range(B + 1)]),
                                          ints(list(range(B * held))), lens, max_q, 0.0)
    torch.cuda.synchronize()
    return k, v, pools


@pytest.mark.parametrize("q_indptr,total_q,max_q", [([3, 5, 9], 12, 4), ([0, 2, 4], 10, 2), ([2, 9, 10], 10, 3), ([0, 0, 7], 9, 7), ([4, 4, 4], 6, 1)])
def test_rows_of_no_sequence_and_past_the_bound(q_indptr, total_q, max_q):
    before, held, page = [3, 0], 2, 16
    k, v, pools = call(q_indptr, total_q, max_q, before)
    for x, pool in zip((k, v), pools):
        expected = torch.full_like(pool, 7.0)
        for b in range(2):
            for i in range(min(q_indptr[b + 1] - q_indptr[b], max_q)):
                n = before[b] + i
                expected[b * held + n // page, n % page] = x[q_indptr[b] + i]
        assert torch.equal(pool, expected)


@pytest.mark.parametrize("page_indptr", [[0, 2, 4], [0, 3, -2 ** 31], [3, -2 ** 31, 2 ** 31 - 1], [-2 ** 31, 4, 1]])
@pytest.mark.parametrize("q_indptr", [[5, 3, 1], [-4, 2, 30], [0, 2 ** 31 - 1, 4], [-2 ** 31, -1, 6], [7, 0, 7], [0, 8, -2 ** 31], [0, 5, 8]])
def test_offsets_that_mean_nothing(q_indptr, page_indptr):
    total_q, D, page = 8, 64, 16
    k, v = (torch.randn((total_q, 1, D), device="cuda") for _ in range(2))
    guard = [torch.full((6, page, 1, D), 7.0, device="cuda") for _ in range(2)]
    pools = [g[1:5] for g in guard]
    binding.respec_norm_rope_append_paged(None, k, v, None, None, None, None, None, *pools, None, None, ints(q_indptr), ints(page_indptr), ints([0, 1, 2, 3]), ints([20, 9]),
                                          8, 0.0)
    torch.cuda.synchronize()
    for g in guard:
        assert (g[0] == 7.0).all() and (g[5] == 7.0).all() and torch.isfinite(g).all()
    # and the attention over them
    q, out = torch.randn((total_q, 2, D), device="cuda"), torch.full((total_q + 8, 2, D), 5.0, device="cuda")
    for groups in ((None, None), (ints([0, 2]), ints([16]))):
        ws = torch.empty(binding.respec_verify_attention_shared_workspace_bytes(2, total_q, 1, 8, 64, 2, 1, D, 0), dtype=torch.uint8, device="cuda")
        binding.respec_verify_attention_shared(q, *pools, None, None, ints(q_indptr), ints(page_indptr), ints([0, 1, 2, 3]), ints([20, 9]), *groups, None, out[:total_q], None,
                                               8, 64, 0.1, ws)
        torch.cuda.synchronize()
        assert (out[total_q:] == 5.0).all() and torch.isfinite(out).all()
