"""Appended rows whose place lies outside what the sequence holds, or that the call is not asked to write."""
import pytest
import torch

from paper_2510_26475_amd import binding

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("max_q", [9, 4, 1])
def test_rows_go_to_their_positions_or_nowhere(dtype, max_q):
    """Row i of a sequence goes to kv_len - R + i if its pages have that place and i < max_q, and everything else stays as it was."""
    Hkv, D, ps, num_pages = 2, 64, 16, 12
    R = [8, 4, 4, 0, 9, 5, 3, 2, 4]
    kv = [20, 40, 2, 7, 32, 33, -5, 2 ** 31 - 1, 18]        # of pages of 16: past one page; far past it; below the rows; no rows; to the end; ...
    held = [1, 1, 1, 1, 2, 2, 1, 1, 2]
    table = [5, 0, 7, 3, 2, 9, 4, 99, 1, 6, -5, 8]           # (99, -5: no pages)
    indptr = [0] + torch.tensor(held).cumsum(0).tolist()
    gen = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((sum(R), Hkv, D), generator=gen, device="cuda").to(dtype) for _ in range(2))
    pools = [torch.randn((num_pages, ps, Hkv, D), generator=gen, device="cuda").to(dtype) for _ in range(2)]
    want, written = [p.clone() for p in pools], 0
    at = 0
    for b, r in enumerate(R):
        for i in range(min(r, max_q)):
            pos = kv[b] - r + i
            if 0 <= pos < ps * held[b] and 0 <= table[indptr[b] + pos // ps] < num_pages:
                for w, new in zip(want, (k, v)):
                    w[table[indptr[b] + pos // ps], pos % ps] = new[at + i]
                written += 1
        at += r
    assert written > 0
    binding.respec_append_paged(k, v, *pools, ints([0] + R).cumsum(0).to(torch.int32), ints(indptr), ints(table), ints(kv), max_q)
    for w, p in zip(want, pools):
        assert torch.equal(w, p)


def test_a_sequence_that_got_no_pages_keeps_its_tokens():
    """The lengths are raised for all sequences of a batch, one of which was not served: what it holds stays."""
    ps, Hkv, D = 16, 1, 64
    indptr, table, count, kv, refs = ints([0, 3, 6]), ints([-1] * 6), ints([0, 0]), ints([0, 0]), ints([0] * 3)
    src, dst, missing = ints([0] * 2), ints([0] * 2), ints([0] * 2)
    ws = torch.empty(binding.respec_pages_workspace_bytes(2, 3), dtype=torch.uint8, device="cuda")
    binding.respec_pages_resize(ints([16, 16]), indptr, table, count, kv, refs, src, dst, missing, ps, ws)
    kv.copy_(ints([16, 16]))
    binding.respec_pages_resize(ints([24, 24]), indptr, table, count, kv, refs, src, dst, missing, ps, ws)
    assert missing.tolist() == [0, 1]
    pools = [torch.randn((3, ps, Hkv, D), device="cuda") for _ in range(2)]
    want = [p.clone() for p in pools]
    new = torch.randn((16, Hkv, D), device="cuda")
    kv.add_(8)
    binding.respec_append_paged(new, new, *pools, ints([0, 8, 16]), indptr, table, kv, 8)
    for w, p in zip(want, pools):
        w[table[1].item(), :8] = new[:8]
        assert torch.equal(w, p)
