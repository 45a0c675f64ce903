"""The profiling hook around the main kernel of every attention call over the paged cache."""
import pytest
import torch

from paper_2510_26475_amd import binding
from plain_cache import Cache, ints, offsets
from test_gpu_shared import BF16, workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("entry", ["shared", "next_layer", "quantised", "paged"])
def test_the_next_call_records_the_events_and_forgets_them(entry):
    c = Cache([300, 200], 2, 64, 16, BF16, pool="e4m3" if entry == "quantised" else "same", seed=3)
    q = torch.randn((8, 4, 64), device="cuda").to(BF16)
    out, ws = torch.empty_like(q), workspace(2, 8, 0, 4, 300, 4, 2, 64, BF16)
    tables = offsets([4, 4]), *c.tables()

    def call():
        if entry == "quantised":
            binding.respec_verify_attention_paged_quantised(q, *c.args(), *tables, out, None, 4, 300, 0.125, ws)
        elif entry == "paged":
            n = binding.respec_verify_attention_workspace_bytes(2, 8, 16 * c.page_table.numel(), 4, 300, 4, 2, 64, int(q.dtype == BF16))
            binding.respec_verify_attention_paged(q, c.k, c.v, *tables, out, None, 4, 300, 0.125, torch.empty(max(n, 1), dtype=torch.uint8, device="cuda"))
        else:
            name = "respec_verify_attention_shared" + ("_next_layer" if entry == "next_layer" else "")
            getattr(binding, name)(q, *c.args(), *tables, None, None, None, out, None, 4, 300, 0.125, ws)

    if entry == "next_layer":
        binding.respec_verify_attention_shared(q, *c.args(), *tables, None, None, None, out, None, 4, 300, 0.125, ws)
    before, after, end = (torch.cuda.Event(enable_timing=True) for _ in range(3))
    before.record()
    after.record()
    big = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    for _ in range(4):                                            # (some hundred microseconds between the two recordings)
        big.zero_()
    end.record()
    torch.cuda.synchronize()
    old = before.elapsed_time(end)
    binding.respec_profile_mark_main(before, after)
    try:
        call()
        torch.cuda.synchronize()
        assert end.elapsed_time(before) > 0 and old > 0          # (recorded again, behind `end`)
        took = before.elapsed_time(after)
        assert took > 0
        again = end.elapsed_time(before)
        call()
        torch.cuda.synchronize()
        assert end.elapsed_time(before) == again and before.elapsed_time(after) == took
    finally:
        binding.respec_profile_mark_main(None, None)
