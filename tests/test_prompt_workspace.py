"""The prompt attention's workspace: one for the largest sizes does for all smaller ones."""
import random

import pytest
import torch

from paper_2510_26475_amd import binding

HEADS = [(28, 4, 128, binding.RESPEC_BF16), (16, 2, 128, binding.RESPEC_BF16), (32, 32, 64, binding.RESPEC_BF16), (4, 1, 64, binding.RESPEC_F32),
         (300, 2, 128, binding.RESPEC_F32)]


def size(sizes, heads):
    B, total_q, total_kv, max_q, max_kv = sizes
    return binding.respec_prompt_attention_workspace_bytes(B, total_q, total_kv, max_q, max_kv, *heads)


@pytest.mark.parametrize("heads", HEADS, ids=str)
def test_no_smaller_sizes_need_more(heads):
    rng = random.Random(1)
    for _ in range(2000):
        large = [int(2 ** rng.uniform(0, hi)) for hi in (8, 16, 20, 13, 18)]
        small = [rng.choice([x, rng.randrange(1, x + 1), min(x, int(2 ** rng.uniform(0, 18)))]) for x in large]
        assert 256 <= size(small, heads) <= size(large, heads) <= 130 << 20, (small, large)


def test_chunks_in_the_workspace_of_a_batch_of_prompts():
    heads = (28, 4, 128, binding.RESPEC_BF16)
    assert size((1, 40, 9000, 40, 2048), heads) <= size((16, 16 * 2048, 16 * 2048, 2048, 2048), heads)
    assert size((1, 512, 2048, 512, 2048), heads) <= size((16, 16 * 2048, 16 * 2048, 2048, 2048), heads)


@pytest.mark.gpu
def test_one_workspace_for_many_sizes():
    import plain
    from test_gpu_prompt import offsets, randn, split_keys
    Hq, Hkv, D = 28, 4, 128
    largest = (16, 4096, 1 << 20, 2048, 8192)
    ws = torch.empty(size(largest, (Hq, Hkv, D, binding.RESPEC_BF16)), dtype=torch.uint8, device="cuda")
    for R, L in (([40], [8000]), ([512], [2048]), ([1, 70, 0, 5], [6000, 70, 900, 8192]), ([300, 200], [300, 200]), ([1] * 16, [8192] + [100] * 15)):
        q = randn(sum(R), Hq, D, dt=torch.bfloat16, seed=1)
        k, v = (randn(sum(L), Hkv, D, dt=torch.bfloat16, seed=s) for s in (2, 3))
        out, lse = torch.full_like(q, 7.0), torch.full((sum(R), Hq), 7.0, device="cuda")
        ws.fill_(0xff)
        binding.respec_prompt_attention(q, k, v, offsets(R, torch.int32), offsets(L, torch.int64), out, lse, max(R), max(L), D ** -0.5, ws)
        plain.check_prompt(out, lse, plain.prompt_attention(q, split_keys(k, L), split_keys(v, L), R, L, D ** -0.5))
