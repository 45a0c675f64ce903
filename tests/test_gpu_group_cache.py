"""One rollout group through the calls as they are used together: prompts normalised, rotated and written into the cache (in its type or in 8 bits), attended,
forked into their responses, chunks, verify steps over the shared pages, trees with their commit, and plain decoding."""
import math

import pytest
import torch

import plain
import plain_cache as pc
from paper_2510_26475_amd import binding
from plain_cache import ints, offsets, scratch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,pool", [(torch.float32, "same"), (torch.bfloat16, "same"), (torch.bfloat16, "e4m3")])
def test_a_group(dtype, pool):
    Hq, Hkv, D, ps, layers, eps = 8, 2, 64, 16, 2, 1e-6
    code, scale, quantised = int(dtype == torch.bfloat16), 1 / math.sqrt(64), pool == "e4m3"
    prompts, per = [70, 33], 3
    P, B = len(prompts), len(prompts) * (1 + per)
    gen = torch.Generator(device="cuda").manual_seed(1)
    inv = (1e4 ** (-torch.arange(0, 32, dtype=torch.float64) / 32)).float().cuda()
    cap, num_pages = 9, 60
    page_indptr, table = ints([i * cap for i in range(B + 1)]), ints([-1] * (cap * B))
    count, kv, refs = ints([0] * B), ints([0] * B), ints([0] * num_pages)
    src, dst, missing = ints([0] * B), ints([0] * B), ints([0] * B)
    pages_ws = scratch(binding.respec_pages_workspace_bytes(B, num_pages))

    def pools():
        if quantised:
            return [torch.full((num_pages, ps, Hkv, D), 0x7f, dtype=torch.uint8, device="cuda") for _ in range(2)] + [
                torch.full((num_pages, Hkv, ps), 255, dtype=torch.uint8, device="cuda") for _ in range(2)]
        return [torch.full((num_pages, ps, Hkv, D), math.nan, dtype=dtype, device="cuda") for _ in range(2)] + [None, None]

    layer = [dict(pools=pools(), w=[1 + 0.2 * torch.randn(D, generator=gen, device="cuda") for _ in range(2)], seen=[([], []) for _ in range(B)]) for _ in range(layers)]

    def resize(want):
        binding.respec_pages_resize(ints(want), page_indptr, table, count, kv, refs, src, dst, missing, ps, pages_ws)
        for y in layer:
            (binding.respec_pages_copy_quantised if quantised else binding.respec_pages_copy)(*[x for x in y["pools"] if x is not None], src, dst)
        assert missing.tolist() == [0] * B

    def write(y, R, ip, lens, first, positions=None):
        """New tokens of sequences first .. into layer y; returns Q as it was written and keeps what the cache holds of K and V."""
        n = sum(R)
        qkv = torch.randn((n, Hq + 2 * Hkv, D), generator=gen, device="cuda").to(dtype)
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        out = torch.empty((n, Hq, D), dtype=dtype, device="cuda")
        binding.respec_norm_rope_append_paged(q, k, v, *y["w"], inv, positions, out, *y["pools"], offsets(R), ip, table, lens, max(R), eps)
        L = lens.tolist()
        pos = positions.long() if positions is not None else ints([L[b] - r + i for b, r in enumerate(R) for i in range(r)], torch.int64)
        ref, tol = pc.norm_rope(q, y["w"][0], eps, pos, inv, False)
        pc.check_rounded(out, ref, tol, "q")
        refs_kv = [pc.norm_rope(k, y["w"][1], eps, pos, inv, False), (v.double(), torch.zeros((), device="cuda"))]
        at = 0
        for b, r in enumerate(R):
            for i in range(r):
                p = L[b] - r + i
                page, slot = table[ip[b] + p // ps].item(), p % ps
                for j, (want, bound) in enumerate(refs_kv):
                    got = y["pools"][j][page, slot]
                    bound = bound if bound.dim() == 0 else bound[at + i]
                    if quantised:
                        got = pc.values(got, y["pools"][2 + j][page, :, slot])
                        pc.check_quantised(got, want[at + i], bound, "kv")
                    else:
                        pc.check_rounded(got, want[at + i], bound, "kv")
                    y["seen"][first + b][j].append(got.double())
            at += r
        return out

    def held(y, first, n):
        empty = torch.empty((0, Hkv, D), dtype=torch.float64, device="cuda")
        return [[torch.stack(y["seen"][b][j]) if y["seen"][b][j] else empty for b in range(first, first + n)] for j in (0, 1)]

    def prompt(R):
        """Prompts or their next chunks: over a cache of 8 bits what it holds is read back first."""
        kv.add_(ints(R))
        L = kv.tolist()
        ws = scratch(binding.respec_prompt_attention_workspace_bytes(B, sum(R), max(sum(L), num_pages * ps), max(R), max(L), Hq, Hkv, D, code))
        for y in layer:
            q = write(y, R, page_indptr, kv, 0)
            out, lse = torch.empty_like(q), torch.empty((sum(R), Hq), device="cuda")
            if quantised:
                back = [torch.full((sum(L), Hkv, D), math.nan, dtype=dtype, device="cuda") for _ in range(2)]
                kv_indptr = offsets(L, torch.int64)
                binding.respec_read_paged_quantised(*y["pools"], page_indptr, table, kv, kv_indptr, *back, max(L))
                binding.respec_prompt_attention(q, *back, offsets(R), kv_indptr, out, lse, max(R), max(L), scale, ws)
            else:
                binding.respec_prompt_attention_paged(q, *y["pools"][:2], offsets(R), page_indptr, table, kv, out, lse, max(R), max(L), scale, ws)
            plain.check_prompt(out, lse, pc.attention(q, *held(y, 0, B), R, L, scale))

    resize(prompts + [0] * (B - P))
    prompt([40, 33] + [0] * (B - P))
    prompt([30, 0] + [0] * (B - P))
    parent = [-1] * P + [p for p in range(P) for _ in range(per)]
    binding.respec_pages_fork(ints(parent), page_indptr, table, count, kv, refs, missing)
    for y in layer:
        for b, p in enumerate(parent):
            if p >= 0:
                y["seen"][b] = tuple(list(x) for x in y["seen"][p])
    resize([0] * P + [-1] * (B - P))
    n, ip = B - P, page_indptr[P:]
    groups, shared = ints([0, per, 2 * per]), ints([p // ps * ps for p in prompts])

    parents = {"chain": [-1, 0, 1, 2], "tree": [-1, 0, 0, 1, 2, 1], "one": [-1]}
    for step, shape in enumerate(("chain", "tree", "one", "tree", "chain")):
        tree = parents[shape]
        r = len(tree)
        before = kv.tolist()[P:]
        resize([-1] * P + [x + r for x in before])
        masks, depth = [], []
        for i, p in enumerate(tree):
            masks.append((masks[p] if p >= 0 else 0) | 1 << i)
            depth.append(depth[p] + 1 if p >= 0 else 0)
        kv[P:] += r
        lens, R = kv[P:], [r] * n
        L = lens.tolist()
        positions = ints([x + d for x in before for d in depth]) if shape == "tree" else None
        ws = scratch(binding.respec_verify_attention_shared_workspace_bytes(n, n * r, 2, r, max(L), Hq, Hkv, D, code))
        for i, y in enumerate(layer):
            q = write(y, R, ip, lens, P, positions)
            out, lse = torch.empty_like(q), torch.empty((n * r, Hq), device="cuda")
            call = binding.respec_verify_attention_shared_next_layer if i else binding.respec_verify_attention_shared
            call(q, *y["pools"], offsets(R), ip, table, lens, groups, shared, ints(masks * n, torch.int64) if shape == "tree" else None, out, lse, r, max(L), scale, ws)
            plain.check_prompt(out, lse, pc.attention(q, *held(y, P, n), R, L, scale, masks * n if shape == "tree" else None))
            if not quantised and step < 2:                       # the same as without sharing
                alone = torch.empty_like(out)
                ws2 = scratch(binding.respec_verify_attention_workspace_bytes(n, n * r, num_pages * ps, r, max(L), Hq, Hkv, D, code))
                binding.respec_verify_attention_paged(q, *y["pools"][:2], offsets(R), ip, table, lens, alone, None, r, max(L), scale, ws2,
                                                      tree_mask=ints(masks * n, torch.int64) if shape == "tree" else None)
                assert (alone.double() - out.double()).abs().max() <= (2e-2 if code else 1e-5)
        path = [[1, 3, 0], [2, 4, 0], [1, 5, 0], [2, 0, 0], [1, 0, 0], [0, 0, 0]] if shape == "tree" else [[1, 2, 3]] * n
        accepted = [2, 2, 2, 1, 1, 0] if shape == "tree" else [min(b, r - 1) for b in range(n)]
        after = None
        for y in layer:
            mine = lens.clone()
            if quantised:
                binding.respec_commit_accepted_paged_quantised(*y["pools"], offsets(R), ip, table, mine, ints(accepted), n * r, r, path=ints(path) if shape == "tree" else None)
            else:
                binding.respec_commit_accepted_paged(*y["pools"][:2], offsets(R), ip, table, mine, ints(accepted), n * r, r, path=ints(path) if shape == "tree" else None)
            after = mine
            for b in range(n):
                rows = [0] + (path[b][:accepted[b]] if shape == "tree" else list(range(1, accepted[b] + 1)))
                y["seen"][P + b] = tuple(x[:before[b]] + [x[before[b] + i] for i in rows] for x in y["seen"][P + b])
        kv[P:] = after
        assert kv.tolist()[P:] == [x + 1 + a for x, a in zip(before, accepted)]
    resize([0] * B)
    assert refs.tolist() == [0] * num_pages
