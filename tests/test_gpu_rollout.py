"""One group of a rollout through the calls as they are used together: prompts into the paged cache, each forked into its responses,
a verify step and its commit, the log-probabilities of what was emitted and their gradient, the pages moved together and given back."""
import torch
import pytest

import plain
from paper_2510_26475_amd import binding

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def ws(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_group_of_responses(dtype):
    Hq, Hkv, D, ps, V, k, layers = 8, 2, 64, 16, 1000, 3, 2
    code, scale = int(dtype == torch.bfloat16), 64 ** -0.5
    prompts, children = [37, 16, 50], 2
    P = len(prompts)
    B = P * (1 + children)
    gen = torch.Generator(device="cuda").manual_seed(1)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda").to(dtype)

    cap, num_pages = [6] * B, 40
    page_indptr = ints([i * 6 for i in range(B + 1)])
    table, count, kv, refs = ints([-1] * (6 * B)), ints([0] * B), ints([0] * B), ints([0] * num_pages)
    src, dst, missing = ints([0] * B), ints([0] * B), ints([0] * B)
    pages_ws = ws(binding.respec_pages_workspace_bytes(B, num_pages))
    pools = [(torch.full((num_pages, ps, Hkv, D), float("nan"), dtype=dtype, device="cuda"),
              torch.full((num_pages, ps, Hkv, D), float("nan"), dtype=dtype, device="cuda")) for _ in range(layers)]
    seen = [[([], []) for _ in range(B)] for _ in range(layers)]     # K and V of every sequence, as the model has them

    def resize(want):
        binding.respec_pages_resize(ints(want), page_indptr, table, count, kv, refs, src, dst, missing, ps, pages_ws)
        for kp, vp in pools:
            binding.respec_pages_copy(kp, vp, src, dst)
        assert missing.tolist() == [0] * B

    def forward(R, rows, entry):
        """New tokens of all sequences into every layer, and the attention over what they hold then."""
        q_indptr = ints([0] + R).cumsum(0).to(torch.int32)
        kv.add_(ints(R))
        L = kv.tolist()
        for layer, (kp, vp) in enumerate(pools):
            q, kn, vn = randn(sum(R), Hq, D), randn(sum(R), Hkv, D), randn(sum(R), Hkv, D)
            binding.respec_append_paged(kn, vn, kp, vp, q_indptr, page_indptr, table, kv, max(R))
            at = 0
            for b, r in enumerate(R):
                for mine, new in zip(seen[layer][b], (kn, vn)):
                    mine += list(new[at:at + r])
                at += r
            out, lse = torch.empty_like(q), torch.empty((sum(R), Hq), device="cuda")
            size = getattr(binding, entry + "_workspace_bytes")(B, sum(R), num_pages * ps, max(R), max(L), Hq, Hkv, D, code)
            getattr(binding, entry + "_paged")(q, kp, vp, q_indptr, page_indptr, table, kv, out, lse, max(R), max(L), scale, ws(size))
            keys, values = ([torch.stack(s[i]) if s[i] else torch.empty((0, Hkv, D), dtype=dtype, device="cuda") for s in seen[layer]] for i in (0, 1))
            ref = plain.prompt_attention(q, keys, values, R, L, scale)
            plain.check_prompt(out, lse, ref)

    R = prompts + [0] * (B - P)
    resize(R)
    forward(R, None, "respec_prompt_attention")
    parent = [-1] * P + [p for p in range(P) for _ in range(children)]
    binding.respec_pages_fork(ints(parent), page_indptr, table, count, kv, refs, missing)
    for layer in range(layers):
        for b, p in enumerate(parent):
            if p >= 0:
                seen[layer][b] = tuple(list(x) for x in seen[layer][p])
    resize([0] * P + [-1] * (B - P))                 # the prompts' own slots are not needed any more
    for layer in range(layers):
        for b in range(P):
            seen[layer][b] = ([], [])
    lens = kv.tolist()
    resize([-1] * P + [n + k + 1 for n in lens[P:]])

    # a verify step: k drafts and one more row for each response (the attention wants rows for every sequence it is given)
    live = list(range(P, B))
    sub = (page_indptr[P:], kv[P:].clone())
    n, rows = len(live), (k + 1) * len(live)
    q_indptr = ints([(k + 1) * i for i in range(n + 1)])
    sub[1].add_(k + 1)
    for layer, (kp, vp) in enumerate(pools):
        q, kn, vn = randn(rows, Hq, D), randn(rows, Hkv, D), randn(rows, Hkv, D)
        binding.respec_append_paged(kn, vn, kp, vp, q_indptr, sub[0], table, sub[1], k + 1)
        keys, values = [], []
        for i, b in enumerate(live):
            for mine, new in zip(seen[layer][b], (kn, vn)):
                mine += list(new[i * (k + 1):(i + 1) * (k + 1)])
            keys.append(torch.stack(seen[layer][b][0]))
            values.append(torch.stack(seen[layer][b][1]))
        L = sub[1].tolist()
        verify, prompt = torch.empty_like(q), torch.empty_like(q)
        size = binding.respec_verify_attention_workspace_bytes(n, rows, num_pages * ps, k + 1, max(L), Hq, Hkv, D, code)
        binding.respec_verify_attention_paged(q, kp, vp, q_indptr, sub[0], table, sub[1], verify, None, k + 1, max(L), scale, ws(size))
        size = binding.respec_prompt_attention_workspace_bytes(n, rows, num_pages * ps, k + 1, max(L), Hq, Hkv, D, code)
        binding.respec_prompt_attention_paged(q, kp, vp, q_indptr, sub[0], table, sub[1], prompt, None, k + 1, max(L), scale, ws(size))
        ref = plain.prompt_attention(q, keys, values, [k + 1] * n, L, scale)
        plain.check_prompt(prompt, None, ref)
        assert (verify.double() - ref[0]).abs().max() <= (2e-2 if code else 1e-5)

    target = randn(rows, V)
    draft, drafted = randn(rows - n, V), torch.randint(0, V, (rows - n,), generator=gen, device="cuda", dtype=torch.int32)
    u, u_final = torch.rand(rows - n, generator=gen, device="cuda"), torch.rand(n, generator=gen, device="cuda")
    tokens, accepted = torch.empty((n, k + 1), dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
    binding.respec_rejection_sample(target, draft, drafted, q_indptr, u, u_final, tokens, accepted, None, k, 0.6)
    flat = tokens.view(-1)                           # row (b, i) of the target's logits emitted tokens[b, i]; -1 behind the last one
    lp, lse, ent = (torch.empty(rows, device="cuda") for _ in range(3))
    binding.respec_token_logprobs(target, flat, lp, lse, ent, None, None, 0.6,
                                  ws(binding.respec_token_logprobs_workspace_bytes(rows, V, 0, code)))
    ref = plain.token_logprobs(target, flat, 0.6)
    for a, b in zip((lp, lse, ent), ref):
        assert (a.double() - b).abs().max() <= 1e-4
    assert (lp[flat < 0] == 0).all() and (lp[flat >= 0] < 0).all()
    grad = torch.empty_like(target)
    binding.respec_token_logprobs_grad(target, flat, lse, ent, torch.ones_like(lp), None, grad, 0.6)
    want = plain.logprob_grad(target, flat, 0.6, torch.ones_like(lp), torch.zeros_like(lp))
    assert (grad.double() - want).abs().max() <= (2.0 ** -8 if code else 1e-5) * want.abs().max()

    for kp, vp in pools:                             # the commit cuts the lengths (a chain: nothing moves)
        lens = sub[1].clone()
        binding.respec_commit_accepted_paged(kp, vp, q_indptr, sub[0], table, lens, accepted, rows, k + 1)
    held = list(zip(sub[1].tolist(), accepted.tolist()))
    kv[P:] = lens
    for i, b in enumerate(live):
        assert kv[b].item() == held[i][0] - (k - held[i][1])
        for layer in range(layers):
            seen[layer][b] = tuple(x[:kv[b].item()] for x in seen[layer][b])
    resize([-1] * P + kv.tolist()[P:])               # pages of rejected drafts go back

    moves = num_pages // 2
    a, b2, end = ints([0] * moves), ints([0] * moves), ints([0])
    binding.respec_pages_compact(table, refs, table, refs, a, b2, end, pages_ws)
    for kp, vp in pools:
        binding.respec_pages_copy(kp, vp, a, b2)
    used = (refs > 0).sum().item()
    assert end.item() == used and (refs[used:] == 0).all()
    resize([-1] * P + [x + 5 for x in kv.tolist()[P:]])
    forward([0] * P + [5] * (B - P), None, "respec_prompt_attention")
    resize([0] * B)
    assert refs.tolist() == [0] * num_pages and kv.tolist() == [0] * B
