"""Calls of a rollout around the verify step, as timed cases: prompts, token log-probabilities, pages of the cache.

A generation engine runs the attention of whole prompts (or of a prompt's next chunk over the paged cache), forks a
prompt's pages into the responses of its group, gives their pages back, moves pages together before it shrinks its
pools, and records the log-probabilities of what was sampled; the learner takes their gradient.  Heads, vocabularies,
page sizes and temperatures are those of the package's own workloads.

A case names its shape by plain values; lengths are part of the shape (drawn from `shape_seed`).  Where `own` is true
the package's calls run, else plain torch operations in 32 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

HEADS = {  # (query heads, KV heads, head size)
    "tiny": (4, 1, 64), "3b": (16, 2, 128), "7b": (28, 4, 128), "14b": (40, 8, 128),
}


def listed():
    return [
        # four short prompts of a toy model in fp32: launch-bound
        {"name": "prompt_f32_tiny", "kind": "prompt", "dtype": "f32", "heads": "tiny", "B": 4, "lo": 16, "hi": 200, "prefix": 0,
         "page": 0, "shape_seed": 1},
        # a batch of prompts of different lengths, packed, Q, K and V as the slices of one projection's output
        {"name": "prompt_7b_packed16", "kind": "prompt", "dtype": "bf16", "heads": "7b", "B": 16, "lo": 65, "hi": 2048, "prefix": 0,
         "page": 0, "shape_seed": 2},
        # the next 512 tokens of eight long prompts: written into the paged cache, then attended over all of it
        {"name": "chunk_14b_paged16_b8", "kind": "prompt", "dtype": "bf16", "heads": "14b", "B": 8, "lo": 512, "hi": 512,
         "prefix": 8192, "page": 16, "shape_seed": 3},
        # one long prompt
        {"name": "prompt_3b_16k", "kind": "prompt", "dtype": "bf16", "heads": "3b", "B": 1, "lo": 16384, "hi": 16384, "prefix": 0,
         "page": 0, "shape_seed": 4},
        # the end of a rollout: a few tokens with their 20 best alternatives
        {"name": "logprobs_8_top20", "kind": "logprobs", "dtype": "bf16", "rows": 8, "V": 151936, "top": 20, "T": 0.6, "entropy": True},
        # one verify step's rows (256 sequences, 3 drafts and one more)
        {"name": "logprobs_1024_top5", "kind": "logprobs", "dtype": "bf16", "rows": 1024, "V": 151936, "top": 5, "T": 1.0, "entropy": True},
        # fp32 rows that start at odd places
        {"name": "logprobs_f32_v50257_96", "kind": "logprobs", "dtype": "f32", "rows": 96, "V": 50257, "top": 1, "T": 0.4, "entropy": True},
        # the learner: log-probabilities and entropies of one batch of replayed rows, and the gradient of a loss over them
        {"name": "logprobs_step_2048", "kind": "logprobs_step", "dtype": "bf16", "rows": 2048, "V": 151936, "T": 1.0, "entropy": True},
        # the same in fp32 over a small vocabulary, without the entropy's part
        {"name": "logprobs_step_f32_64", "kind": "logprobs_step", "dtype": "f32", "rows": 64, "V": 32000, "T": 0.6, "entropy": False},
        # the next group of responses in a toy model's cache: the old group's pages given back, four children of two prompts
        {"name": "group_tiny_2x4", "kind": "group", "dtype": "f32", "heads": "tiny", "parents": 2, "children": 4, "lo": 40, "hi": 200,
         "grow": 8, "page": 16, "layers": 1, "shape_seed": 5},
        # 32 prompts, eight responses each, 7B heads, the pools of four layers
        {"name": "group_7b_32x8", "kind": "group", "dtype": "bf16", "heads": "7b", "parents": 32, "children": 8, "lo": 256, "hi": 4096,
         "grow": 64, "page": 64, "layers": 4, "shape_seed": 6},
        # a cache moved together after its rollouts have ended at different times
        {"name": "compact_7b_paged16_b256", "kind": "compact", "dtype": "bf16", "heads": "7b", "B": 256, "lo": 256, "hi": 4096, "page": 16,
         "spare": 1.6, "layers": 2, "shape_seed": 7},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    kind = rng.choice(["prompt", "prompt", "prompt", "logprobs", "logprobs", "logprobs_step", "group", "compact"])
    seed = rng.randrange(1 << 20)
    if kind == "prompt":
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        heads = rng.choice(["3b", "7b", "14b"] if dtype == "bf16" else ["tiny"])
        lo = _log_int(rng, 1, 512)
        hi = _log_int(rng, lo, 8192 if dtype == "bf16" else 1024)
        c = {"kind": kind, "dtype": dtype, "heads": heads, "B": _log_int(rng, 1, 32), "lo": lo, "hi": hi,
             "prefix": rng.choice([0, 0, _log_int(rng, 16, 16384 if dtype == "bf16" else 2048)]),
             "page": rng.choice([0, 16, 64, 256]), "shape_seed": seed}
        # no more scores in all (as a padded batch has them) than the largest listed case
        while c["B"] > 1 and c["B"] * hi * (hi + c["prefix"]) * HEADS[heads][0] > 16 * 16384 * 16384 / 2:
            c["B"] = c["B"] * 2 // 3
        return c
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind in ("logprobs", "logprobs_step"):
        V = rng.choice([151936, 32000, _log_int(rng, 1000, 152000)])
        c = {"kind": kind, "dtype": dtype, "rows": _log_int(rng, 1, 2048 if dtype == "bf16" else 1024), "V": V,
             "T": rng.choice([1.0, 0.6, 0.4])}
        c["entropy"] = rng.random() < 0.7
        if kind == "logprobs":
            c["top"] = rng.choice([0, 1, 5, 20, 32])
        return c
    heads = rng.choice(["tiny", "3b", "7b", "14b"])
    c = {"kind": kind, "dtype": dtype, "heads": heads, "lo": _log_int(rng, 1, 256), "hi": _log_int(rng, 256, 4096),
         "page": rng.choice([16, 64, 256]), "layers": rng.choice([1, 2, 4]), "shape_seed": seed}
    if kind == "group":
        return {**c, "parents": _log_int(rng, 1, 32), "children": _log_int(rng, 1, 16), "grow": _log_int(rng, 1, 256)}
    return {**c, "B": _log_int(rng, 2, 192), "spare": rng.uniform(1.1, 3.0), "layers": min(c["layers"], 2)}


# ------------------------------------------------------------------------------------ shapes
def _dt(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _size(case):
    return 4 if case["dtype"] == "f32" else 2


def _lengths(case, n, hi=None):
    """n lengths between lo and hi, spread over their logarithm; the same for every seed of a case."""
    rng = random.Random(case["shape_seed"])
    lo, hi = case["lo"], hi or case["hi"]
    return [min(hi, max(lo, _log_int(rng, lo, hi))) for _ in range(n)]


def _prompt_shape(case):
    """(new rows, cached tokens with them) of every prompt."""
    R = _lengths(case, case["B"])
    rng = random.Random(case["shape_seed"] + 1)
    pre = [rng.randrange(case["prefix"] // 8, case["prefix"] + 1) if case["prefix"] else 0 for _ in R]
    return R, [r + p for r, p in zip(R, pre)]


def _offsets(n, dtype, dev):
    return torch.tensor([0] + n, device=dev).cumsum(0).to(dtype)


# ------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev).manual_seed(seed)
    st = {"case": case, "dev": dev}
    {"prompt": _prepare_prompt, "logprobs": _prepare_logprobs, "logprobs_step": _prepare_logprobs, "group": _prepare_group,
     "compact": _prepare_compact}[case["kind"]](case, st, gen)
    return st


def _randn(shape, gen, dt):
    return torch.randn(shape, generator=gen, device=gen.device, dtype=torch.float32).to(dt)


def _prepare_prompt(case, st, gen):
    Hq, Hkv, D = HEADS[case["heads"]]
    dt, dev = _dt(case), st["dev"]
    R, L = _prompt_shape(case)
    st.update(R=R, L=L, B=case["B"], heads=(Hq, Hkv, D), scale=1.0 / math.sqrt(D), max_q=max(R), max_kv=max(L),
              q_indptr=_offsets(R, torch.int32, dev), total_q=sum(R))
    qkv = _randn((sum(R), Hq + 2 * Hkv, D), gen, dt)
    st["q"], st["k_new"], st["v_new"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    st["out"] = torch.empty((sum(R), Hq, D), dtype=dt, device=dev)
    st["lse"] = torch.empty((sum(R), Hq), dtype=torch.float32, device=dev)
    if case["page"]:
        ps = case["page"]
        pages = [-(-n // ps) for n in L]
        n = sum(pages) + 7
        order = torch.randperm(n, generator=torch.Generator().manual_seed(case["shape_seed"]))[:sum(pages)]
        st.update(k_pages=_randn((n, ps, Hkv, D), gen, dt), v_pages=_randn((n, ps, Hkv, D), gen, dt),
                  page_indptr=_offsets(pages, torch.int32, dev), page_table=order.to(torch.int32).to(dev),
                  kv_len=torch.tensor(L, dtype=torch.int32, device=dev))
        st["total_kv"] = n * ps
    elif case["prefix"]:  # the prompt's earlier tokens and the new ones, back to back
        kv = _randn((sum(L), 2 * Hkv, D), gen, dt)
        st["k"], st["v"] = kv[:, :Hkv], kv[:, Hkv:]
        st["total_kv"] = sum(L)
    else:
        st["k"], st["v"], st["total_kv"] = st["k_new"], st["v_new"], sum(R)
    st["kv_indptr"] = _offsets(L, torch.int64, dev)
    if own:
        from paper_2510_26475_amd import binding
        st["ws"] = torch.empty(binding.respec_prompt_attention_workspace_bytes(
            case["B"], sum(R), st["total_kv"], max(R), max(L), Hq, Hkv, D, int(case["dtype"] == "bf16")), dtype=torch.uint8, device=dev)


def _prepare_logprobs(case, st, gen):
    rows, V, dev = case["rows"], case["V"], st["dev"]
    st["logits"] = _randn((rows, V), gen, torch.float32).mul_(3.0).to(_dt(case))
    u = torch.rand((rows,), generator=gen, device=dev)
    best = st["logits"].argmax(dim=1).to(torch.int32)
    any_ = torch.randint(0, V, (rows,), generator=gen, device=dev, dtype=torch.int32)
    st["tokens"] = torch.where(u < 0.5, best, torch.where(u < 0.93, any_, torch.full_like(any_, -1)))  # -1: an unused slot
    f = dict(dtype=torch.float32, device=dev)
    st.update(logprob=torch.empty(rows, **f), lse=torch.empty(rows, **f), ent=torch.empty(rows, **f) if case["entropy"] else None)
    top = case.get("top", 0)
    st["top_tokens"] = torch.empty((rows, top), dtype=torch.int32, device=dev) if top else None
    st["top_logprobs"] = torch.empty((rows, top), **f) if top else None
    if case["kind"] == "logprobs_step":
        st["g_lp"] = torch.randn((rows,), generator=gen, device=dev)
        st["g_ent"] = 0.01 * torch.randn((rows,), generator=gen, device=dev) if case["entropy"] else None
        st["grad"] = torch.empty_like(st["logits"])
    if own:
        from paper_2510_26475_amd import binding
        st["ws"] = torch.empty(binding.respec_token_logprobs_workspace_bytes(rows, V, top, int(case["dtype"] == "bf16")),
                               dtype=torch.uint8, device=dev)


def _pools(case, num_pages, gen):
    _, Hkv, D = HEADS[case["heads"]]
    return [tuple(_randn((num_pages, case["page"], Hkv, D), gen, _dt(case)) for _ in range(2)) for _ in range(case["layers"])]


def _tables(held, cap, num_pages, seed):
    """Page tables of sequences that hold held[b] pages of cap[b] entries, in scattered order; counts of references."""
    order = torch.randperm(num_pages, generator=torch.Generator().manual_seed(seed))[:sum(held)].to(torch.int32)
    table = torch.full((sum(cap),), -1, dtype=torch.int32)
    at, used = 0, 0
    for h, c in zip(held, cap):
        table[at:at + h] = order[used:used + h]
        at, used = at + c, used + h
    refs = torch.zeros(num_pages, dtype=torch.int32)
    refs[order.long()] = 1
    return table, refs


def _prepare_group(case, st, gen):
    dev, ps, P, C = st["dev"], case["page"], case["parents"], case["children"]
    L = _lengths(case, P)
    B = P * (1 + C)                       # prompts first, then the children of each
    parent = [-1] * P + [p for p in range(P) for _ in range(C)]
    lens = L + [0] * (P * C)
    own_pages = [-(-n // ps) for n in L]
    cap = own_pages + [-(-(L[p] + case["grow"]) // ps) for p in parent[P:]]
    old = [min(2, c) for c in cap[P:]]    # what the group before this one still holds
    num_pages = sum(own_pages) + sum(old) + sum(1 + -(-case["grow"] // ps) + 1 for _ in parent[P:]) + 5
    table, refs = _tables(own_pages + old, cap, num_pages, case["shape_seed"])
    i32 = dict(dtype=torch.int32, device=dev)
    st.update(B=B, P=P, num_pages=num_pages, page_indptr=_offsets(cap, torch.int32, dev), page_table=table.to(dev), page_refs=refs.to(dev),
              page_count=torch.tensor(own_pages + old, **i32), kv_len=torch.tensor(lens[:P] + [o * ps for o in old], **i32),
              parent=torch.tensor(parent, **i32), give_back=torch.tensor([-1] * P + [0] * (P * C), **i32),
              want=torch.tensor([-1] * P + [L[p] + case["grow"] for p in parent[P:]], **i32),
              copy_src=torch.empty(B, **i32), copy_dst=torch.empty(B, **i32), missing=torch.empty(B, **i32), pools=_pools(case, num_pages, gen))
    if own:
        from paper_2510_26475_amd import binding
        st["ws"] = torch.empty(binding.respec_pages_workspace_bytes(B, num_pages), dtype=torch.uint8, device=dev)


def _prepare_compact(case, st, gen):
    dev, ps, B = st["dev"], case["page"], case["B"]
    held = [-(-n // ps) for n in _lengths(case, B)]
    cap = [h + 2 for h in held]
    num_pages = int(sum(held) * case["spare"]) + 3
    table, refs = _tables(held, cap, num_pages, case["shape_seed"])
    i32 = dict(dtype=torch.int32, device=dev)
    moves = num_pages // 2 + 1
    st.update(B=B, num_pages=num_pages, page_indptr=_offsets(cap, torch.int32, dev), page_table=table.to(dev), page_refs=refs.to(dev),
              page_count=torch.tensor(held, **i32), new_table=torch.empty(sum(cap), **i32), new_refs=torch.empty(num_pages, **i32),
              copy_src=torch.empty(moves, **i32), copy_dst=torch.empty(moves, **i32), num_live=torch.empty(1, **i32),
              pools=_pools(case, num_pages, gen))
    if own:
        from paper_2510_26475_amd import binding
        st["ws"] = torch.empty(binding.respec_pages_workspace_bytes(B, num_pages), dtype=torch.uint8, device=dev)


# ------------------------------------------------------------------------------------ one pass
def run(st):
    return {"prompt": _run_prompt, "logprobs": _run_logprobs, "logprobs_step": _run_logprobs_step, "group": _run_group,
            "compact": _run_compact}[st["case"]["kind"]](st)


def _run_prompt(st):
    paged = bool(st["case"]["page"])
    if own:
        from paper_2510_26475_amd import binding
        if paged:
            binding.respec_append_paged(st["k_new"], st["v_new"], st["k_pages"], st["v_pages"], st["q_indptr"], st["page_indptr"],
                                        st["page_table"], st["kv_len"], st["max_q"])
            binding.respec_prompt_attention_paged(st["q"], st["k_pages"], st["v_pages"], st["q_indptr"], st["page_indptr"],
                                                  st["page_table"], st["kv_len"], st["out"], st["lse"], st["max_q"], st["max_kv"],
                                                  st["scale"], st["ws"])
        else:
            binding.respec_prompt_attention(st["q"], st["k"], st["v"], st["q_indptr"], st["kv_indptr"], st["out"], st["lse"],
                                            st["max_q"], st["max_kv"], st["scale"], st["ws"])
    else:
        _plain_prompt(st)
    return {"out": st["out"], "lse": st["lse"], **({"k_pages": st["k_pages"], "v_pages": st["v_pages"]} if paged else {})}


def _plain_prompt(st):
    """The padded batch: rows and keys past a prompt's own are masked."""
    (Hq, Hkv, D), B, dev, Rm, Lm = st["heads"], st["B"], st["dev"], st["max_q"], st["max_kv"]
    q0, kv0 = st["q_indptr"].long(), st["kv_indptr"]
    R, L = q0[1:] - q0[:-1], kv0[1:] - kv0[:-1]
    i, j = torch.arange(Rm, device=dev), torch.arange(Lm, device=dev)
    row_ok, key_ok = i < R[:, None], j < L[:, None]
    rows = torch.where(row_ok, q0[:-1, None] + i, 0)
    if st["case"]["page"]:
        ps, table = st["case"]["page"], st["page_table"].long()
        entry = st["page_indptr"].long()[:-1, None] + torch.where(key_ok, j, 0) // ps
        slot = table[entry] * ps + torch.where(key_ok, j, 0) % ps
        new = torch.where(row_ok, (L - R)[:, None] + i, 0)
        to = torch.gather(slot, 1, new)[row_ok]
        kf, vf = (st[n].view(-1, Hkv, D) for n in ("k_pages", "v_pages"))
        kf[to], vf[to] = st["k_new"], st["v_new"]
    else:
        slot = torch.where(key_ok, kv0[:-1, None] + j, 0)
        kf, vf = st["k"], st["v"]
    q = st["q"][rows].float().view(B, Rm, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B * Hkv, -1, D)
    k = kf[slot].float().permute(0, 2, 3, 1).reshape(B * Hkv, D, Lm).contiguous()
    v = vf[slot].float().permute(0, 2, 1, 3).reshape(B * Hkv, Lm, D).contiguous()
    s = torch.bmm(q, k).mul_(st["scale"]).view(B, Hkv, Hq // Hkv, Rm, Lm)
    sees = key_ok[:, None, :] & (j <= (L - R)[:, None, None] + i[:, None])
    s.masked_fill_(~sees[:, None, None], -math.inf)
    m = s.amax(dim=-1, keepdim=True).clamp_(min=-3e38)
    p = s.sub_(m).exp_()
    l = p.sum(dim=-1, keepdim=True)
    o = torch.bmm(p.view(B * Hkv, -1, Lm), v).view(B, Hkv, Hq // Hkv, Rm, D).div_(l.clamp(min=1e-38))
    st["out"].copy_(o.permute(0, 3, 1, 2, 4).reshape(B, Rm, Hq, D)[row_ok])
    st["lse"].copy_((m + l.log()).permute(0, 3, 1, 2, 4).reshape(B, Rm, Hq)[row_ok])


def _run_logprobs(st):
    T = st["case"]["T"]
    if own:
        from paper_2510_26475_amd import binding
        binding.respec_token_logprobs(st["logits"], st["tokens"], st["logprob"], st["lse"], st["ent"], st["top_tokens"],
                                      st["top_logprobs"], T, st["ws"])
    else:
        st["logprob"], st["lse"], st["ent"] = _plain_logprobs(st, T)[:3]
        if st["case"]["top"]:
            used = (st["tokens"] >= 0)[:, None]
            z, ids = torch.sort(st["logits"], dim=1, descending=True, stable=True)
            n = st["case"]["top"]
            st["top_tokens"] = torch.where(used, ids[:, :n], -1).to(torch.int32)
            st["top_logprobs"] = torch.where(used, z[:, :n].float() / T - st["lse"][:, None], 0.0)
    names = ["logprob", "lse"] + (["ent"] if st["case"]["entropy"] else []) + (["top_tokens", "top_logprobs"] if st["case"]["top"] else [])
    return {n: st[n] for n in names}


def _plain_logprobs(st, T):
    used = st["tokens"] >= 0
    z = st["logits"].float() / T
    m = z.amax(dim=1, keepdim=True)
    e = (z - m).exp()
    total = e.sum(dim=1, keepdim=True)
    lse = m + total.log()
    lp = torch.gather(z, 1, st["tokens"].clamp(min=0).long()[:, None]) - lse
    p = e / total
    ent = total.log()[:, 0] - (p * (z - m)).sum(dim=1) if st["case"]["entropy"] else None
    zero = torch.zeros((), device=z.device)
    return (torch.where(used, lp[:, 0], zero), torch.where(used, lse[:, 0], zero),
            None if ent is None else torch.where(used, ent, zero), p, z - lse)


def _run_logprobs_step(st):
    T = st["case"]["T"]
    if own:
        from paper_2510_26475_amd import binding
        binding.respec_token_logprobs(st["logits"], st["tokens"], st["logprob"], st["lse"], st["ent"], None, None, T, st["ws"])
        binding.respec_token_logprobs_grad(st["logits"], st["tokens"], st["lse"], st["ent"], st["g_lp"], st["g_ent"], st["grad"], T)
    else:
        st["logprob"], st["lse"], st["ent"], p, log_p = _plain_logprobs(st, T)
        g = p * -st["g_lp"][:, None]
        if st["case"]["entropy"]:
            g -= st["g_ent"][:, None] * p * (log_p + st["ent"][:, None])
        at = st["tokens"].clamp(min=0).long()[:, None]
        g.scatter_add_(1, at, st["g_lp"][:, None])
        st["grad"].copy_(torch.where((st["tokens"] >= 0)[:, None], g / T, torch.zeros((), device=g.device)))
    return {n: st[n] for n in ["logprob", "lse", "grad"] + (["ent"] if st["case"]["entropy"] else [])}


def _run_group(st):
    names = ("page_table", "page_count", "kv_len", "page_refs", "copy_src", "copy_dst", "missing")
    if own:
        from paper_2510_26475_amd import binding
        s = (st["page_indptr"], st["page_table"], st["page_count"], st["kv_len"], st["page_refs"])
        ps = st["case"]["page"]
        binding.respec_pages_resize(st["give_back"], *s, st["copy_src"], st["copy_dst"], st["missing"], ps, st["ws"])
        binding.respec_pages_fork(st["parent"], *s, st["missing"])
        binding.respec_pages_resize(st["want"], *s, st["copy_src"], st["copy_dst"], st["missing"], ps, st["ws"])
        for k, v in st["pools"]:
            binding.respec_pages_copy(k, v, st["copy_src"], st["copy_dst"])
    else:
        _plain_resize(st, st["give_back"])
        _plain_fork(st)
        _plain_resize(st, st["want"])
        _plain_copy(st)
    return {**{n: st[n] for n in names}, "pools": st["pools"]}


def _places(st, first, count):
    """(sequence, entry of page_table, running number) of entries first[b] .. first[b]+count[b]-1 of every sequence."""
    seq = torch.repeat_interleave(torch.arange(st["B"], device=st["dev"]), count)
    nth = torch.arange(seq.numel(), device=st["dev"]) - (count.cumsum(0) - count)[seq]
    return seq, st["page_indptr"].long()[seq] + first[seq] + nth, nth


def _plain_resize(st, want):
    ps, table, refs = st["case"]["page"], st["page_table"], st["page_refs"]
    ip, count, kv, want = st["page_indptr"].long(), st["page_count"].long(), st["kv_len"].long(), want.long()
    pages = (want + ps - 1) // ps
    grow = torch.where(want >= 0, pages - count, 0).clamp(min=0)
    writes = (want > kv) & (kv % ps != 0) & (kv // ps < count)
    at = (ip[:-1] + kv // ps).clamp(max=table.numel() - 1)
    old = table[at].long()
    own_page = writes & (refs[old.clamp(min=0)] > 1)
    fits = pages <= ip[1:] - ip[:-1]
    need = grow + own_page
    free = (refs == 0).nonzero()[:, 0]
    begin = (need * fits).cumsum(0) - need * fits
    ok = fits & ((need == 0) | (begin + need <= free.numel()))
    st["missing"].copy_(torch.where(ok, 0, need))
    drop = torch.where(ok & (want >= 0), count - pages, 0).clamp(min=0)
    own_page, grow = own_page & ok, torch.where(ok, grow, 0)
    _, gone, _ = _places(st, count - drop, drop)
    refs.index_add_(0, table[gone].long(), torch.full_like(gone, -1, dtype=torch.int32))
    table[gone] = -1
    st["copy_src"].copy_(torch.where(own_page, old, -1))
    fresh = free[begin[own_page]]
    st["copy_dst"].fill_(-1)
    st["copy_dst"][own_page] = fresh.to(torch.int32)
    refs.index_add_(0, old[own_page], torch.full_like(fresh, -1, dtype=torch.int32))
    table[at[own_page]] = fresh.to(torch.int32)
    refs[fresh] = 1
    seq, new, nth = _places(st, count, grow)
    fresh = free[begin[seq] + own_page[seq] + nth]
    table[new] = fresh.to(torch.int32)
    refs[fresh] = 1
    st["page_count"].copy_(count + grow - drop)
    st["kv_len"].copy_(torch.where(ok & (want >= 0), torch.minimum(kv, want), kv))


def _plain_fork(st):
    parent = st["parent"].long()
    child = parent >= 0
    count = torch.where(child, st["page_count"].long()[parent.clamp(min=0)], 0)
    seq, to, nth = _places(st, torch.zeros_like(count), count)
    page = st["page_table"][st["page_indptr"].long()[parent[seq]] + nth]
    st["page_table"][to] = page
    st["page_refs"].index_add_(0, page.long(), torch.ones_like(page))
    st["page_count"].copy_(torch.where(child, count, st["page_count"].long()))
    st["kv_len"].copy_(torch.where(child, st["kv_len"][parent.clamp(min=0)], st["kv_len"]))
    st["missing"].zero_()


def _plain_copy(st):
    used = st["copy_src"] >= 0
    src, dst = st["copy_src"][used].long(), st["copy_dst"][used].long()
    for k, v in st["pools"]:
        k[dst], v[dst] = k[src], v[src]


def _run_compact(st):
    if own:
        from paper_2510_26475_amd import binding
        binding.respec_pages_compact(st["page_table"], st["page_refs"], st["new_table"], st["new_refs"], st["copy_src"],
                                     st["copy_dst"], st["num_live"], st["ws"])
        for k, v in st["pools"]:
            binding.respec_pages_copy(k, v, st["copy_src"], st["copy_dst"])
    else:
        refs = st["page_refs"]
        live = refs > 0
        n = live.sum()
        low = torch.arange(st["num_pages"], device=st["dev"]) < n
        src = (live & ~low).nonzero()[:, 0].flip(0)
        dst = (~live & low).nonzero()[:, 0]
        st["copy_src"].fill_(-1)
        st["copy_dst"].fill_(-1)
        st["copy_src"][:src.numel()] = src.to(torch.int32)
        st["copy_dst"][:dst.numel()] = dst.to(torch.int32)
        st["num_live"].copy_(n)
        to = torch.arange(st["num_pages"], device=st["dev"], dtype=torch.int32)
        to[src] = dst.to(torch.int32)
        st["new_refs"].copy_(refs)
        st["new_refs"][dst] = refs[src]
        st["new_refs"][src] = 0
        _, at, _ = _places(st, torch.zeros_like(st["page_count"]).long(), st["page_count"].long())
        st["new_table"].copy_(st["page_table"])
        st["new_table"][at] = to[st["page_table"][at].long()]
        _plain_copy(st)
    return {n: st[n] for n in ("new_table", "new_refs", "copy_src", "copy_dst", "num_live", "pools")}


# ------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    if case["kind"] == "prompt":
        return _exact_prompt(st)
    if case["kind"] in ("logprobs", "logprobs_step"):
        return _exact_logprobs(st)
    return _exact_group(st) if case["kind"] == "group" else _exact_compact(st)


def _exact_prompt(st):
    (Hq, Hkv, D), case = st["heads"], st["case"]
    out = torch.empty((st["total_q"], Hq, D), dtype=torch.float64, device=st["dev"])
    lse = torch.empty((st["total_q"], Hq), dtype=torch.float64, device=st["dev"])
    r0 = l0 = p0 = 0
    for R, L in zip(st["R"], st["L"]):
        if case["page"]:
            n = -(-L // case["page"])
            ids = st["page_table"][p0:p0 + n].long()
            for name, new in (("k_pages", "k_new"), ("v_pages", "v_new")):
                flat = st[name][ids].flatten(0, 1)
                flat[L - R:L] = st[new][r0:r0 + R]
                st[name][ids] = flat.view(n, case["page"], Hkv, D)
            k, v = (st[x][ids].flatten(0, 1)[:L].double() for x in ("k_pages", "v_pages"))
            p0 += n
        else:
            k, v = st["k"][l0:l0 + L].double(), st["v"][l0:l0 + L].double()
        l0 += L
        hidden = torch.arange(L, device=st["dev"])[None, :] > (L - R) + torch.arange(R, device=st["dev"])[:, None]
        for h in range(Hq):
            s = st["q"][r0:r0 + R, h].double() @ k[:, h * Hkv // Hq].t().contiguous() * st["scale"]
            s[hidden] = -math.inf
            z = torch.logsumexp(s, dim=1)
            lse[r0:r0 + R, h] = z
            out[r0:r0 + R, h] = torch.exp(s - z[:, None]) @ v[:, h * Hkv // Hq]
        r0 += R
    res = {"out": out, "lse": lse}
    return {**res, "k_pages": None, "v_pages": None} if case["page"] else res


def _exact_logprobs(st):
    case, T, rows = st["case"], st["case"]["T"], st["case"]["rows"]
    f64 = dict(dtype=torch.float64, device=st["dev"])
    res = {"logprob": torch.zeros(rows, **f64), "lse": torch.zeros(rows, **f64)}
    if case["entropy"]:
        res["ent"] = torch.zeros(rows, **f64)
    if case.get("top"):
        res.update(top_tokens=None, top_logprobs=torch.zeros((rows, case["top"]), **f64))
    if case["kind"] == "logprobs_step":
        res["grad"] = torch.zeros((rows, case["V"]), **f64)
    for a in range(0, rows, 64):
        tok = st["tokens"][a:a + 64].long()
        z = st["logits"][a:a + 64].double() / T
        log_p = torch.log_softmax(z, dim=1)
        p = log_p.exp()
        H = -(p * log_p).sum(dim=1)
        part = {"logprob": log_p.gather(1, tok.clamp(min=0)[:, None])[:, 0], "lse": torch.logsumexp(z, dim=1), "ent": H}
        if case.get("top"):
            part["top_logprobs"] = log_p.topk(case["top"], dim=1).values
        if case["kind"] == "logprobs_step":
            hit = torch.zeros_like(p).scatter_(1, tok.clamp(min=0)[:, None], 1.0)
            g = st["g_lp"][a:a + 64, None].double() * (hit - p)
            if case["entropy"]:
                g -= st["g_ent"][a:a + 64, None].double() * p * (log_p + H[:, None])
            part["grad"] = g / T
        for n in part:
            if n in res:
                res[n][a:a + 64][tok >= 0] = part[n][tok >= 0]
    return res


def _host(st, *names):
    return [st[n].tolist() for n in names]


def _like(st, **lists):
    return {n: torch.tensor(v, dtype=torch.int32, device=st["dev"]) for n, v in lists.items()}


def _copied(st, src, dst):
    for a, b in zip(src, dst):
        if a >= 0:
            for k, v in st["pools"]:
                k[b], v[b] = k[a], v[a]
    return [(k.double(), v.double()) for k, v in st["pools"]]


def _exact_group(st):
    """The group's pages one sequence after another, with a free list that each call takes at its beginning."""
    ps, B = st["case"]["page"], st["B"]
    ip, table, count, kv, refs, parent = _host(st, "page_indptr", "page_table", "page_count", "kv_len", "page_refs", "parent")

    def resize(want):
        free = [i for i, r in enumerate(refs) if r == 0]
        before, src, dst, missing = list(refs), [-1] * B, [-1] * B, [0] * B
        at = 0
        for b in range(B):
            if want[b] < 0:
                continue
            n = -(-want[b] // ps)
            split = want[b] > kv[b] and kv[b] % ps and kv[b] // ps < count[b] and before[table[ip[b] + kv[b] // ps]] > 1
            need = max(n - count[b], 0) + int(bool(split))
            if n > ip[b + 1] - ip[b]:
                missing[b] = need
                continue
            mine, at = free[at:at + need], at + need
            if len(mine) < need:
                missing[b] = need
                continue
            for e in range(n, count[b]):
                refs[table[ip[b] + e]] -= 1
                table[ip[b] + e] = -1
            if split:
                e = ip[b] + kv[b] // ps
                src[b], dst[b] = table[e], mine.pop(0)
                refs[table[e]] -= 1
                table[e], refs[dst[b]] = dst[b], 1
            for e in range(count[b], n):
                table[ip[b] + e] = mine.pop(0)
                refs[table[ip[b] + e]] = 1
            count[b], kv[b] = n, min(kv[b], want[b])
        return src, dst, missing

    resize(st["give_back"].tolist())
    for b, p in enumerate(parent):
        if p >= 0:
            for e in range(count[p]):
                table[ip[b] + e] = table[ip[p] + e]
                refs[table[ip[p] + e]] += 1
            count[b], kv[b] = count[p], kv[p]
    src, dst, missing = resize(st["want"].tolist())
    return {**_like(st, page_table=table, page_count=count, kv_len=kv, page_refs=refs, copy_src=src, copy_dst=dst, missing=missing),
            "pools": _copied(st, src, dst)}


def _exact_compact(st):
    table, refs = _host(st, "page_table", "page_refs")
    live = [i for i, r in enumerate(refs) if r > 0]
    low = [i for i, r in enumerate(refs) if r == 0 and i < len(live)]
    moved = dict(zip(reversed([i for i in live if i >= len(live)]), low))
    new_refs = list(refs)
    for a, b in moved.items():
        new_refs[a], new_refs[b] = 0, refs[a]
    pad = [-1] * (st["copy_src"].numel() - len(moved))
    src, dst = list(moved) + pad, list(moved.values()) + pad
    return {**_like(st, new_table=[moved.get(e, e) for e in table], new_refs=new_refs, copy_src=src, copy_dst=dst, num_live=[len(live)]),
            "pools": _copied(st, src, dst)}


# ------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["kind"] == "prompt":
        Hq, Hkv, D = HEADS[case["heads"]]
        R, L = _prompt_shape(case)
        pairs = sum(r * (2 * n - r + 1) // 2 for r, n in zip(R, L))
        tokens = sum(L) + (2 * sum(R) if case["page"] else 0)  # (new tokens are read and written once more on their way into the pages)
        return {"bytes": 2 * sum(R) * Hq * D * _size(case) + 2 * tokens * Hkv * D * _size(case) + 4 * sum(R) * Hq, "flops": 4 * D * Hq * pairs}
    if case["kind"] in ("logprobs", "logprobs_step"):
        n = case["rows"] * case["V"]
        step = case["kind"] == "logprobs_step"
        return {"bytes": n * _size(case) * (2 if step else 1) + case["rows"] * (16 + 8 * case.get("top", 0)), "flops": n * (10 if step else 6)}
    _, Hkv, D = HEADS[case["heads"]]
    page = 2 * case["page"] * Hkv * D * _size(case) * case["layers"]  # K and V
    if case["kind"] == "group":
        L, C = _lengths(case, case["parents"]), case["children"]
        copies = C * sum(n % case["page"] != 0 for n in L)
        entries = C * sum(-(-n // case["page"]) for n in L)
        return {"bytes": 2 * copies * page + 8 * entries, "flops": 0}
    held = sum(-(-n // case["page"]) for n in _lengths(case, case["B"]))
    total = int(held * case["spare"]) + 3
    moved = held * (total - held) // total  # expected: pages lie at random places
    return {"bytes": 2 * moved * page + 8 * (total + held), "flops": 0}
