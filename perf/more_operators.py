"""The K/V cache of a rollout as timed cases: written by a forward, kept in 8 bits, read once for all responses of a group.

A layer of the target's forward normalises and rotates the heads of Q and K and puts K and V into the pages of the cache ("write"); a cache
of 8 bits halves what the verify attention reads ("attend" without groups) and is read back where a prompt's next chunk needs it whole; the
responses of a group hold the same pages of their prompt, which the attention then reads once for all of them ("attend" with groups).  "step" is
a plain decoding step of some layers: one token per sequence through both.  Heads, page sizes, lengths and draft shapes are those of the package's
own workloads.

A case names its shape by plain values; lengths are part of the shape (drawn from `shape_seed`).  Where `own` is true the package's calls run,
else plain torch operations in 32 bits (angles in 64).
"""
from __future__ import annotations

import math
import random

import torch

own = False

HEADS = {  # (query heads, KV heads, head size)
    "tiny": (4, 1, 64), "3b": (16, 2, 128), "7b": (28, 4, 128), "14b": (40, 8, 128),
}
EPS = 1e-6

WRITE = {"kind": "write", "tree": "", "norm": True, "rotary": "half", "part": 1.0, "pool": "same", "page": 16}
ATTEND = {"kind": "attend", "groups": 0, "per": 0, "shared_lo": 0, "shared_hi": 0, "tree": "", "layers": 1, "page": 16}


def listed():
    return [
        # one token of each of four toy sequences in fp32: launch-bound
        {**WRITE, "name": "write_f32_tiny", "dtype": "f32", "heads": "tiny", "B": 4, "lo": 1, "hi": 1, "prefix": 300, "shape_seed": 1},
        # the new tokens of one verify step (256 sequences, three drafts and one more)
        {**WRITE, "name": "write_7b_b256_k3", "dtype": "bf16", "heads": "7b", "B": 256, "lo": 4, "hi": 4, "prefix": 1024, "shape_seed": 2},
        # the next 512 tokens of eight long prompts into a cache of 8 bits, and the whole of it back for their attention
        {**WRITE, "name": "write_14b_chunk8_e4m3", "dtype": "bf16", "heads": "14b", "B": 8, "lo": 512, "hi": 512, "prefix": 8192, "pool": "e4m3",
         "shape_seed": 3},
        # a long prompt and some shorter ones without norms, pairs side by side, half of each head rotated
        {**WRITE, "name": "write_3b_prompts_pairs", "dtype": "bf16", "heads": "3b", "B": 6, "lo": 512, "hi": 16384, "prefix": 0, "norm": False,
         "rotary": "pairs", "part": 0.5, "page": 64, "shape_seed": 4},
        # the end of a rollout over a cache of 8 bits: a few long responses, latency
        {**ATTEND, "name": "attend_3b_b8_k4_e4m3", "dtype": "bf16", "pool": "e4m3", "heads": "3b", "B": 8, "k": 4, "lo": 512, "hi": 4096, "shape_seed": 5},
        # the ordinary verify step of a rollout batch over a cache of 8 bits
        {**ATTEND, "name": "attend_7b_b256_k3_e4m3", "dtype": "bf16", "pool": "e4m3", "heads": "7b", "B": 256, "k": 3, "lo": 512, "hi": 4096, "shape_seed": 6},
        # trees of drafts, three levels of two candidates
        {**ATTEND, "name": "attend_14b_b96_tree3x2_e4m3", "dtype": "bf16", "pool": "e4m3", "heads": "14b", "B": 96, "k": 6, "tree": "3x2", "lo": 256, "hi": 8192,
         "page": 64, "shape_seed": 7},
        # two toy prompts with four responses each in fp32: launch-bound
        {**ATTEND, "name": "shared_f32_tiny_2x4", "dtype": "f32", "pool": "same", "heads": "tiny", "groups": 2, "per": 4, "B": 8, "k": 3, "shared_lo": 64,
         "shared_hi": 200, "lo": 1, "hi": 60, "shape_seed": 8},
        # 32 prompts with eight responses each, two layers of one forward
        {**ATTEND, "name": "shared_7b_32x8_k3", "dtype": "bf16", "pool": "same", "heads": "7b", "groups": 32, "per": 8, "B": 256, "k": 3, "shared_lo": 256,
         "shared_hi": 4096, "lo": 16, "hi": 1024, "page": 64, "layers": 2, "shape_seed": 9},
        # sixteen responses to each of eight long prompts, in 8 bits, and some sequences by themselves
        {**ATTEND, "name": "shared_14b_8x16_e4m3", "dtype": "bf16", "pool": "e4m3", "heads": "14b", "groups": 8, "per": 16, "B": 136, "k": 4, "shared_lo": 2048,
         "shared_hi": 8192, "lo": 64, "hi": 2048, "shape_seed": 10},
        # one very long prompt, 64 responses, a token each
        {**ATTEND, "name": "shared_7b_1x64_decode", "dtype": "bf16", "pool": "same", "heads": "7b", "groups": 1, "per": 64, "B": 64, "k": 0, "shared_lo": 16384,
         "shared_hi": 16384, "lo": 16, "hi": 512, "page": 64, "shape_seed": 11},
        # plain decoding, four layers: one token of each sequence into the cache of 8 bits and its attention
        {**ATTEND, "kind": "step", "name": "step_7b_b32_e4m3", "dtype": "bf16", "pool": "e4m3", "heads": "7b", "B": 32, "k": 0, "lo": 256, "hi": 4096, "layers": 4,
         "norm": True, "rotary": "half", "part": 1.0, "shape_seed": 12},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    kind = rng.choice(["write", "write", "attend", "attend", "shared", "shared", "shared", "step"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    heads = rng.choice(["tiny", "3b", "7b", "14b"] if dtype == "bf16" else ["tiny", "tiny", "3b"])
    c = {"dtype": dtype, "heads": heads, "page": rng.choice([16, 64, 256]), "shape_seed": rng.randrange(1 << 20),
         "pool": rng.choice(["same", "e4m3"]) if dtype == "bf16" else "same", "tree": rng.choice(["", "", "", "2x2", "3x2", "4x3"])}
    turn = {"norm": rng.random() < 0.7, "rotary": rng.choice(["half", "half", "pairs"]), "part": rng.choice([1.0, 1.0, 0.5, 0.25])}
    if kind == "write":
        lo = _log_int(rng, 1, 512)
        hi = _log_int(rng, lo, 8192)
        c.update(turn, kind="write", B=_log_int(rng, 1, 256), lo=lo, hi=hi, prefix=rng.choice([0, _log_int(rng, 16, 8192)]), tree="")
        while c["B"] > 1 and work(c)["bytes"] > 300e6:
            c["B"] = c["B"] * 2 // 3
        return c
    c["k"] = _tree_rows(c) - 1 if c["tree"] else rng.choice([0, 1, 2, 3, 4, 5, 8])
    lo = _log_int(rng, 1, 512)
    c.update(kind="attend", layers=rng.choice([1, 1, 2]), lo=lo, hi=_log_int(rng, lo, 4096), groups=0, per=0, shared_lo=0, shared_hi=0)
    if kind == "shared":
        low = _log_int(rng, 16, 2048)
        c.update(groups=_log_int(rng, 1, 32), per=_log_int(rng, 1, 32), shared_lo=low, shared_hi=_log_int(rng, low, 16384))
        c["B"] = c["groups"] * c["per"] + rng.choice([0, 0, rng.randrange(1, 9)])
    else:
        c["B"] = _log_int(rng, 1, 256)
        if dtype == "bf16":
            c["pool"] = "e4m3"
        else:  # (a cache of 8 bits is read by bf16 queries: in fp32 a group takes its place)
            c.update(groups=1, per=c["B"], shared_lo=32, shared_hi=512)
    if kind == "step":
        c.update(turn, kind="step", tree="", k=0, layers=rng.choice([1, 2, 4]))
    # no more padded keys, over all layers, and no more bytes and operations than the largest listed cases
    def large():
        padded = c["layers"] * c["B"] * (c["hi"] + c["shared_hi"]) * HEADS[heads][1] * HEADS[heads][2]
        return padded > 2 * 256 * 5120 * 4 * 128 or work(c)["bytes"] > 450e6 or work(c)["flops"] > 60e9

    while large() and (c["B"] > 1 or c["layers"] > 1):
        if c["layers"] > 1:
            c["layers"] //= 2
        elif c["groups"]:
            extra = c["B"] - c["groups"] * c["per"]
            if c["groups"] > 1:
                c["groups"] = c["groups"] * 2 // 3
            else:
                c["per"] = max(1, c["per"] * 2 // 3)
                extra = 0
            c["B"] = c["groups"] * c["per"] + extra
        else:
            c["B"] = c["B"] * 2 // 3
    return c


# ------------------------------------------------------------------------------------ shapes
def _dt(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _size(case):
    return 4 if case["dtype"] == "f32" else 2


def _pool_token(case):
    """Bytes of K and V of one token."""
    _, Hkv, D = HEADS[case["heads"]]
    return 2 * Hkv * ((D + 1) if case["pool"] == "e4m3" else D * _size(case))


def _lengths(case, n, lo, hi, turn=0):
    """n lengths between lo and hi, spread over their logarithm; the same for every seed of a case."""
    rng = random.Random(case["shape_seed"] * 8 + turn)
    return [min(hi, max(lo, _log_int(rng, lo, hi))) for _ in range(n)]


def _tree_rows(case):
    depth, branch = (int(x) for x in case["tree"].split("x"))
    return 1 + depth * branch


def _tree_parents(case):
    """`branch` candidates on each level, the children of the first candidate of the level before."""
    depth, branch = (int(x) for x in case["tree"].split("x"))
    parent, last = [-1], 0
    for _ in range(depth):
        first = len(parent)
        parent += [last] * branch
        last = first
    return parent


def _write_shape(case):
    """(new tokens, tokens held with them) of every sequence."""
    R = _lengths(case, case["B"], case["lo"], case["hi"])
    rng = random.Random(case["shape_seed"] + 1)
    return R, [r + (rng.randrange(case["prefix"] // 8, case["prefix"] + 1) if case["prefix"] else 0) for r in R]


def _attend_shape(case):
    """(rows, tokens held, tokens shared) of every sequence: groups first, then sequences by themselves; shared tokens fill whole pages."""
    r, ps = case["k"] + 1, case["page"]
    own_tokens = _lengths(case, case["B"], case["lo"], case["hi"])
    prompts = _lengths(case, case["groups"], case["shared_lo"], case["shared_hi"], 1) if case["groups"] else []
    S = [p // ps * ps for p in prompts for _ in range(case["per"])]
    S += [0] * (case["B"] - len(S))
    of = [p for p in prompts for _ in range(case["per"])] + [0] * (case["B"] - len(prompts) * case["per"])
    return [r] * case["B"], [p + n + r for p, n in zip(of, own_tokens)], S


def _offsets(n, dtype, dev):
    return torch.tensor([0] + n, device=dev).cumsum(0).to(dtype)


# ------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev).manual_seed(seed)
    Hq, Hkv, D = HEADS[case["heads"]]
    st = {"case": case, "dev": dev, "heads": (Hq, Hkv, D), "scale": 1.0 / math.sqrt(D), "B": case["B"]}
    if case["kind"] == "write":
        st["R"], st["L"] = _write_shape(case)
        st["S"] = [0] * case["B"]
    else:
        st["R"], st["L"], st["S"] = _attend_shape(case)
    R, L = st["R"], st["L"]
    st.update(total_q=sum(R), max_q=max(R), max_kv=max(L), q_indptr=_offsets(R, torch.int32, dev), kv_indptr=_offsets(L, torch.int64, dev),
              kv_len=torch.tensor(L, dtype=torch.int32, device=dev))
    _prepare_tables(case, st)
    st["layers"] = [_prepare_layer(case, st, gen) for _ in range(case.get("layers", 1))]
    if case["kind"] != "attend":
        rot = int(D * case["part"])
        st["inv_freq"] = (1e6 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).to(torch.float32).to(dev)
    if case["tree"]:
        masks = []
        for i, p in enumerate(_tree_parents(case)):
            masks.append((masks[p] if p >= 0 else 0) | 1 << i)
        st["tree_mask"] = torch.tensor(masks * case["B"], dtype=torch.int64, device=dev)
    if case["kind"] == "write" and case["pool"] == "e4m3":
        st["k_back"], st["v_back"] = (torch.empty((sum(L), Hkv, D), dtype=_dt(case), device=dev) for _ in range(2))
    if case["kind"] != "write" and own:
        from paper_2510_26475_amd import binding
        st["ws"] = torch.empty(binding.respec_verify_attention_shared_workspace_bytes(
            case["B"], sum(R), case["groups"], max(R), max(L), Hq, Hkv, D, int(case["dtype"] == "bf16")), dtype=torch.uint8, device=dev)
    return st


def _prepare_tables(case, st):
    """Pages in scattered order; the members of a group name the same ones for the tokens they share."""
    ps, dev, per = case["page"], st["dev"], case.get("per", 0)
    held = [-(-n // ps) for n in st["L"]]
    shared = [n // ps for n in st["S"]]
    fresh, entries = 0, []
    for b in range(case["B"]):
        first = b - b % per if per and b < case["groups"] * per else b
        if first == b:
            mine = list(range(fresh, fresh + held[b]))
            fresh += held[b]
        else:
            mine = entries[first][:shared[b]] + list(range(fresh, fresh + held[b] - shared[b]))
            fresh += held[b] - shared[b]
        entries.append(mine)
    st["num_pages"] = fresh + 3
    order = torch.randperm(st["num_pages"], generator=torch.Generator().manual_seed(case["shape_seed"]))
    st["page_table"] = order[torch.tensor([e for mine in entries for e in mine])].to(torch.int32).to(dev)
    st["page_indptr"] = _offsets(held, torch.int32, dev)
    if case.get("groups"):
        st["group_indptr"] = torch.arange(0, case["groups"] + 1, dtype=torch.int32, device=dev) * per
        st["shared_len"] = torch.tensor(st["S"][0:case["groups"] * per:per], dtype=torch.int32, device=dev)


def _randn(shape, gen, dt):
    return torch.randn(shape, generator=gen, device=gen.device, dtype=torch.float32).to(dt)


def _prepare_layer(case, st, gen):
    (Hq, Hkv, D), dt, dev = st["heads"], _dt(case), st["dev"]
    y = {}
    shape = (st["num_pages"], case["page"], Hkv, D)
    y["k_pages"], y["v_pages"] = (_randn(shape, gen, dt) for _ in range(2))
    y["k_scale"] = y["v_scale"] = None
    if case["pool"] == "e4m3":
        for n in "kv":
            code, e = _quantise(y[n + "_pages"].float())
            y[n + "_pages"], y[n + "_scale"] = code, e.transpose(1, 2).contiguous()
    if case["kind"] == "attend":
        y["q"] = _randn((st["total_q"], Hq, D), gen, dt)
    else:  # the slices of one projection's output
        qkv = _randn((st["total_q"], Hq + 2 * Hkv, D), gen, dt)
        y["q_new"], y["k_new"], y["v_new"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        y["q"] = torch.empty((st["total_q"], Hq, D), dtype=dt, device=dev)
        y["q_weight"], y["k_weight"] = ((1.0 + 0.2 * _randn((D,), gen, torch.float32)) if case["norm"] else None for _ in range(2))
    if case["kind"] != "write":
        y["out"] = torch.empty((st["total_q"], Hq, D), dtype=dt, device=dev)
        y["lse"] = torch.empty((st["total_q"], Hq), dtype=torch.float32, device=dev)
    return y


def _quantise(x):
    """Codes of e4m3 and the exponent byte of the power of two that they are multiplied by: the least one that the largest magnitude
    of a token's head does not exceed 448 times."""
    m, e = torch.frexp(x.abs().amax(dim=-1))
    e = (e.to(torch.int32) - 9 + (m > 0.875)).clamp(-126, 127)
    return (x * _power(127 - e)[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _power(byte):
    """2^(byte - 127) in fp32, by its bits."""
    return (byte.to(torch.int32) << 23).view(torch.float32)


def _values(code, scale):
    """What codes [..., Hkv, D] with exponent bytes [..., Hkv] stand for."""
    return code.to(torch.float32) * _power(scale)[..., None]


# ------------------------------------------------------------------------------------ one pass
def run(st):
    case = st["case"]
    for i, y in enumerate(st["layers"]):
        if case["kind"] != "attend":
            _write(st, y)
        if case["kind"] != "write":
            _attend(st, y, i)
    if case["kind"] == "write":
        y = st["layers"][0]
        if case["pool"] == "e4m3":
            _read_back(st, y)
            return {"q": y["q"], "k": st["k_back"], "v": st["v_back"]}
        return {"q": y["q"], "k_pages": y["k_pages"], "v_pages": y["v_pages"]}
    names = ("out", "lse") + (("q",) if case["kind"] == "step" else ())
    return [{n: y[n] for n in names} for y in st["layers"]]


def _tables(st):
    return st["q_indptr"], st["page_indptr"], st["page_table"], st["kv_len"]


def _write(st, y):
    if own:
        from paper_2510_26475_amd import binding
        binding.respec_norm_rope_append_paged(y["q_new"], y["k_new"], y["v_new"], y["q_weight"], y["k_weight"], st["inv_freq"], None, y["q"],
                                              y["k_pages"], y["v_pages"], y["k_scale"], y["v_scale"], *_tables(st), st["max_q"], EPS,
                                              interleaved=st["case"]["rotary"] == "pairs")
        return
    B, dev, ps = st["B"], st["dev"], st["case"]["page"]
    q0 = st["q_indptr"].long()
    R, L = q0[1:] - q0[:-1], st["kv_len"].long()
    seq = torch.repeat_interleave(torch.arange(B, device=dev), R)
    pos = (L - R)[seq] + torch.arange(st["total_q"], device=dev) - q0[:-1][seq]
    y["q"].copy_(_turned(st, y["q_new"].float(), y["q_weight"], pos))
    page = st["page_table"].long()[st["page_indptr"].long()[seq] + pos // ps]
    for n, x in (("k", _turned(st, y["k_new"].float(), y["k_weight"], pos)), ("v", y["v_new"].float())):
        if st["case"]["pool"] == "e4m3":
            code, e = _quantise(x)
            y[n + "_pages"].view(torch.uint8)[page, pos % ps] = code.view(torch.uint8)
            y[n + "_scale"][page, :, pos % ps] = e
        else:
            y[n + "_pages"][page, pos % ps] = x.to(y[n + "_pages"].dtype)


def _turned(st, x, weight, pos):
    """Heads normalised by their root mean square and rotated."""
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * weight
    rot = 2 * st["inv_freq"].numel()
    angle = pos.double()[:, None, None] * st["inv_freq"].double()
    cos, sin = angle.cos().to(x.dtype), angle.sin().to(x.dtype)
    out = x.clone()
    if st["case"]["rotary"] == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        out[..., :rot // 2], out[..., rot // 2:rot] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        out[..., 0:rot:2], out[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
    return out


def _read_back(st, y):
    if own:
        from paper_2510_26475_amd import binding
        binding.respec_read_paged_quantised(y["k_pages"], y["v_pages"], y["k_scale"], y["v_scale"], st["page_indptr"], st["page_table"], st["kv_len"],
                                            st["kv_indptr"], st["k_back"], st["v_back"], st["max_kv"])
        return
    kv0, ps = st["kv_indptr"], st["case"]["page"]
    seq = torch.repeat_interleave(torch.arange(st["B"], device=st["dev"]), kv0[1:] - kv0[:-1])
    pos = torch.arange(seq.numel(), device=st["dev"]) - kv0[:-1][seq]
    page = st["page_table"].long()[st["page_indptr"].long()[seq] + pos // ps]
    for n in "kv":
        code = y[n + "_pages"].view(torch.uint8)[page, pos % ps].view(torch.float8_e4m3fn)
        st[n + "_back"].copy_(_values(code, y[n + "_scale"][page, :, pos % ps]))


def _attend(st, y, layer):
    if own:
        from paper_2510_26475_amd import binding
        args = (*_tables(st), st.get("group_indptr"), st.get("shared_len"), st.get("tree_mask"), y["out"], y["lse"], st["max_q"], st["max_kv"],
                st["scale"], st["ws"])
        call = binding.respec_verify_attention_shared_next_layer if layer else binding.respec_verify_attention_shared
        call(y["q"], y["k_pages"], y["v_pages"], y["k_scale"], y["v_scale"], *args)
        return
    # the padded batch: rows and keys past a sequence's own are masked
    (Hq, Hkv, D), B, dev, Rm, Lm, ps = st["heads"], st["B"], st["dev"], st["max_q"], st["max_kv"], st["case"]["page"]
    q0 = st["q_indptr"].long()
    R, L = q0[1:] - q0[:-1], st["kv_len"].long()
    i, j = torch.arange(Rm, device=dev), torch.arange(Lm, device=dev)
    key_ok = j < L[:, None]
    at = torch.where(key_ok, j, 0)
    page = st["page_table"].long()[st["page_indptr"].long()[:-1, None] + at // ps]
    if st["case"]["pool"] == "e4m3":
        k, v = (_values(y[n + "_pages"].view(torch.uint8)[page, at % ps].view(torch.float8_e4m3fn), y[n + "_scale"][page, :, at % ps]) for n in "kv")
    else:
        k, v = (y[n + "_pages"][page, at % ps].float() for n in "kv")
    rows = torch.where(i < R[:, None], q0[:-1, None] + i, 0)
    q = y["q"][rows].float().view(B, Rm, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B * Hkv, -1, D)
    k = k.permute(0, 2, 3, 1).reshape(B * Hkv, D, Lm).contiguous()
    v = v.permute(0, 2, 1, 3).reshape(B * Hkv, Lm, D).contiguous()
    s = torch.bmm(q, k).mul_(st["scale"]).view(B, Hkv, Hq // Hkv, Rm, Lm)
    new = j - (L - R)[:, None]                                # the number of a key among a sequence's new tokens
    if st["case"]["tree"]:
        bit = (st["tree_mask"].view(B, Rm)[:, :, None] >> new.clamp(0, 62)[:, None, :]) & 1
        sees = key_ok[:, None, :] & ((new < 0)[:, None, :] | (bit == 1))
    else:
        sees = key_ok[:, None, :] & (new[:, None, :] <= i[None, :, None])
    s.masked_fill_(~sees[:, None, None], -math.inf)
    m = s.amax(dim=-1, keepdim=True).clamp_(min=-3e38)
    p = s.sub_(m).exp_()
    total = p.sum(dim=-1, keepdim=True)
    o = torch.bmm(p.view(B * Hkv, -1, Lm), v).view(B, Hkv, Hq // Hkv, Rm, D).div_(total.clamp(min=1e-38))
    ok = i < R[:, None]
    y["out"].copy_(o.permute(0, 3, 1, 2, 4).reshape(B, Rm, Hq, D)[ok])
    y["lse"].copy_((m + total.log()).permute(0, 3, 1, 2, 4).reshape(B, Rm, Hq)[ok])


# ------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    results = []
    for y in st["layers"]:
        r = {}
        if case["kind"] != "attend":
            r["q"] = _exact_write(st, y)
        if case["kind"] != "write":
            r["out"], r["lse"] = _exact_attend(st, y, r.get("q"))
        results.append(r)
    if case["kind"] != "write":
        return [{n: r[n] for n in ("out", "lse") + (("q",) if case["kind"] == "step" else ())} for r in results]
    y = st["layers"][0]
    if case["pool"] == "e4m3":
        return {"q": results[0]["q"], **{n: torch.cat([_exact_tokens(st, y, n, b) for b in range(st["B"])]) for n in "kv"}}
    return {"q": results[0]["q"], "k_pages": y["k_pages"].double(), "v_pages": y["v_pages"].double()}


def _pages_of(st, b):
    first, end = st["page_indptr"][b:b + 2].tolist()
    return st["page_table"][first:end].long()


def _exact_head(st, x, weight, pos):
    """x [tokens, heads, D] at positions pos, each pair of entries as a complex number."""
    x = x.double()
    if weight is not None:
        x = weight.double() * x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS)
    n = st["inv_freq"].numel()
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=st["dev"]), torch.outer(pos.double(), st["inv_freq"].double()))[:, None]
    if st["case"]["rotary"] == "half":
        z = torch.complex(x[..., :n].contiguous(), x[..., n:2 * n].contiguous()) * turn
        return torch.cat([z.real, z.imag, x[..., 2 * n:]], dim=-1)
    z = torch.view_as_complex(x[..., :2 * n].unflatten(-1, (n, 2)).contiguous()) * turn
    return torch.cat([torch.view_as_real(z).flatten(-2), x[..., 2 * n:]], dim=-1)


def _exact_write(st, y):
    """Q in 64 bits; K and V go into the pools (float64 copies, or values of 8 bits with their scales)."""
    if st["case"]["pool"] != "e4m3":
        y["k_pages"], y["v_pages"] = y["k_pages"].double(), y["v_pages"].double()
    q = torch.empty(y["q"].shape, dtype=torch.float64, device=st["dev"])
    at, ps = 0, st["case"]["page"]
    for b, (r, n) in enumerate(zip(st["R"], st["L"])):
        pos = torch.arange(n - r, n, device=st["dev"])
        q[at:at + r] = _exact_head(st, y["q_new"][at:at + r], y["q_weight"], pos)
        page = _pages_of(st, b)[pos // ps]
        for name, x in (("k", _exact_head(st, y["k_new"][at:at + r], y["k_weight"], pos)), ("v", y["v_new"][at:at + r].double())):
            if st["case"]["pool"] == "e4m3":
                top = x.abs().amax(-1)
                e = torch.ceil(torch.log2(top.clamp(min=1e-300) / 448.0)).clamp(-126, 127)
                e = torch.where(448.0 * torch.exp2(e - 1) >= top, e - 1, e)
                code = (x / torch.exp2(e)[..., None]).float().to(torch.float8_e4m3fn)
                y[name + "_pages"].view(torch.uint8)[page, pos % ps] = code.view(torch.uint8)
                y[name + "_scale"][page, :, pos % ps] = (e + 127).to(torch.uint8)
            else:
                y[name + "_pages"][page, pos % ps] = x
        at += r
    return q


def _exact_tokens(st, y, name, b):
    """K or V of a sequence, [L, Hkv, D]."""
    ids, n = _pages_of(st, b), st["L"][b]
    if st["case"]["pool"] != "e4m3":
        return y[name + "_pages"][ids].flatten(0, 1)[:n].double()
    x = y[name + "_pages"].view(torch.uint8)[ids].view(torch.float8_e4m3fn).float().double()
    x *= torch.exp2(y[name + "_scale"][ids].double() - 127.0).transpose(1, 2)[..., None]
    return x.flatten(0, 1)[:n]


def _exact_attend(st, y, q):
    (Hq, Hkv, D), G = st["heads"], st["heads"][0] // st["heads"][1]
    q = y["q"].double() if q is None else q.to(y["q"].dtype).double()
    out = torch.empty((st["total_q"], Hq, D), dtype=torch.float64, device=st["dev"])
    lse = torch.empty((st["total_q"], Hq), dtype=torch.float64, device=st["dev"])
    parent = _tree_parents(st["case"]) if st["case"]["tree"] else None
    at = 0
    for b, (r, n) in enumerate(zip(st["R"], st["L"])):
        k, v = (_exact_tokens(st, y, name, b).permute(1, 0, 2).contiguous() for name in "kv")       # [Hkv, n, D]
        qb = q[at:at + r].view(r, Hkv, G, D).permute(1, 2, 0, 3).reshape(Hkv, G * r, D)
        s = (qb @ k.transpose(1, 2).contiguous() * st["scale"]).view(Hkv, G, r, n)
        seen = torch.zeros((r, n), dtype=torch.bool)
        seen[:, :n - r] = True
        for i in range(r):
            node = i
            while node >= 0:
                seen[i, n - r + node] = True
                node = parent[node] if parent else node - 1
        s[:, :, ~seen.to(st["dev"])] = -math.inf
        z = torch.logsumexp(s, dim=-1)
        o = torch.exp(s - z[..., None]).view(Hkv, G * r, n) @ v
        out[at:at + r] = o.view(Hkv, G, r, D).permute(2, 0, 1, 3).reshape(r, Hq, D)
        lse[at:at + r] = z.permute(2, 0, 1).reshape(r, Hq)
        at += r
    return out, lse


# ------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    Hq, Hkv, D = HEADS[case["heads"]]
    if case["kind"] == "write":
        R, L = _write_shape(case)
        moved = sum(R) * ((2 * Hq + 2 * Hkv) * D * _size(case) + _pool_token(case))
        if case["pool"] == "e4m3":
            moved += sum(L) * (_pool_token(case) + 2 * Hkv * D * _size(case))
        return {"bytes": moved, "flops": sum(R) * (Hq + 2 * Hkv) * D * 8}
    R, L, S = _attend_shape(case)
    r, per = case["k"] + 1, case["per"]
    tokens = sum(n - s for n, s in zip(L, S)) + sum(S[0:case["groups"] * per:per] if per else [])
    if case["tree"]:
        parent = _tree_parents(case)
        depth = [0] * r
        for i in range(1, r):
            depth[i] = depth[parent[i]] + 1
        inside = sum(d + 1 for d in depth)
    else:
        inside = r * (r + 1) // 2
    pairs = sum(r * (n - r) + inside for n in L)
    one = {"bytes": tokens * _pool_token(case) + sum(R) * Hq * (2 * D * _size(case) + 4), "flops": 4 * D * Hq * pairs}
    if case["kind"] == "step":
        one["bytes"] += sum(R) * ((2 * Hq + 2 * Hkv) * D * _size(case) + _pool_token(case))
        one["flops"] += sum(R) * (Hq + 2 * Hkv) * D * 8
    return {n: case["layers"] * x for n, x in one.items()}
