"""Plain implementations in 64 bits of what goes into the paged cache and of the attention over it, with the bounds that rounding errors are
held to; and a paged cache on the host's terms to build inputs with."""
from __future__ import annotations

import math

import torch

from plain import HALF_STEP


def ints(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


def offsets(n, dtype=torch.int32):
    return ints([0] + list(n), dtype).cumsum(0).to(dtype)


def scratch(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def quantise(x):
    """Codes and exponent bytes of x [..., D]: the least byte >= 1 with max |x| <= 448 2^(byte - 127), over what is finite."""
    x = x.double()
    finite = torch.isfinite(x)
    top = torch.where(finite, x.abs(), 0.0).amax(dim=-1)
    byte = torch.ones(top.shape, dtype=torch.int64, device=x.device)
    for power in (128, 64, 32, 16, 8, 4, 2, 1):                 # the largest byte that is too small, by bisection
        more = byte + power
        byte = torch.where((more <= 254) & (top > 448.0 * torch.ldexp(torch.ones_like(top), (more - 1 - 127).clamp(-126, 127))), more, byte)
    step = torch.ldexp(torch.ones_like(top), byte - 127)[..., None]
    code = torch.where(finite, x / step, math.nan).float().to(torch.float8_e4m3fn).view(torch.uint8)
    return torch.where(finite, code, 0x7f).to(torch.uint8), byte.to(torch.uint8)


def values(code, byte):
    return code.view(torch.float8_e4m3fn).float().double() * torch.ldexp(torch.ones(byte.shape, dtype=torch.float64, device=byte.device), byte.long() - 127)[..., None]


def norm_rope(x, weight, eps, pos, inv_freq, interleaved):
    """Heads x [tokens, H, D] at positions pos, in float64, and the bound of what fp32 makes of them before any rounding to fewer bits.

    The sum of squares is 16 products in a row and 3 sums of lanes (20 half steps, of which the root leaves half), the root, the division and two
    products 5 more; an angle is off by the rounding of a number of half turns up to 1 (pi 2^-25) and sine and cosine by two units; two products
    and a sum: no more than 32 half steps of |a| + |b|."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(dim=-1, keepdim=True) + eps) * weight.double()
    out, size = x.clone(), x.abs()
    if inv_freq is not None:
        n = inv_freq.numel()
        t = pos.double()[:, None, None] * inv_freq.double()
        a = slice(0, 2 * n, 2) if interleaved else slice(0, n)
        b = slice(1, 2 * n, 2) if interleaved else slice(n, 2 * n)
        out[..., a] = x[..., a] * t.cos() - x[..., b] * t.sin()
        out[..., b] = x[..., b] * t.cos() + x[..., a] * t.sin()
        size[..., a] = size[..., b] = (x[..., a].abs() + x[..., b].abs())
    # (an angle of many turns: the product is rounded in 64 bits, 2^-53 of it)
    far = 0.0 if inv_freq is None else float((pos.double().abs().max() * inv_freq.double().abs().max()).item()) * 2.0 ** -52
    return out, size * (32 * 2.0 ** -24 + far)


def check_rounded(got, ref, tol, name):
    """got, rounded once to its type, against ref with the bound tol of what was rounded."""
    over = (got.double() - ref).abs() - tol * 1.01 - HALF_STEP[got.dtype] * (ref.abs() + tol)
    assert over.max() <= 0, f"{name}: {over.max():.3e} over its bound"


def check_quantised(got, ref, tol, name):
    """Values read back against what was written: half a step of e4m3 (2^-4 of a number; 2^-10 of the scale for those near zero, whose scale is at
    most 2 max / 256, or twice that where the largest is off and another power of two)."""
    top = (ref.abs() + tol).amax(dim=-1, keepdim=True)
    over = (got.double() - ref).abs() - tol * 1.1 - torch.maximum(2.0 ** -4 * ref.abs(), 2.0 ** -10 * top / 64)
    assert over.max() <= 0, f"{name}: {over.max():.3e} over its bound"


def attention(q, k, v, R, L, scale, masks=None):
    """q [sum R, Hq, D]; k, v: a list of [L_b, Hkv, D]; masks: a list of 64-bit words per row (trees).  Returns out, lse and element-wise bounds of both, in
    float64; the bound is that of plain.prompt_attention, whose parts are joined by a handful of roundings more (2^-20 in it)."""
    Hq, D = q.shape[1:]
    Hkv = k[0].shape[1]
    out = torch.zeros((sum(R), Hq, D), dtype=torch.float64, device=q.device)
    lse = torch.full((sum(R), Hq), -math.inf, dtype=torch.float64, device=q.device)
    tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    at = 0
    for b, (r, n) in enumerate(zip(R, L)):
        if r and n:
            sees = torch.arange(n, device=q.device)[None, :] <= n - r + torch.arange(r, device=q.device)[:, None]
            if masks is not None:
                sees = torch.arange(n, device=q.device)[None, :].repeat(r, 1) < n - r
                for i in range(r):
                    for j in range(r):
                        sees[i, n - r + j] = bool(masks[at + i] >> j & 1)
            for h in range(Hq):
                qh, kh, vh = q[at:at + r, h].double(), k[b][:, h * Hkv // Hq].double(), v[b][:, h * Hkv // Hq].double()
                s = (qh @ kh.t().contiguous() * scale).masked_fill(~sees, -math.inf)
                most = (qh.abs() @ kh.abs().t().contiguous()).max() * abs(scale)
                err = (D + 8) * 2.0 ** -24 * most + (n + 8) * 2.0 ** -24 + 2.0 ** -20
                z = torch.logsumexp(s, dim=1)
                p = torch.where(sees.any(dim=1)[:, None], torch.exp(s - z[:, None]), 0.0)
                o, size = p @ vh, p @ vh.abs()
                step = HALF_STEP[q.dtype]
                out[at:at + r, h] = o
                tol[at:at + r, h] = size * 2 * err + step * o.abs() * 1.01 + (step * size * 1.01 if q.dtype == torch.bfloat16 else 0.0) + 1e-30
                lse[at:at + r, h] = z
                lse_tol[at:at + r, h] = 2 * err + z.abs() * 2.0 ** -22
        at += r
    return out, lse, tol, lse_tol


class Cache:
    """Pools of one layer with the tokens of sequences whose groups share pages: members of a group name the first one's pages for whole pages of
    `shared` tokens.  lens[b]: tokens of sequence b; what lies behind them in their last pages, and pages of nobody, hold NaN."""

    def __init__(self, lens, Hkv, D, page, dtype, groups=(), shared=(), pool="same", seed=0, table_room=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.lens, self.page, self.Hkv, self.D = list(lens), page, Hkv, D
        first, keep = {}, {}
        for g, s in zip(groups, shared):
            for b in g[1:]:
                first[b], keep[b] = g[0], s // page
        pages, n = [], 0
        for b, length in enumerate(lens):
            held = -(-length // page)
            mine = pages[first[b]][:keep[b]] if b in first else []
            pages.append(mine + list(range(n, n + held - len(mine))))
            n += held - len(mine)
        self.num_pages = n + 3
        order = torch.randperm(self.num_pages, generator=torch.Generator().manual_seed(seed + 1))
        self.pages = [[int(order[i]) for i in p] for p in pages]
        self.page_indptr = offsets([len(p) + table_room for p in self.pages])
        self.page_table = ints([i for p in self.pages for i in p + [-1] * table_room] or [0])
        self.kv_len = ints(self.lens)
        shape = (self.num_pages, page, Hkv, D)
        k, v = (torch.randn(shape, generator=gen, device="cuda").to(dtype) for _ in range(2))
        used = torch.zeros(shape[:2], dtype=torch.bool, device="cuda")
        for p, length in zip(self.pages, lens):
            for i, page_id in enumerate(p):
                used[page_id, :min(page, length - i * page)] = True
        k[~used], v[~used] = math.nan, math.nan
        self.k_scale = self.v_scale = None
        if pool == "e4m3":
            (k, ks), (v, vs) = quantise(k), quantise(v)
            self.k_scale, self.v_scale = (s.transpose(1, 2).contiguous() for s in (ks, vs))
            k, v = k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn)
        self.k, self.v = k, v

    def tokens(self, name, b):
        """K or V of sequence b as [L_b, Hkv, D]; a cache of 8 bits: what the codes stand for, in float64."""
        n = self.lens[b]
        if n == 0:
            return torch.zeros((0, self.Hkv, self.D), device="cuda")
        ids = ints(self.pages[b], torch.int64)
        x = getattr(self, name)
        if self.k_scale is not None:
            x = values(x.view(torch.uint8)[ids], getattr(self, name + "_scale")[ids].transpose(1, 2).contiguous())
            return x.flatten(0, 1)[:n]
        return x[ids].flatten(0, 1)[:n]

    def both(self):
        return [[self.tokens(n, b) for b in range(len(self.lens))] for n in "kv"]

    def args(self):
        return self.k, self.v, self.k_scale, self.v_scale

    def tables(self):
        return self.page_indptr, self.page_table, self.kv_len
