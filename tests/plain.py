"""Plain implementations in 64 bits that the tests of prompts, token log-probabilities and cache pages compare with,
each with the bound that its rounding errors are held to."""
from __future__ import annotations

import math

import torch

HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}   # relative error of one rounding


def prompt_attention(q, k, v, R, L, scale):
    """q [sum R, Hq, D]; k, v: a list of [L_b, Hkv, D].  Returns out, lse and element-wise bounds of both, in float64.

    The bound: scores are sums of D products in fp32 and enter an exponential (relative error of a probability: (D + 8) steps of
    the largest sum of |q||k|); sums over the keys add a step per key at most; a bf16 call rounds probabilities and result."""
    Hq, D = q.shape[1:]
    Hkv = k[0].shape[1]
    dt = q.dtype
    out = torch.zeros((sum(R), Hq, D), dtype=torch.float64, device=q.device)
    lse = torch.full((sum(R), Hq), -math.inf, dtype=torch.float64, device=q.device)
    tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    at = 0
    for b, (r, n) in enumerate(zip(R, L)):
        if r and n:
            sees = torch.arange(n, device=q.device)[None, :] <= n - r + torch.arange(r, device=q.device)[:, None]
            for h in range(Hq):
                qh, kh, vh = q[at:at + r, h].double(), k[b][:, h * Hkv // Hq].double(), v[b][:, h * Hkv // Hq].double()
                s = (qh @ kh.t().contiguous() * scale).masked_fill(~sees, -math.inf)
                most = (qh.abs() @ kh.abs().t().contiguous()).max() * abs(scale)
                err = (D + 8) * 2.0 ** -24 * most + (n + 8) * 2.0 ** -24 + 2.0 ** -20
                any_ = sees.any(dim=1)
                z = torch.logsumexp(s, dim=1)
                p = torch.where(any_[:, None], torch.exp(s - z[:, None]), 0.0)
                o, size = p @ vh, p @ vh.abs()
                step = HALF_STEP[dt]
                out[at:at + r, h] = o
                tol[at:at + r, h] = size * 2 * err + step * o.abs() * 1.01 + (step * size * 1.01 if dt == torch.bfloat16 else 0.0) + 1e-30
                lse[at:at + r, h] = z
                lse_tol[at:at + r, h] = 2 * err + z.abs() * 2.0 ** -22
        at += r
    return out, lse, tol, lse_tol


def check_prompt(out, lse, ref):
    o, z, tol, z_tol = ref
    assert torch.isfinite(out).all()
    over = (out.double() - o).abs() - tol
    assert over.max() <= 0, f"out: {over.max():.3e} over its bound at {over.argmax().item()}"
    if lse is not None:
        none = torch.isinf(z)
        assert torch.equal(torch.isinf(lse) & (lse < 0), none)
        over = torch.where(none, -1.0, (lse.double() - z).abs() - z_tol)
        assert over.max() <= 0, f"lse: {over.max():.3e} over its bound"


def token_logprobs(logits, tokens, T, top=0):
    """logprob, lse, entropy, top tokens and top logprobs in float64; T a number or [rows]."""
    rows, V = logits.shape
    T = torch.as_tensor(T, dtype=torch.float64, device=logits.device).expand(rows)
    z = logits.double() / T[:, None]
    lse = torch.logsumexp(z, dim=1)
    log_p = z - lse[:, None]
    p = log_p.exp()
    ent = -(p * torch.where(p > 0, log_p, 0.0)).sum(dim=1)
    used = (tokens >= 0) & (tokens < V)
    lp = log_p.gather(1, tokens.long().clamp(0, V - 1)[:, None])[:, 0]
    n = min(top, V)
    ids = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :n]
    best = log_p.gather(1, ids)
    pad = (rows, top - n)
    ids = torch.cat([ids, torch.full(pad, -1, device=ids.device)], 1)
    best = torch.cat([best, torch.full(pad, -math.inf, dtype=torch.float64, device=ids.device)], 1)
    w = used[:, None]
    return (torch.where(used, lp, 0.0), torch.where(used, lse, 0.0), torch.where(used, ent, 0.0), torch.where(w, ids, -1),
            torch.where(w, best, 0.0))


def logprob_grad(logits, tokens, T, g, h):
    """d(sum g logprob + sum h entropy) / dlogits in float64."""
    rows, V = logits.shape
    T = torch.as_tensor(T, dtype=torch.float64, device=logits.device).expand(rows)
    z = logits.double() / T[:, None]
    log_p = z - torch.logsumexp(z, dim=1, keepdim=True)
    p = log_p.exp()
    log_p = torch.where(p > 0, log_p, 0.0)
    H = -(p * log_p).sum(dim=1, keepdim=True)
    hit = torch.zeros_like(p).scatter_(1, tokens.long().clamp(0, V - 1)[:, None], 1.0)
    grad = (g[:, None].double() * (hit - p) - h[:, None].double() * p * (log_p + H)) / T[:, None]
    return torch.where(((tokens >= 0) & (tokens < V))[:, None], grad, 0.0)


class Pages:
    """The page tables of a cache, one sequence after another, on the host."""

    def __init__(self, cap, num_pages, page_size):
        self.ps, self.B, self.cap = page_size, len(cap), list(cap)
        self.table = [[-1] * c for c in cap]
        self.count, self.kv, self.refs = [0] * self.B, [0] * self.B, [0] * num_pages

    def resize(self, want):
        before = list(self.refs)
        free = [i for i, r in enumerate(before) if r == 0]
        src, dst, missing, used = [-1] * self.B, [-1] * self.B, [0] * self.B, 0
        for b, w in enumerate(want):
            if w < 0:
                continue
            n, row, at = -(-w // self.ps), self.table[b], self.kv[b] // self.ps
            split = w > self.kv[b] and self.kv[b] % self.ps != 0 and at < self.count[b] and before[row[at]] > 1
            need = max(0, n - self.count[b]) + split
            if n > self.cap[b]:
                missing[b] = need
                continue
            mine, used = free[used:used + need], used + need   # (a sequence that finds too few takes its place in the order all the same)
            if len(mine) < need:
                missing[b] = need
                continue
            for e in range(n, self.count[b]):
                self.refs[row[e]] -= 1
                row[e] = -1
            if split:
                src[b], dst[b] = row[at], mine.pop(0)
                self.refs[row[at]] -= 1
                row[at] = dst[b]
                self.refs[dst[b]] = 1
            for e in range(self.count[b], n):
                row[e] = mine.pop(0)
                self.refs[row[e]] = 1
            self.count[b], self.kv[b] = n, min(self.kv[b], w)
        return src, dst, missing

    def fork(self, parent):
        missing = [0] * self.B
        for b, p in enumerate(parent):
            if p < 0:
                continue
            if p >= self.B or parent[p] >= 0 or self.count[b] or self.count[p] > self.cap[b]:
                missing[b] = -1
                continue
            for e in range(self.count[p]):
                self.table[b][e] = self.table[p][e]
                self.refs[self.table[p][e]] += 1
            self.count[b], self.kv[b] = self.count[p], self.kv[p]
        return missing

    def compact(self, max_moves):
        live = [i for i, r in enumerate(self.refs) if r > 0]
        n = len(live)
        moves = list(zip([i for i in reversed(live) if i >= n], [i for i in range(n) if self.refs[i] == 0]))[:max_moves]
        to = dict(moves)
        for a, b in moves:
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.table = [[to.get(e, e) for e in row] for row in self.table]
        pad = [-1] * (max_moves - len(moves))
        end = 1 + max([i for i, r in enumerate(self.refs) if r > 0], default=-1)
        return [a for a, _ in moves] + pad, [b for _, b in moves] + pad, end
