"""The attention operators' definition in 64 bits, one sequence and head after
another, with the gradients written out (no differentiation library). Test
infrastructure: shares no code with the kernels or their binding."""
from __future__ import annotations

import dataclasses

import numpy as np
import torch


@dataclasses.dataclass
class Problem:
    q_lens: list
    k_lens: list
    heads: int = 1
    kv_heads: int = 1
    dim: int = 64
    causal: bool = False
    prefix: list | None = None
    scale: float | None = None
    cap: float = 0.0
    table: torch.Tensor | None = None      # [buckets, heads]
    bucket_of: torch.Tensor | None = None  # [2*reach + 1]

    def __post_init__(self):
        if self.scale is None:
            self.scale = self.dim ** -0.5

    def offsets(self, which):
        lens = self.q_lens if which == "q" else self.k_lens
        return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def _one(p: Problem, b, q, k, v, h):
    """Scores' parts of one sequence and head: (visible, t or None, probabilities)."""
    nq, nk = q.shape[0], k.shape[0]
    x = (q @ k.T) * p.scale
    t = None
    if p.cap:
        t = torch.tanh(x / p.cap)
        x = p.cap * t
    pos = torch.arange(nq, device=q.device)[:, None] + (nk - nq)
    j = torch.arange(nk, device=q.device)[None, :]
    bucket = None
    if p.table is not None:
        r = (p.bucket_of.numel() - 1) // 2
        bucket = p.bucket_of.to(q.device).long()[(j - pos).clamp(-r, r) + r]
        x = x + p.table.to(q.device).double()[bucket, h]
    seen = torch.ones((nq, nk), dtype=torch.bool, device=q.device)
    if p.causal:
        seen = j <= pos
        if p.prefix is not None:
            seen = seen | (j < p.prefix[b])
    x = torch.where(seen, x, torch.full_like(x, -torch.inf))
    top = x.amax(-1, keepdim=True) if nk else x.new_full((nq, 1), -torch.inf)
    top = torch.where(top == -torch.inf, torch.zeros_like(top), top)
    e = torch.where(seen, torch.exp(x - top), torch.zeros_like(x))
    total = e.sum(-1, keepdim=True)
    prob = e / torch.where(total == 0, torch.ones_like(total), total)
    return seen, t, bucket, prob, (torch.log(total) + top)[:, 0]


def attention(p: Problem, q, k, v, dout=None):
    """q [Tq, H, D], k, v [Tk, KV, D] -> dict of out and lse [H, Tq], and with
    dout dq, dk, dv and dtable."""
    dev = q.device
    q, k, v = q.double(), k.double(), v.double()
    share = p.heads // p.kv_heads
    res = dict(out=torch.zeros_like(q), lse=torch.full((p.heads, q.shape[0]), -torch.inf,
                                                       dtype=torch.float64, device=dev))
    if dout is not None:
        dout = dout.double()
        res.update(dq=torch.zeros_like(q), dk=torch.zeros_like(k), dv=torch.zeros_like(v))
        if p.table is not None:
            res["dtable"] = torch.zeros(p.table.shape, dtype=torch.float64, device=dev)
            res["terms"] = 0.0  # sum of |ds|
    qo, ko = p.offsets("q"), p.offsets("k")
    for b in range(len(p.q_lens)):
        qs, ks = slice(qo[b], qo[b + 1]), slice(ko[b], ko[b + 1])
        if qo[b] == qo[b + 1]:
            continue
        for h in range(p.heads):
            c = h // share
            qq, kk, vv = q[qs, h].contiguous(), k[ks, c].contiguous(), v[ks, c].contiguous()
            seen, t, bucket, prob, lse = _one(p, b, qq, kk, vv, h)
            # what a query does not see has no part in its sums, NaN included
            clean = torch.where(seen[:, :, None], vv[None], torch.zeros_like(vv)[None]) \
                if not torch.isfinite(vv).all() else None
            out = prob @ vv if clean is None else (prob[:, :, None] * clean).sum(1)
            res["out"][qs, h] = out
            res["lse"][h, qs] = lse
            if dout is None:
                continue
            go = dout[qs, h].contiguous()
            dp = go @ vv.T
            ds = prob * (dp - (go * out).sum(-1, keepdim=True))
            res["dv"][ks, c] += prob.T @ go
            if bucket is not None:
                res["terms"] += ds.abs().sum().item()
                res["dtable"][:, h] += torch.zeros_like(res["dtable"][:, h]).index_add_(
                    0, bucket.reshape(-1), ds.reshape(-1))
            g = ds * p.scale
            if t is not None:
                g = g * (1 - t * t)
            res["dq"][qs, h] = g @ kk
            res["dk"][ks, c] += g.T @ qq
    return res


# --- the 8-bit cache's values --------------------------------------------------


def e4m3_value(bits: np.ndarray) -> np.ndarray:
    """Value of e4m3 codes (0x7f and 0xff are NaN)."""
    bits = bits.astype(np.int64)
    sign = np.where(bits & 128, -1.0, 1.0)
    power, frac = (bits >> 3) & 15, bits & 7
    mag = np.where(power > 0, (8 + frac) * 2.0 ** (power - 10.0), frac * 2.0 ** -9)
    return np.where((bits & 127) == 127, np.nan, sign * mag)


def quantise_rows(x: np.ndarray):
    """Codes and exponent bytes of rows x (float64 [..., dim]) by search: the
    least exponent that holds the row, then the nearest e4m3 value, ties to
    the even code."""
    values = e4m3_value(np.arange(127))  # ascending, 0 .. 448
    amax = np.abs(x).max(-1)
    e = np.full(amax.shape, -126)
    for n in range(-126, 128):
        e = np.where(amax > 448.0 * 2.0 ** n, n + 1, e)
    e = np.where(amax == 0, 0, e)
    y = np.abs(x) * 2.0 ** (-e[..., None].astype(np.float64))
    hi = np.clip(np.searchsorted(values, y), 1, 126)
    lo = hi - 1
    up = (y - values[lo] > values[hi] - y) | ((y - values[lo] == values[hi] - y) & (hi % 2 == 0))
    code = np.where(up, hi, lo).astype(np.uint8)
    code = np.where(np.signbit(x), code | 128, code)
    bad = ~np.isfinite(x).all(-1)
    return np.where(bad[..., None], 127, code).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)
