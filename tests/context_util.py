"""Plain 64-bit forms of the eviction and block operators, and drawn caches for their tests (torch, on the CPU)."""

from __future__ import annotations

import math

import numpy as np
import torch

KS, VS = 2.0 ** -5, 2.0 ** -5
LOG2E = 1.4426950408889634


def wide(t, dtype, scale=KS):
    """Cache values in 64 bits."""
    if dtype == "fp8":
        return t.cpu().view(torch.float8_e4m3fn).float().double() * scale
    return t.cpu().double()


def cache_dtype(dtype):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.uint8}[dtype]


def query_dtype(dtype):
    return torch.float32 if dtype == "f32" else torch.bfloat16


def drawn(shape, dtype, gen, spread=1.0):
    x = torch.randn(shape, generator=gen) * spread
    if dtype == "fp8":
        return (x / KS).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    return x.to(cache_dtype(dtype))


class Context:
    """Sequences of a packed (page 0) or paged cache. layout: "dense", "fused" (K and V side by side in a token's row), or
    "heads" (a head's rows side by side). Rows that belong to no sequence are NaN."""

    def __init__(self, lens, dtype, hkv, d, page, gen, layout="dense", width=None, spread=1.0, both=False):
        self.lens, self.dtype, self.hkv, self.d, self.page = list(lens), dtype, hkv, d, page
        batch, step = len(lens), page or 1
        counts = [-(-n // step) for n in lens]
        total = sum(counts) + 3
        rows = total * step
        self.rows = rows
        order = torch.randperm(total, generator=gen) if page else torch.arange(total) + 1
        poison = 0x7f if dtype == "fp8" else float("nan")
        lead = (total, step) if page else (rows,)

        def empty():
            if layout == "fused":
                return torch.full(lead + (2, hkv, d), poison, dtype=cache_dtype(dtype)).select(len(lead), 0)
            if layout == "heads":
                return torch.full((hkv,) + lead + (d,), poison, dtype=cache_dtype(dtype)).movedim(0, len(lead))
            return torch.full(lead + (hkv, d), poison, dtype=cache_dtype(dtype))

        self.k = empty()
        self.v = empty() if both else None
        width = width or max(max(counts), 1)
        self.table = torch.full((batch, width), -1, dtype=torch.int32)
        self.seq_start = torch.zeros(batch, dtype=torch.int64)
        self.at, first = [], 0
        for b, n in enumerate(lens):
            mine = order[first:first + counts[b]]
            first += counts[b]
            self.table[b, :counts[b]] = mine.to(torch.int32)
            t = torch.arange(n)
            self.at.append(mine[t // step] * step + t % step if n else t)
            self.seq_start[b] = int(mine[0]) if n and not page else 0
            for cache in (self.k, self.v):
                if cache is not None and n:
                    x = drawn((n, hkv, d), dtype, gen, spread)
                    if page:
                        cache[self.at[b] // step, self.at[b] % step] = x
                    else:
                        cache[self.at[b]] = x
        self.ctx_lens = torch.tensor(lens, dtype=torch.int32)

    def keys(self, b, cache=None):
        """K rows of sequence b in 64 bits, [n, hkv, d]."""
        k = self.k if cache is None else cache
        at = self.at[b]
        return wide(k[at // self.page, at % self.page] if self.page else k[at], self.dtype)

    def to(self, device):
        """The tensors on the device, strides kept."""
        def moved(t):
            if t is None:
                return None
            out = torch.empty_strided(t.size(), t.stride(), dtype=t.dtype, device=device)
            out.copy_(t)
            return out

        return dict(k=moved(self.k), v=moved(self.v), block_table=self.table.to(device),
                    seq_start=self.seq_start.to(device), ctx_lens=self.ctx_lens.to(device))


def logsumexp_rows(ctx, q, new, scale):
    """lse [rows, hq] in 64 bits of the packed new tokens' queries."""
    hq = q.shape[1]
    group, out, first = hq // ctx.hkv, torch.zeros(q.shape[:2], dtype=torch.float64), 0
    for b, m in enumerate(new):
        k, n = ctx.keys(b), ctx.lens[b]
        for h in range(hq):
            s = scale * (q[first:first + m, h].double() @ k[:, h // group].T)
            seen = torch.arange(n)[None, :] <= (n - m + torch.arange(m))[:, None]
            out[first:first + m, h] = torch.logsumexp(s.masked_fill(~seen, -math.inf), 1)
        first += m
    return out


def weights_of(ctx, q, lse, new, scale, prior=None, decay=1.0):
    """(weights, bound) of each sequence: the sums in 64 bits, and how far float32 sums of float32 weights may be off.

    A score's float32 sum of D products is off by at most D 2^-23 of the sum of their magnitudes; x = score * scale * log2(e)
    - lse * log2(e) takes 2^-23 of both parts (two constants' and two products' roundings); exp2 one unit in the last
    place, 2^-23. A relative error of e^delta - 1 in the weight, delta = ln 2 * the exponent's. Adding up n weights in any
    order costs n 2^-24 of the sum; decay * prior one more rounding.
    """
    hq, d = q.shape[1:]
    group, got, first = hq // ctx.hkv, [], 0
    for b, m in enumerate(new):
        k, n = ctx.keys(b), ctx.lens[b]
        total, off = torch.zeros(n, dtype=torch.float64), torch.zeros(n, dtype=torch.float64)
        for h in range(hq):
            qh, kh, l = q[first:first + m, h].double(), k[:, h // group], lse[first:first + m, h].double()[:, None]
            s = scale * (qh @ kh.T)
            size = scale * (qh.abs() @ kh.abs().T)
            seen = (torch.arange(n)[None, :] <= (n - m + torch.arange(m))[:, None]) & (l > -math.inf)
            w = torch.where(seen, torch.exp(s - l), 0.0)
            delta = d * 2.0 ** -23 * size + 2.0 ** -22 * (s.abs() + torch.where(seen, l, 0.0).abs()) + 2.0 ** -23
            total += w.sum(0)
            off += torch.where(seen, w * torch.expm1(delta), 0.0).sum(0)
        off += (m * hq + 8) * 2.0 ** -24 * total + 1e-37
        if prior is not None and decay != 0:
            old = torch.arange(n) < n - m
            total = total + torch.where(old, decay * prior[b, :n].double(), 0.0)
            off += 2.0 ** -23 * total.abs()
        got.append((total, off))
        first += m
    return got


def near(got, want, off):
    """Whether every element is within its bound, which a NaN is not."""
    return bool(((got - want).abs() <= off).all())


def chosen(scores, count, first, last):
    """Positions of the `count` entries of a row (1-D) that stay, ascending."""
    x = np.asarray(scores, dtype=np.float32)
    n = len(x)
    rank = sorted(range(n), key=lambda i: (0 if i < first or i >= n - last else 1, 0 if np.isnan(x[i]) else 1,
                                           0.0 if np.isnan(x[i]) else -float(x[i]), i))
    return sorted(rank[:count])


def ordered(bits, width):
    """Bit patterns as integers that order -NaN .. -0, +0 .. NaN."""
    x = bits.to(torch.int64)
    top = 1 << (width - 1)
    return torch.where(x >= top, (2 * top - 1 - x) - top, x)


def patterns(t):
    """(unsigned bit patterns, width) of a cache tensor."""
    if t.dtype == torch.uint8:
        return t.to(torch.int64), 8
    if t.dtype == torch.bfloat16:
        return t.contiguous().view(torch.int16).to(torch.int64) & 0xffff, 16
    return t.contiguous().view(torch.int32).to(torch.int64) & 0xffffffff, 32


def ends_of(rows):
    """Least and greatest bit patterns of [tokens, hkv, d] rows, [hkv, 2, d]."""
    bits, width = patterns(rows)
    o = ordered(bits, width)
    pick = lambda i: bits.gather(0, i[None])[0]  # noqa: E731
    return torch.stack([pick(o.argmin(0)), pick(o.argmax(0))], dim=1)


def reach(q, ends, scale):
    """(scores, sizes): scale * max over the group's queries [G, d] of the bound of blocks [n, 2, d], and the largest sum
    of magnitudes that a score is made of."""
    s = q.clamp(min=0) @ ends[:, 1].T + q.clamp(max=0) @ ends[:, 0].T
    size = q.clamp(min=0) @ ends[:, 1].abs().T + q.clamp(max=0).abs() @ ends[:, 0].abs().T
    return scale * s.max(0).values, scale * size.max(0).values
