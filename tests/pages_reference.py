"""Definitions in 64 bits of the norm of heads and of a cache in pages, with bounds on what 32-bit sums and one rounding may be off
by; for the tests.  All tensors are torch tensors on any device."""
import math

import torch

import block_reference as ref
from block_reference import U16, U32

E4M3 = torch.float8_e4m3fn


# --------------------------------------------------------------------------------------------------
# norm of heads
# --------------------------------------------------------------------------------------------------
def turn(x, off, positions, freqs, sections, interleaved, back=False):
    """x's pairs turned by positions * freqs, and what that may be off by where x is off by `off`."""
    if positions is None:
        return x, off
    pairs = freqs.shape[0]
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    angle = positions.double().view(x.shape[0], -1)[:, axis] * freqs.double() * (-1 if back else 1)
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    i = torch.arange(pairs, device=x.device)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
    y, e = x.clone(), off.clone()
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    # (the angle, below pi, is rounded to 32 bits: 2 units; cosine and sine to 2 more, product, sum)
    size = 8 * U32 * (x[..., a].abs() + x[..., b].abs())
    e[..., a] = size + off[..., a] * cos.abs() + off[..., b] * sin.abs()
    e[..., b] = size + off[..., b] * cos.abs() + off[..., a] * sin.abs()
    return y, e


def _normed(x, eps, centred):
    """(n, its bound, rstd, its relative bound) of heads in 64 bits: a sum of D floats is off by at most D units of the mean magnitude."""
    D = x.shape[-1]
    mean = x.mean(-1, keepdim=True) if centred else torch.zeros_like(x[..., :1])
    c = x - mean
    d_c = (D + 4) * U32 * x.abs().mean(-1, keepdim=True) + 2 * U32 * (x.abs() + mean.abs()) if centred else torch.zeros_like(x)
    square = c.square().mean(-1, keepdim=True) + eps
    rstd = square.rsqrt()
    d_r = (D + 8) * U32 + (c.abs() * d_c + d_c.square()).mean(-1, keepdim=True) / square
    n = c * rstd
    return n, n.abs() * (d_r + 2 * U32) + d_c * rstd, rstd, d_r


def _weights(weight, heads, H, like):
    if weight is None:
        return torch.ones_like(like[:1])
    w = weight.double()
    return torch.cat([w[:1].expand(heads, -1), w[1:].expand(H - heads, -1)])[None] if w.dim() == 2 else w[None, None]


def head_norm(X, weight, heads, eps, centred, turned, dtype):
    """(y, bound); turned: (positions, freqs, sections, interleaved)."""
    x = X.double()
    n, d_n, _, _ = _normed(x, eps, centred)
    w = _weights(weight, heads, x.shape[1], x)
    y, off = turn(n * w, d_n * w.abs() + U32 * (n * w).abs(), *turned)
    return y, off + ref.rounding(dtype) * (y.abs() + off)


def head_norm_grad(dY, X, weight, heads, eps, centred, turned, dtype):
    """((dx, bound), (dweight, bound) or None)."""
    x, dy = X.double(), dY.double()
    D = x.shape[-1]
    n, d_n, r, d_r = _normed(x, eps, centred)
    w = _weights(weight, heads, x.shape[1], x)
    d, d_d = turn(dy, torch.zeros_like(dy), *turned, back=True)
    g, d_g = d * w, d_d * w.abs() + U32 * (d * w).abs()
    m1 = g.mean(-1, keepdim=True) if centred else torch.zeros_like(r)
    m2 = (g * n).mean(-1, keepdim=True)
    e1 = ((D + 4) * U32 * g.abs() + d_g).mean(-1, keepdim=True) if centred else torch.zeros_like(r)
    e2 = ((D + 4) * U32 * (g * n).abs() + d_g * n.abs() + g.abs() * d_n).mean(-1, keepdim=True)
    dx = r * (g - m1 - n * m2)
    size = g.abs() + m1.abs() + (n * m2).abs()
    off = r * (d_g + e1 + n.abs() * e2 + d_n * (m2.abs() + e2) + (6 * U32 + d_r) * size)
    out = (dx, off + ref.rounding(dtype) * (dx.abs() + off))
    if weight is None:
        return out, None
    each, d_each = d * n, d_d * n.abs() + d.abs() * d_n
    parts = [slice(0, heads), slice(heads, None)] if weight.dim() == 2 else [slice(None)]
    dw = torch.stack([each[:, p].sum((0, 1)) for p in parts])
    count = each.shape[0] * each.shape[1]
    bound = torch.stack([((count + 4) * U32 * each[:, p].abs() + d_each[:, p]).sum((0, 1)) for p in parts])
    return out, (dw.view(weight.shape), bound.view(weight.shape))


# --------------------------------------------------------------------------------------------------
# rows in 8 bits
# --------------------------------------------------------------------------------------------------
NUMBERS = [m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:-1]


def rounded(x):
    """(values, exponent bytes) of rows as the cache holds them in 8 bits, by the definition: of all numbers of the format times the row's
    power of two the nearest, to an even code where two are as near."""
    x = x.double()
    finite = x.isfinite()
    top = torch.where(finite, x.abs(), 0.0).amax(-1, keepdim=True)
    power = torch.full_like(top, 119.0)
    for e in range(118, -101, -1):
        power = torch.where(top <= 448 * 2.0 ** e, float(e), power)
    numbers = torch.tensor(NUMBERS, dtype=torch.float64, device=x.device)
    y = torch.where(finite, x, 0.0) * torch.exp2(-power)
    above = torch.searchsorted(numbers, y.abs()).clamp(max=len(NUMBERS) - 1)
    below = (above - 1).clamp(min=0)
    up, down = numbers[above] - y.abs(), y.abs() - numbers[below]
    code = torch.where((up < down) | ((up == down) & (above % 2 == 0)), above, below)
    value = torch.copysign(numbers[code], x) * torch.exp2(power)
    return torch.where(finite, value, math.nan), (power + 127).squeeze(-1).to(torch.uint8)


class Cache:
    """Pages of a test: `table` in an order of chance, pages and scales filled with `waste` (what must not be read)."""

    def __init__(self, lengths, room, heads, size, page, codes, seed=0, order="heads", spare=2, waste=math.nan):
        g = torch.Generator().manual_seed(seed)
        self.page, self.codes, self.lens = page, codes, list(lengths)
        width = -(-room // page)
        self.count = len(lengths) * width + spare
        self.table = torch.randperm(self.count, generator=g)[:len(lengths) * width].view(-1, width).to(torch.int32).cuda()
        self.lengths = torch.tensor(self.lens, dtype=torch.int32, device="cuda")

        def rows(*extra, dtype, value):
            if order == "heads":
                t = torch.full((self.count, heads, page) + extra, value, device="cuda", dtype=dtype).transpose(1, 2)
            else:
                t = torch.full((self.count, page, heads) + extra, value, device="cuda", dtype=dtype)
            return t

        self.K, self.V = (rows(size, dtype=torch.bfloat16, value=waste) for _ in range(2))
        self.K_scales = self.V_scales = None
        if codes:
            self.K, self.V = self.K.to(E4M3), self.V.to(E4M3)
            self.K_scales, self.V_scales = (rows(dtype=torch.uint8, value=127) for _ in range(2))

    @property
    def args(self):
        return self.K, self.V, self.table, self.lengths

    @property
    def scales(self):
        return {"K_scales": self.K_scales, "V_scales": self.V_scales}

    def places(self, b, at):
        return self.table[b, at // self.page].long(), at % self.page

    def put(self, b, at, k, v):
        """Tokens `at` of sequence b by indexing, in the definition's values."""
        entry, slot = self.places(b, at)
        for pages, scales, x in ((self.K, self.K_scales, k), (self.V, self.V_scales, v)):
            if self.codes:
                x, power = rounded(x)
                scales[entry, slot] = power
                x = (x * torch.exp2(127 - power.double())[..., None]).float().to(E4M3)
                pages.view(torch.uint8)[entry, slot] = x.view(torch.uint8)
            else:
                pages[entry, slot] = x

    def rows(self, b, at):
        """(k, v) of tokens `at` of sequence b in 64 bits."""
        entry, slot = self.places(b, at)
        out = []
        for pages, scales in ((self.K, self.K_scales), (self.V, self.V_scales)):
            if self.codes:
                x = pages.view(torch.uint8)[entry, slot].view(E4M3).float().double()
                out.append(x * torch.exp2(scales[entry, slot].double() - 127)[..., None])
            else:
                out.append(pages[entry, slot].double())
        return out

    def fill(self, seed, scale=1.0):
        """Every sequence's tokens; what lies behind them stays what it was."""
        g = torch.Generator("cuda").manual_seed(seed)
        H, D = self.K.shape[2:]
        for b, n in enumerate(self.lens):
            k, v = (torch.randn(n, H, D, generator=g, device="cuda").mul(scale).to(torch.bfloat16) for _ in range(2))
            self.put(b, torch.arange(n, device="cuda"), k, v)
        return self


def paged(Q, cache, counts, scale, window=0, sinks=0, gone=()):
    """(O, bound, lse, bound); gone: (sequence, page of it) that are not there."""
    Q = Q.double()
    H, D = cache.K.shape[2:]
    group = Q.shape[1] // H
    O, bO = torch.zeros_like(Q), torch.zeros_like(Q)
    lse = torch.full((Q.shape[1], Q.shape[0]), -math.inf, dtype=torch.float64, device=Q.device)
    bl = torch.zeros_like(lse)
    q0 = 0
    for b, (L, n) in enumerate(zip(counts, cache.lens)):
        rows = slice(q0, q0 + L)
        q0 += L
        if L == 0 or n == 0:
            continue
        at, p = torch.arange(n, device=Q.device), torch.arange(n - L, n, device=Q.device)[:, None]
        seen = at <= p
        if window:
            seen = seen & ((at > p - window) | (at < sinks))
        for s, page in gone:
            if s == b:
                seen = seen & (at // cache.page != page)
        at = at[seen.any(0)]
        seen = seen[:, at]
        if len(at) == 0:
            continue
        k_all, v_all = cache.rows(b, at)
        for h in range(Q.shape[1]):
            q, k, v = Q[rows, h], k_all[:, h // group].contiguous(), v_all[:, h // group].contiguous()
            s, ds = ref._scores(q, k, scale, seen)
            any_seen = seen.any(1, keepdim=True)
            top = torch.where(any_seen, s.amax(1, keepdim=True), 0.0)
            e = torch.exp(s - top).masked_fill(~seen, 0.0)
            total = e.sum(1, keepdim=True)
            pr = torch.where(any_seen, e / total.clamp(min=1e-300), 0.0)
            off = torch.where(seen, ds, 0.0).amax(1, keepdim=True) * 2 + (len(at) + 16) * U32 + 64 * U32
            o = pr @ v
            # the probabilities rounded to bfloat16, their own error, the 32-bit sum (as for attention over contiguous keys)
            bound = (U16 * (1 + 2 * off) + 2 * off + (len(at) + 8) * U32) * (pr @ v.abs())
            O[rows, h] = o
            bO[rows, h] = bound + U16 * (o.abs() + bound)
            lse[h, rows] = torch.where(any_seen, top + total.log(), -math.inf).squeeze(1)
            bl[h, rows] = (off + 8 * U32 * (top.abs() + total.clamp(min=1).log() + 1)).squeeze(1)
    return O, bO, lse, bl
