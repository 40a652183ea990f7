"""Definitions in 64 bits of the operators between the linear layers, with bounds on what 32-bit sums and one rounding to
bfloat16 may be off by; for the tests.  All tensors are torch tensors on any device."""
import math

import torch

U32, U16 = 2.0 ** -24, 2.0 ** -8  # relative rounding error of a float and of a bfloat16: 24 and 8 significant bits


def rounding(dtype):
    return U16 if dtype == torch.bfloat16 else U32


def close(got, want, bound, what=""):
    """Every element within its bound; the same infinities."""
    got = got.double()
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), what
    err = torch.where(inf, 0.0, (got - torch.where(inf, 0.0, want)).abs())
    assert bool(torch.isfinite(got[~inf]).all()), what
    worst = (err / bound.clamp(min=1e-300)).max() if err.numel() else torch.tensor(0.0)
    assert bool((err <= bound).all()), (what, float(worst))
    return float(worst)


# --------------------------------------------------------------------------------------------------
# layer norm
# --------------------------------------------------------------------------------------------------
def norm(x, w, b, eps, dtype):
    """(y, bound, mean, rstd) of rows x (64 bits): the mean of C floats is off by at most (log2-deep or lane-serial sums) C u
    of the mean magnitude, the difference to it by as much again, rstd by a few units of its sums."""
    C = x.shape[1]
    mean = x.mean(1, keepdim=True)
    var = (x - mean).square().mean(1, keepdim=True)
    rstd = (var + eps).rsqrt()
    n = (x - mean) * rstd
    y = n * w + b
    d_mean = (C + 2) * U32 * x.abs().mean(1, keepdim=True)
    # (a constant error e of the mean adds e^2 to the variance, of second order, and e rstd to every n)
    d_rstd = (C + 8) * U32 + (d_mean * rstd) ** 2
    d_n = (d_mean + U32 * (x.abs() + mean.abs())) * rstd + n.abs() * (d_rstd + 4 * U32)
    bound = d_n * w.abs() + 4 * U32 * (n * w).abs() + 2 * U32 * y.abs()
    return y, bound + rounding(dtype) * (y.abs() + bound), mean, rstd, d_mean, d_rstd


def norm_grad(dy, x, mean, rstd, w, ds, dtype):
    """((dx, bound), (dw, bound), (db, bound)) with the statistics as given."""
    T, C = x.shape
    n = (x - mean) * rstd
    d_n = 4 * U32 * (x.abs() + mean.abs()) * rstd
    g = dy * w
    m1, m2 = g.mean(1, keepdim=True), (g * n).mean(1, keepdim=True)
    e1 = (C + 4) * U32 * g.abs().mean(1, keepdim=True)
    e2 = (C + 6) * U32 * (g * n).abs().mean(1, keepdim=True) + (g.abs() * d_n).mean(1, keepdim=True)
    dx = rstd * (g - m1 - n * m2)
    size = g.abs() + m1.abs() + (n * m2).abs()
    bound = rstd * (6 * U32 * size + e1 + n.abs() * e2 + d_n * m2.abs())
    if ds is not None:
        dx = dx + ds
        bound = bound + 2 * U32 * (dx.abs() + ds.abs())
    dw, db = (dy * n).sum(0), dy.sum(0)
    b_w = (T + 4) * U32 * (dy * n).abs().sum(0) + (dy.abs() * d_n).sum(0)
    b_b = (T + 4) * U32 * dy.abs().sum(0)
    return (dx, bound + rounding(dtype) * (dx.abs() + bound)), (dw, b_w), (db, b_b)


# --------------------------------------------------------------------------------------------------
# rotary positions
# --------------------------------------------------------------------------------------------------
def rotary(x, positions, freqs, sections, interleaved, inverse, dtype):
    pairs = freqs.shape[0]
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    angle = (positions.float()[:, axis] * freqs).double() * (-1 if inverse else 1)  # (the definition's 32-bit product)
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    i = torch.arange(pairs, device=x.device)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
    y, bound = x.clone(), torch.zeros_like(x)
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    size = x[..., a].abs() + x[..., b].abs()
    bound[..., a] = bound[..., b] = 6 * U32 * size  # (cosine and sine to 2 units in the last place, product, sum)
    return y, bound + rounding(dtype) * (y.abs() + bound)


# --------------------------------------------------------------------------------------------------
# attention
# --------------------------------------------------------------------------------------------------
def spans(total, offsets, lengths, count):
    if offsets is None:
        return [(0, total if lengths is None else min(total, int(lengths[0])))] * count
    at = [int(v) for v in offsets]
    return [(at[b], at[b + 1] - at[b] if lengths is None else min(at[b + 1] - at[b], int(lengths[b]))) for b in range(count)]


def _seen(Lq, Lk, causal, device):
    seen = torch.ones(Lq, Lk, dtype=torch.bool, device=device)
    return seen.tril(Lk - Lq) if causal else seen


def _scores(q, k, scale, seen):
    """Scores [Lq, Lk] with what the 32-bit sums of exact products, and the exponent's argument, may be off by."""
    s = (q @ k.T) * scale
    size = (q.abs() @ k.abs().T) * scale
    return s.masked_fill(~seen, -math.inf), (q.shape[1] + 4) * U32 * size + 8 * U32 * s.abs()


def attention(Q, K, V, causal, scale, q_spans, k_spans):
    """(O, bound, lse, bound) in 64 bits."""
    Q, K, V = Q.double(), K.double(), V.double()
    group = Q.shape[1] // K.shape[1]
    O, bO = torch.zeros_like(Q), torch.zeros_like(Q)
    lse = torch.full((Q.shape[1], Q.shape[0]), -math.inf, dtype=torch.float64, device=Q.device)
    bl = torch.zeros_like(lse)
    for (q0, Lq), (k0, Lk) in zip(q_spans, k_spans):
        if Lq == 0 or Lk == 0:
            continue
        seen = _seen(Lq, Lk, causal, Q.device)
        for h in range(Q.shape[1]):
            q, k, v = Q[q0:q0 + Lq, h], K[k0:k0 + Lk, h // group], V[k0:k0 + Lk, h // group]
            s, ds = _scores(q, k, scale, seen)
            any_seen = seen.any(1, keepdim=True)
            top = torch.where(any_seen, s.amax(1, keepdim=True), 0.0)
            e = torch.exp(s - top).masked_fill(~seen, 0.0)
            total = e.sum(1, keepdim=True)
            p = torch.where(any_seen, e / total.clamp(min=1e-300), 0.0)
            off = torch.where(seen, ds, 0.0).amax(1, keepdim=True) * 2 + (Lk + 16) * U32 + 64 * U32
            A = p @ v.abs()
            o = p @ v
            bound = (U16 * (1 + 2 * off) + 2 * off + (Lk + 8) * U32) * A  # p rounded, p's own error, the 32-bit sum
            O[q0:q0 + Lq, h] = o
            bO[q0:q0 + Lq, h] = bound + U16 * (o.abs() + bound)
            lse[h, q0:q0 + Lq] = torch.where(any_seen, top + total.log(), -math.inf).squeeze(1)
            bl[h, q0:q0 + Lq] = (off + 8 * U32 * (top.abs() + total.clamp(min=1).log() + 1)).squeeze(1)
    return O, bO, lse, bl


def attention_grad(dO, Q, K, V, O, lse, causal, scale, q_spans, k_spans):
    """((dQ, bound), (dK, bound), (dV, bound)) in 64 bits from O and lse as given."""
    dO, Q, K, V, O, lse = (t.double() for t in (dO, Q, K, V, O, lse))
    group = Q.shape[1] // K.shape[1]
    out = [torch.zeros_like(t) for t in (Q, K, V)]
    bounds = [torch.zeros_like(t) for t in (Q, K, V)]
    D = Q.shape[2]
    for (q0, Lq), (k0, Lk) in zip(q_spans, k_spans):
        if Lq == 0 or Lk == 0:
            continue
        seen = _seen(Lq, Lk, causal, Q.device)
        rq, rk = slice(q0, q0 + Lq), slice(k0, k0 + Lk)
        for h in range(Q.shape[1]):
            q, k, v, g, o = Q[rq, h], K[rk, h // group], V[rk, h // group], dO[rq, h], O[rq, h]
            s, ds_off = _scores(q, k, scale, seen)
            row = lse[h, rq, None]
            row = torch.where(torch.isinf(row), 0.0, row)
            p = torch.exp(s - row).masked_fill(~seen, 0.0)
            off = torch.where(seen, ds_off + 16 * U32 * (row.abs() + 1), 0.0)  # relative error of p
            delta, dp = (g * o).sum(1, keepdim=True), g @ v.T
            dp_off = (D + 4) * U32 * (g.abs() @ v.abs().T + (g * o).abs().sum(1, keepdim=True))
            z = p * (dp - delta)
            z_off = (U16 + 2 * off) * z.abs() + (1 + U16) * p * dp_off  # its rounding, p's error, the sums' errors
            p_off = (U16 + 2 * off) * p
            out[0][rq, h] = (z @ k) * scale
            b = ((z_off + (Lk + 8) * U32 * z.abs()) @ k.abs()) * scale
            bounds[0][rq, h] = b
            n = (group * Lq + 8) * U32
            out[1][rk, h // group] += (z.T @ q) * scale
            bounds[1][rk, h // group] += ((z_off + n * z.abs()).T @ q.abs()) * scale
            out[2][rk, h // group] += p.T @ g
            bounds[2][rk, h // group] += (p_off + n * p).T @ g.abs()
    return [(t, b + U16 * (t.abs() + b)) for t, b in zip(out, bounds)]
