"""The operators that stand between the linear layers of a transformer block, as a program that uses them meets them.

A block is: layer norm, the joint q/k/v projection, rotary positions on q and k, attention, the output projection added
to the residual stream, layer norm, the MLP.  The projections are the N:M-sparse layers of this library; what is measured
here is the rest:
  norm       layer norm of rows, optionally of the sum of two inputs (the residual stream and the branch just computed),
             which is returned too; backward: the input's gradient and the reductions over the rows for weight and bias
  rotary     rotary positions with one axis (text), two (height, width of an image) or three (time, height, width)
  attention  softmax attention over packed sequences of different lengths with grouped heads, causal or not; its backward
             pass; and a few new tokens per sequence against a long cache

Shapes are those of the blocks in `paper_2409_09708_amd.workloads` (width 768 in 12 heads of 64, images of 197 tokens;
the four-stage hierarchy that starts at 3136 tokens x 128 per image) and generic ones for text.  A case is a dict of
plain values, `kind` and `pass` name what is done.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6
LIMIT = 1 << 31  # scores of one attention case that the plain form may write out
INFINITY = float("inf")


# ------------------------------------------------------------------------------------------------------
# cases
# ------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one new token's row through a norm while decoding: nothing but latency
        {"name": "norm_one_row", "kind": "norm", "pass": "forward", "T": 1, "C": 768, "x": "bf16", "y": "bf16",
         "residual": True, "train": False, "pad": 0},
        # the first stage of the hierarchy at 64 images, fp32 residual stream: many short rows
        {"name": "norm_stage_64_images", "kind": "norm", "pass": "forward", "T": 200704, "C": 128, "x": "f32",
         "y": "bf16", "residual": True, "train": True, "pad": 0},
        # a training step at 256 images: gradients of the input, the weight and the bias
        {"name": "norm_backward_256_images", "kind": "norm", "pass": "backward", "T": 50432, "C": 768, "x": "bf16",
         "y": "bf16", "residual": True, "train": True, "pad": 0},
        # wide rows of an odd number of text tokens, width off every vector size, padded rows
        {"name": "norm_backward_ragged", "kind": "norm", "pass": "backward", "T": 4099, "C": 5003, "x": "f32", "y": "f32",
         "residual": False, "train": True, "pad": 5},
        # q and k of 64 images inside the joint projection's output, height and width of the patch grid
        {"name": "rotary_64_images", "kind": "rotary", "pass": "forward", "T": 12608, "H": 24, "D": 64, "R": 64, "axes": 2,
         "interleaved": False, "x": "bf16", "y": "bf16", "fused": True},
        # gradients of a video's q and k: time, height and width, part of each head turned, fp32 in and bf16 out
        {"name": "rotary_video_backward", "kind": "rotary", "pass": "backward", "T": 16399, "H": 10, "D": 128, "R": 96,
         "axes": 3, "interleaved": True, "x": "f32", "y": "bf16", "fused": False},
        # one image: a single short sequence
        {"name": "attention_1_image", "kind": "attention", "pass": "forward", "B": 1, "L": 197, "ctx": 0, "Hq": 12,
         "Hkv": 12, "D": 64, "causal": False, "ragged": 0},
        # a throughput batch of images through one block
        {"name": "attention_256_images", "kind": "attention", "pass": "forward", "B": 256, "L": 197, "ctx": 0, "Hq": 12,
         "Hkv": 12, "D": 64, "causal": False, "ragged": 0},
        # prompts of different lengths, packed, with four query heads to a key head: the largest case
        {"name": "attention_prompts", "kind": "attention", "pass": "forward", "B": 2, "L": 8191, "ctx": 0, "Hq": 16,
         "Hkv": 4, "D": 128, "causal": True, "ragged": 3},
        # a training step at 64 images
        {"name": "attention_backward_64_images", "kind": "attention", "pass": "backward", "B": 64, "L": 197, "ctx": 0,
         "Hq": 12, "Hkv": 12, "D": 64, "causal": False, "ragged": 0},
        # a training step on packed text with shared key heads
        {"name": "attention_backward_text", "kind": "attention", "pass": "backward", "B": 5, "L": 4093, "ctx": 0, "Hq": 16,
         "Hkv": 4, "D": 128, "causal": True, "ragged": 5},
        # one new token in each of 24 conversations against caches of up to 16k tokens
        {"name": "attention_cache_24", "kind": "attention", "pass": "cache", "B": 24, "L": 1, "ctx": 16384, "Hq": 32,
         "Hkv": 8, "D": 128, "causal": True, "ragged": 7},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "rotary", "attention", "attention", "attention"])
    if kind == "norm":
        C = rng.choice([128, 256, 384, 512, 768, 1024, 2048, 4096, 8 * rng.randint(8, 700), rng.randint(64, 5003)])
        T = _log_int(rng, 1, min(200704, 50432 * 768 // C))
        residual = rng.random() < 0.5
        return {"kind": kind, "pass": rng.choice(["forward", "backward"]), "T": T, "C": C, "x": rng.choice(["bf16", "f32"]),
                "y": rng.choice(["bf16", "bf16", "f32"]), "residual": residual, "train": rng.random() < 0.5,
                "pad": rng.choice([0, 0, 8, rng.randint(1, 9)])}
    if kind == "rotary":
        axes, D = rng.choice([1, 2, 3]), rng.choice([32, 64, 80, 96, 128])
        return {"kind": kind, "pass": rng.choice(["forward", "backward"]), "T": _log_int(rng, 1, 16399),
                "H": rng.randint(1, 24), "D": D, "R": rng.choice([D, D, D // 2]), "axes": axes,
                "interleaved": rng.random() < 0.3, "x": rng.choice(["bf16", "bf16", "f32"]), "y": rng.choice(["bf16", "f32"]),
                "fused": rng.random() < 0.5}
    Hkv, group, D = rng.choice([1, 2, 4, 8, 12]), rng.choice([1, 1, 2, 4, 8]), rng.choice([32, 64, 64, 80, 128, 128])
    what = rng.choice(["forward", "backward", "cache"])
    if what == "cache":
        L, ctx, causal = rng.choice([1, 1, 1, rng.randint(2, 8)]), _log_int(rng, 16, 16384), True
        B = _log_int(rng, 1, max(2, min(64, 24 * 16384 * 1024 // (ctx * Hkv * D))))
    else:
        most = LIMIT // (16 * Hkv * group)
        L, ctx, causal = _log_int(rng, 1, min(8191, math.isqrt(most))), 0, rng.random() < 0.6
        B = _log_int(rng, 1, max(1, min(256, most // (L * L))))
    return {"kind": kind, "pass": what, "B": B, "L": L, "ctx": ctx, "Hq": Hkv * group, "Hkv": Hkv, "D": D, "causal": causal,
            "ragged": rng.choice([0, rng.randint(1, 1 << 20)])}


def _lengths(case):
    """(tokens, keys) of each sequence.  Ragged: spread over the logarithm, the first one whole; a fourth and a fifth
    sequence are there with one token and with none.  Of a cache, keys count the new tokens too."""
    B, most = case["B"], case["ctx"] or case["L"]
    spread = [most] * B
    if case["ragged"]:
        rng = random.Random(case["ragged"])
        spread = [most] + [_log_int(rng, max(1, most // 64), most) for _ in range(B - 1)]
        if B > 4:
            spread[3], spread[4] = 1, 0
    if not case["ctx"]:
        return spread, spread
    return [case["L"]] * B, [min(most, n + case["L"]) for n in spread]


def _sections(case):
    """Rotated pairs of each axis: equal shares, the rest to the first."""
    pairs, axes = case["R"] // 2, case["axes"]
    return (pairs - (axes - 1) * (pairs // axes),) + (pairs // axes,) * (axes - 1)


# ------------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator("cuda")
    g.manual_seed(seed * 1000003 + 11)

    def normal(*shape, dtype="bf16", scale=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(DTYPES[dtype])

    return {"norm": _prepare_norm, "rotary": _prepare_rotary, "attention": _prepare_attention}[case["kind"]](case, normal, g)


def _prepare_norm(case, normal, g):
    T, C, pad = case["T"], case["C"], case["pad"]

    def rows(dtype, scale=1.0):
        return normal(T, C + pad, dtype=dtype, scale=scale)[:, :C]

    # a residual stream has an offset and a few wide channels; weights are near one
    s = {"case": case, "X": rows(case["x"]), "weight": 1 + 0.1 * normal(C, dtype="f32"), "bias": 0.1 * normal(C, dtype="f32")}
    s["X"] += 0.25 + 3 * (torch.rand(C, generator=g, device="cuda") < 0.01).to(s["X"].dtype)
    if case["pass"] == "forward":
        s["residual"] = rows(case["x"], 2.0) if case["residual"] else None
        return s
    s["stats"] = torch.stack(_plain_stats(s["X"].float()), 1)
    s["dY"] = rows(case["y"], 0.1)
    s["dS"] = rows(case["y"], 0.1) if case["residual"] else None
    return s


def _prepare_rotary(case, normal, g):
    T, H, D, axes = case["T"], case["H"], case["D"], case["axes"]
    if case["fused"]:  # q and k are the first heads of the projection's rows; a third as many again belong to v
        X = normal(T, (H + (H + 1) // 2) * D, dtype=case["x"])[:, :H * D].unflatten(1, (H, D))
    else:
        X = normal(T, H, D, dtype=case["x"])
    at = torch.arange(T, device="cuda")
    if axes == 1:    # text that starts somewhere in a long context
        positions = (at + int(torch.randint(0, 8192, (), generator=g, device="cuda")))[:, None]
    elif axes == 2:  # grids of 14 x 14 patches behind one token that stands for the image
        patch = (at % 197 - 1).clamp(min=0)
        positions = torch.stack([patch // 14, patch % 14], 1)
    else:            # frames of 16 x 16
        positions = torch.stack([at // 256, at // 16 % 16, at % 16], 1)
    freqs = [10000.0 ** (-torch.arange(n, device="cuda", dtype=torch.float32) / max(n, 1)) for n in _sections(case)]
    return {"case": case, "X": X, "positions": positions.to(torch.int32).contiguous(), "freqs": torch.cat(freqs)}


def _offsets(lengths):
    return torch.tensor([0] + lengths, dtype=torch.int64).cumsum(0).to(torch.int32).cuda()


def _prepare_attention(case, normal, g):
    B, Hq, Hkv, D = case["B"], case["Hq"], case["Hkv"], case["D"]
    nq, nk = _lengths(case)
    s = {"case": case, "offsets_q": _offsets(nq), "lengths_k": None, "max_q": max(nq), "max_k": max(nk),
         "scale": D ** -0.5}
    if case["pass"] == "cache":  # a cache of fixed capacity per sequence; what lies past a sequence's length is left over
        s["Q"] = normal(sum(nq), Hq, D)
        s["K"], s["V"] = normal(B * case["ctx"], Hkv, D), normal(B * case["ctx"], Hkv, D)
        s["offsets_k"] = _offsets([case["ctx"]] * B)
        s["lengths_k"] = torch.tensor(nk, dtype=torch.int32, device="cuda")
        return s
    qkv = normal(sum(nq), (Hq + 2 * Hkv) * D)  # the joint projection's output
    s["Q"], s["K"], s["V"] = (t.unflatten(1, (-1, D)) for t in qkv.split([Hq * D, Hkv * D, Hkv * D], 1))
    s["offsets_k"] = s["offsets_q"]
    if case["pass"] == "backward":
        s["O"], s["lse"] = _plain_attention(s)
        s["dO"] = normal(sum(nq), Hq, D)
    return s


# ------------------------------------------------------------------------------------------------------
# the operators
# ------------------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if own:
        return {"norm": _own_norm, "rotary": _own_rotary, "attention": _own_attention}[case["kind"]](s)
    return {"norm": _plain_norm, "rotary": _plain_rotary, "attention": _plain_any_attention}[case["kind"]](s)


def _own_norm(s):
    import paper_2409_09708_amd as nm
    case, out_dtype = s["case"], DTYPES[s["case"]["y"]]
    if case["pass"] == "forward":
        return nm.nm_layer_norm(s["X"], s["weight"], s["bias"], EPS, residual=s["residual"], train=case["train"],
                                out_dtype=out_dtype)
    return nm.nm_layer_norm_backward(s["dY"], s["X"], s["stats"], s["weight"], dS=s["dS"], out_dtype=DTYPES[case["x"]])


def _own_rotary(s):
    import paper_2409_09708_amd as nm
    case = s["case"]
    return nm.nm_rotary(s["X"], s["positions"], s["freqs"], sections=_sections(case), interleaved=case["interleaved"],
                        inverse=case["pass"] == "backward", out_dtype=DTYPES[case["y"]])


def _own_attention(s):
    import paper_2409_09708_amd as nm
    at = {k: s[k] for k in ("scale", "offsets_q", "offsets_k", "lengths_k", "max_q", "max_k")}
    causal, what = s["case"]["causal"], s["case"]["pass"]
    if what == "backward":
        return nm.nm_attention_backward(s["dO"], s["Q"], s["K"], s["V"], s["O"], s["lse"], causal, **at)
    return nm.nm_attention(s["Q"], s["K"], s["V"], causal, lse=what == "forward", **at)


def _plain_stats(x):
    mean = x.mean(1)
    return mean, ((x - mean[:, None]).square().mean(1) + EPS).rsqrt()


def _plain_norm(s):
    case, X = s["case"], s["X"].float()
    if case["pass"] == "forward":
        if s["residual"] is not None:
            X = X + s["residual"].float()
        mean, rstd = _plain_stats(X)
        Y = ((X - mean[:, None]) * rstd[:, None] * s["weight"] + s["bias"]).to(DTYPES[case["y"]])
        outs = (Y,) + ((X.to(DTYPES[case["x"]]),) if case["residual"] else ())
        outs += (torch.stack([mean, rstd], 1),) if case["train"] else ()
        return outs if len(outs) > 1 else Y
    mean, rstd = s["stats"][:, :1], s["stats"][:, 1:]
    dY, hat = s["dY"].float(), (X - mean) * rstd
    g = dY * s["weight"]
    dX = rstd * (g - g.mean(1, keepdim=True) - hat * (g * hat).mean(1, keepdim=True))
    if s["dS"] is not None:
        dX = dX + s["dS"].float()
    return dX.to(DTYPES[case["x"]]), (dY * hat).sum(0), dY.sum(0)


def _plain_rotary(s):
    case, X, R = s["case"], s["X"].float(), s["case"]["R"]
    axis = torch.repeat_interleave(torch.tensor(_sections(case), device="cuda"), output_size=R // 2)
    angle = s["positions"].float()[:, axis] * s["freqs"]
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    if case["pass"] == "backward":
        sin = -sin
    turned, rest = X[..., :R], X[..., R:]
    if case["interleaved"]:
        a, b = turned[..., 0::2], turned[..., 1::2]
        out = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = turned.chunk(2, -1)
        out = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([out, rest], -1).to(DTYPES[case["y"]])


def _padded(s):
    """The packed inputs as [B, key heads, ...] blocks of the longest length, and what of them is there: indices of the rows
    that pad and unpad tokens, and which scores count."""
    offsets_q, offsets_k = s["offsets_q"].long(), s["offsets_k"].long()
    nq = offsets_q.diff()
    nk = s["lengths_k"].long() if s["lengths_k"] is not None else offsets_k.diff()
    at_q, at_k = torch.arange(s["max_q"], device="cuda"), torch.arange(s["max_k"], device="cuda")
    rows_q = (offsets_q[:-1, None] + at_q).clamp(max=s["Q"].shape[0] - 1)
    rows_k = (offsets_k[:-1, None] + at_k).clamp(max=s["K"].shape[0] - 1)
    there_q, there_k = at_q < nq[:, None], at_k < nk[:, None]
    seen = there_k[:, None, :] & there_q[:, :, None]
    if s["case"]["causal"]:
        seen = seen & (at_k[None, None, :] <= at_q[None, :, None] + (nk - nq)[:, None, None])
    return rows_q, rows_k, there_q, there_k, seen


def _heads(x, rows, Hkv, there):
    """[T, H, D] -> [B, Hkv, H / Hkv, L, D] in 32 bits, with zeros where no token is."""
    x = torch.where(there[..., None, None], x[rows].float(), 0.0)
    return x.unflatten(2, (Hkv, -1)).permute(0, 2, 3, 1, 4).contiguous()


def _packed(x, there):
    """[B, Hkv, group, L, D] -> [T, Hkv * group, D]."""
    return x.permute(0, 3, 1, 2, 4).flatten(2, 3)[there]


def _product(a, b):
    """a [B, Hkv, group, L, n] times b [B, Hkv, n, m]: the heads of a group are rows of one product."""
    return (a.flatten(2, 3) @ b).unflatten(2, a.shape[2:4])


def _over_rows(a, b):
    """The sum over a group's heads and tokens of a^T b, [B, Hkv, 1, n, m]."""
    return (a.flatten(2, 3).transpose(-1, -2) @ b.flatten(2, 3)).unsqueeze(2)


def _plain_attention(s):
    Hkv = s["case"]["Hkv"]
    rows_q, rows_k, there_q, there_k, seen = _padded(s)
    Q, K, V = _heads(s["Q"], rows_q, Hkv, there_q), _heads(s["K"], rows_k, Hkv, there_k), _heads(s["V"], rows_k, Hkv, there_k)
    S = torch.where(seen[:, None, None], _product(Q, K.squeeze(2).transpose(-1, -2)) * s["scale"], -INFINITY)
    top = S.amax(-1, keepdim=True)
    P = torch.exp(S - torch.where(top == -INFINITY, 0.0, top))
    total = P.sum(-1, keepdim=True)
    O = torch.where(total > 0, _product(P, V.squeeze(2)) / total, 0.0)
    lse = torch.where(total > 0, top + total.log(), -INFINITY)
    return _packed(O, there_q).to(torch.bfloat16), _packed(lse, there_q).squeeze(-1).T.contiguous()


def _plain_any_attention(s):
    what = s["case"]["pass"]
    if what != "backward":
        O, lse = _plain_attention(s)
        return (O, lse) if what == "forward" else O
    Hkv, scale = s["case"]["Hkv"], s["scale"]
    rows_q, rows_k, there_q, there_k, seen = _padded(s)
    Q, dO, O = (_heads(s[k], rows_q, Hkv, there_q) for k in ("Q", "dO", "O"))
    K, V = (_heads(s[k], rows_k, Hkv, there_k).squeeze(2) for k in ("K", "V"))
    lse = _heads(s["lse"].T[..., None], rows_q, Hkv, there_q)
    S = _product(Q, K.transpose(-1, -2)) * scale
    P = torch.where(seen[:, None, None], torch.exp(S - torch.where(lse == -INFINITY, 0.0, lse)), 0.0)
    dS = P * (_product(dO, V.transpose(-1, -2)) - (dO * O).sum(-1, keepdim=True)) * scale
    dQ, dK, dV = _product(dS, K), _over_rows(dS, Q), _over_rows(P, dO)
    return tuple(_packed(d, t).to(torch.bfloat16) for d, t in ((dQ, there_q), (dK, there_k), (dV, there_k)))


# ------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "rotary": _exact_rotary, "attention": _exact_attention}[case["kind"]](case, s)


def _exact_norm(case, s):
    x = s["X"].double()
    if case["pass"] == "forward":
        if case["residual"]:
            x += s["residual"].double()
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = 1 / torch.sqrt(var + EPS)
        y = torch.addcmul(s["bias"].double(), x.sub(mean[:, None]).mul_(rstd[:, None]), s["weight"].double())
        outs = [y] + ([x] if case["residual"] else []) + ([torch.stack((mean, rstd), 1)] if case["train"] else [])
        return tuple(outs) if len(outs) > 1 else y
    # the normalised row is n; with u = dL/dn the input's gradient is rstd times u with its parts along 1 and n taken out
    mean, rstd = s["stats"].double().unbind(1)
    n = (x - mean[:, None]) * rstd[:, None]
    dy = s["dY"].double()
    u = dy * s["weight"].double()
    along = torch.einsum("tc,tc->t", u, n)[:, None] / case["C"]
    dx = (u - u.sum(1, keepdim=True) / case["C"] - along * n) * rstd[:, None]
    if s["dS"] is not None:
        dx += s["dS"].double()
    return dx, torch.einsum("tc,tc->c", dy, n), dy.sum(0)


def _exact_rotary(case, s):
    # a pair is a complex number, turned by its angle
    x, R, way = s["X"].double(), case["R"], -1 if case["pass"] == "backward" else 1
    out, first = x.clone(), 0
    for axis, n in enumerate(_sections(case)):
        pairs = torch.arange(first, first + n, device="cuda")
        a, b = (2 * pairs, 2 * pairs + 1) if case["interleaved"] else (pairs, pairs + R // 2)
        turn = torch.outer(s["positions"][:, axis].double(), s["freqs"][pairs].double()) * way
        z = torch.complex(x[..., a], x[..., b]) * torch.polar(torch.ones_like(turn), turn)[:, None]
        out[..., a], out[..., b] = z.real, z.imag
        first += n
    return out


def _exact_attention(case, s):
    """One sequence and one key head at a time, over the keys that a token sees."""
    nq, nk = _lengths(case)
    Hkv, group, what = case["Hkv"], case["Hq"] // case["Hkv"], case["pass"]
    if what == "backward":
        outs = [torch.zeros(s[k].shape, dtype=torch.float64, device="cuda") for k in ("Q", "K", "V")]
    else:
        outs = [torch.zeros(s["Q"].shape, dtype=torch.float64, device="cuda"),
                torch.full((case["Hq"], sum(nq)), -INFINITY, dtype=torch.float64, device="cuda")]
    q0 = k0 = 0
    for Lq, Lk in zip(nq, nk):
        rq, rk = slice(q0, q0 + Lq), slice(k0, k0 + Lk)
        q0, k0 = q0 + Lq, k0 + (case["ctx"] or Lk)
        if Lq == 0 or Lk == 0:
            continue
        hidden = None
        if case["causal"]:
            hidden = torch.ones(Lq, Lk, dtype=torch.bool, device="cuda").triu(Lk - Lq + 1)
        for h in range(Hkv):
            hq = slice(h * group, (h + 1) * group)
            q = s["Q"][rq, hq].double().transpose(0, 1).contiguous()
            k, v = s["K"][rk, h].double().contiguous(), s["V"][rk, h].double().contiguous()
            z = torch.matmul(q, k.T.contiguous()) * s["scale"]
            if hidden is not None:
                z.masked_fill_(hidden, -INFINITY)
            if what != "backward":
                outs[1][hq, rq] = torch.logsumexp(z, -1)
                outs[0][rq, hq] = torch.matmul(torch.softmax(z, -1), v).transpose(0, 1)
                continue
            p = torch.exp(z - s["lse"][hq, rq].double()[..., None])
            do, o = (s[n][rq, hq].double().transpose(0, 1).contiguous() for n in ("dO", "O"))
            dz = p * (torch.matmul(do, v.T.contiguous()) - (do * o).sum(-1, keepdim=True)) * s["scale"]
            outs[0][rq, hq] = torch.matmul(dz, k).transpose(0, 1)
            outs[1][rk, h] = dz.flatten(0, 1).T @ q.flatten(0, 1)
            outs[2][rk, h] = p.flatten(0, 1).T @ do.flatten(0, 1)
    return tuple(outs) if what != "cache" else outs[0]


# ------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------------
def work(case):
    size = {"bf16": 2, "f32": 4}
    if case["kind"] == "norm":
        n, x, y = case["T"] * case["C"], size[case["x"]], size[case["y"]]
        if case["pass"] == "forward":
            moved = n * (x + y + (2 * x if case["residual"] else 0)) + 8 * case["C"] + (8 * case["T"] if case["train"] else 0)
            return {"bytes": moved, "flops": 8 * n}
        return {"bytes": n * (2 * x + y + (y if case["residual"] else 0)) + 8 * case["T"] + 12 * case["C"], "flops": 14 * n}
    if case["kind"] == "rotary":
        n = case["T"] * case["H"] * case["D"]
        return {"bytes": n * (size[case["x"]] + size[case["y"]]) + 4 * case["T"] * case["axes"] + 2 * case["R"],
                "flops": 3 * case["T"] * case["H"] * case["R"]}
    nq, nk = _lengths(case)
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    if case["causal"]:
        pairs = sum(Lq * Lk - Lq * (Lq - 1) // 2 if Lk >= Lq else Lk * (Lk + 1) // 2 for Lq, Lk in zip(nq, nk))
    else:
        pairs = sum(a * b for a, b in zip(nq, nk))
    q, k, lse = 2 * sum(nq) * Hq * D, 2 * sum(nk) * Hkv * D, 4 * sum(nq) * Hq
    if case["pass"] == "backward":
        return {"bytes": 4 * q + 4 * k + lse, "flops": 10 * D * pairs * Hq}
    return {"bytes": 2 * q + 2 * k + (lse if case["pass"] == "forward" else 0), "flops": 4 * D * pairs * Hq}
