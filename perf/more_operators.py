"""What a transformer block adds to attention when it serves: norms of queries and keys, and a cache in pages.

  head_norm  each head of q and k is normed over its own elements (root mean square, or layer norm) and turned by its
             rotary position, one pass over the joint projection's output; backward: the gradient of that output and of the
             two weights
  cache      new keys and values go to the pages of their sequences, as bfloat16 or in 8 bits (e4m3 codes and a power of
             two for each head of a token), and tokens are read back from there as bfloat16
  paged      softmax attention of new tokens, one or a chunk per sequence, over such a cache; all keys before a token, or
             the last few of them (window) and the very first (sinks)

Shapes are those of the blocks in `paper_2409_09708_amd.workloads` (heads of 64, images of 197 tokens) and generic ones
for text.  A case is a dict of plain values, `kind` and `pass` name what is done.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
E4M3 = torch.float8_e4m3fn
EPS = 1e-6
LOWEST, HIGHEST = -100, 119  # exponents that a row's power of two may have
INFINITY = float("inf")


# ------------------------------------------------------------------------------------------------------
# cases
# ------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one new token's queries and keys while decoding: nothing but latency
        {"name": "head_norm_one_token", "kind": "head_norm", "pass": "forward", "T": 1, "Hq": 32, "Hk": 8, "D": 128, "R": 128,
         "axes": 1, "interleaved": False, "centred": False, "x": "bf16", "y": "bf16", "fused": True},
        # 64 images: layer norm of 24 heads inside the joint projection's output, height and width of the patch grid
        {"name": "head_norm_64_images", "kind": "head_norm", "pass": "forward", "T": 12608, "Hq": 12, "Hk": 12, "D": 64, "R": 64,
         "axes": 2, "interleaved": False, "centred": True, "x": "bf16", "y": "bf16", "fused": True},
        # a training step on packed text with shared key heads
        {"name": "head_norm_backward_text", "kind": "head_norm", "pass": "backward", "T": 8191, "Hq": 32, "Hk": 8, "D": 128,
         "R": 128, "axes": 1, "interleaved": False, "centred": False, "x": "bf16", "y": "bf16", "fused": True},
        # a video's heads off the powers of two, float, part of each head turned by neighbours
        {"name": "head_norm_backward_video", "kind": "head_norm", "pass": "backward", "T": 16399, "Hq": 7, "Hk": 3, "D": 80,
         "R": 72, "axes": 3, "interleaved": True, "centred": True, "x": "f32", "y": "f32", "fused": False},
        # a decoding step: one token of each of 48 conversations into caches of 8 bits (and as the cache holds it)
        {"name": "cache_write_step", "kind": "cache", "pass": "write", "B": 48, "new": 1, "ctx": 4096, "H": 8, "D": 128,
         "page": 16, "format": "e4m3", "ragged": 3},
        # prompts of different lengths into fresh caches of 8 bits
        {"name": "cache_write_prompts", "kind": "cache", "pass": "write", "B": 7, "new": 8191, "ctx": 8191, "H": 8, "D": 128,
         "page": 64, "format": "e4m3", "ragged": 5},
        # whole caches read back, to be handed to another machine or another format
        {"name": "cache_read_24", "kind": "cache", "pass": "read", "B": 24, "new": 0, "ctx": 16384, "H": 8, "D": 128,
         "page": 16, "format": "e4m3", "ragged": 7},
        # one conversation that has just begun: nothing but latency
        {"name": "paged_one", "kind": "paged", "pass": "decode", "B": 1, "L": 1, "ctx": 200, "Hq": 12, "Hkv": 12, "D": 64,
         "page": 16, "format": "bf16", "window": 0, "sinks": 0, "ragged": 0},
        # one new token in each of 24 conversations against caches of up to 16k tokens in 8 bits
        {"name": "paged_24", "kind": "paged", "pass": "decode", "B": 24, "L": 1, "ctx": 16384, "Hq": 32, "Hkv": 8, "D": 128,
         "page": 16, "format": "e4m3", "window": 0, "sinks": 0, "ragged": 7},
        # three tokens at a time of long streams: the last 4095 tokens and the first four are seen, pages between are gone
        {"name": "paged_streams", "kind": "paged", "pass": "decode", "B": 40, "L": 3, "ctx": 20000, "Hq": 16, "Hkv": 4, "D": 128,
         "page": 64, "format": "bf16", "window": 4095, "sinks": 4, "ragged": 9},
        # the next chunk of two long prompts: the largest case
        {"name": "paged_chunk", "kind": "paged", "pass": "chunk", "B": 2, "L": 2047, "ctx": 16384, "Hq": 16, "Hkv": 4, "D": 128,
         "page": 64, "format": "bf16", "window": 0, "sinks": 0, "ragged": 1},
        # chunks of several prompts on caches of 8 bits and small pages, under a window
        {"name": "paged_chunk_window", "kind": "paged", "pass": "chunk", "B": 5, "L": 1000, "ctx": 6000, "Hq": 16, "Hkv": 8, "D": 128,
         "page": 16, "format": "e4m3", "window": 1024, "sinks": 16, "ragged": 11},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["head_norm", "head_norm", "cache", "paged", "paged", "paged"])
    if kind == "head_norm":
        D = rng.choice([32, 64, 64, 80, 96, 128, 128, 256, rng.randint(9, 256)])
        Hk = rng.choice([1, 2, 3, 4, 8, 12])
        Hq = Hk * rng.choice([1, 1, 2, 4])
        axes = rng.choice([0, 1, 1, 2, 3])
        R = 2 * rng.randint(max(axes, 1), D // 2) if rng.random() < 0.3 else D // 2 * 2
        T = _log_int(rng, 1, min(16399, 8191 * 40 * 128 // ((Hq + Hk) * D)))
        return {"kind": kind, "pass": rng.choice(["forward", "backward"]), "T": T, "Hq": Hq, "Hk": Hk, "D": D, "R": R if axes else 0,
                "axes": axes, "interleaved": rng.random() < 0.3, "centred": rng.random() < 0.4,
                "x": rng.choice(["bf16", "bf16", "f32"]), "y": rng.choice(["bf16", "bf16", "f32"]), "fused": rng.random() < 0.5}
    page, form = rng.choice([1, 8, 16, 16, 32, 64, 64, 128, 256, rng.randint(2, 100)]), rng.choice(["e4m3", "e4m3", "bf16"])
    ragged = rng.choice([0, rng.randint(1, 1 << 20)])
    D = rng.choice([32, 64, 64, 80, 128, 128, 128, rng.randint(8, 128)])
    if kind == "cache":
        H, what = rng.choice([1, 2, 4, 8, 12]), rng.choice(["write", "write", "read"])
        ctx = _log_int(rng, 1, 16384)
        new = 0 if what == "read" else rng.choice([1, min(ctx, rng.randint(2, 8)), ctx])
        B = _log_int(rng, 1, max(2, min(64, 24 * 16384 * 1024 // (8 * ctx * H * D))))
        return {"kind": kind, "pass": what, "B": B, "new": new, "ctx": ctx, "H": H, "D": D, "page": page, "format": form, "ragged": ragged}
    Hkv, group = rng.choice([1, 2, 4, 8, 12]), rng.choice([1, 1, 2, 4, 8])
    what = rng.choice(["decode", "decode", "chunk"])
    window = rng.choice([0, 0, _log_int(rng, 1, 8192)])
    sinks = rng.choice([0, 1, 4, rng.randint(2, 100)]) if window else 0
    if what == "decode":
        L, ctx = rng.choice([1, 1, 1, rng.randint(2, 8)]), _log_int(rng, 16, 16384)
        B = _log_int(rng, 1, max(2, min(64, 24 * 16384 * 1024 // (ctx * Hkv * D))))
    else:
        L = _log_int(rng, 9, 2047)
        ctx = max(L, _log_int(rng, 16, 16384))
        B = _log_int(rng, 1, max(1, min(8, 2047 * 16384 * 16 * 128 // (L * ctx * Hkv * group * max(D, 64)))))
    return {"kind": kind, "pass": what, "B": B, "L": L, "ctx": ctx, "Hq": Hkv * group, "Hkv": Hkv, "D": D, "page": page, "format": form,
            "window": window, "sinks": sinks, "ragged": ragged}


def _spread(rng, most, count):
    """Lengths spread over the logarithm, the first one whole."""
    return [most] + [_log_int(rng, max(1, most // 64), most) for _ in range(count - 1)]


def _lengths(case):
    """(new tokens, tokens in the cache with the new ones) of each sequence.  Ragged: of different lengths, and of six or more
    one has no new tokens and one has nothing but its new ones."""
    B, ctx, new = case["B"], case["ctx"], case["L"] if case["kind"] == "paged" else case["new"]
    if not case["ragged"]:
        return [new] * B, [ctx] * B
    rng = random.Random(case["ragged"])
    tokens = [min(ctx, n + new) for n in _spread(rng, ctx, B)]
    fresh = _spread(rng, new, B) if new > 8 else [new] * B
    fresh = [min(n, t) for n, t in zip(fresh, tokens)]
    if case["kind"] == "cache" and new == ctx:  # (prompts into empty caches)
        tokens = fresh
    if B > 5:
        fresh[4], tokens[5] = 0, fresh[5]
    return fresh, tokens


def _sections(case):
    """Turned pairs of each axis: equal shares, the rest to the first."""
    pairs, axes = case["R"] // 2, case["axes"]
    return (pairs - (axes - 1) * (pairs // axes),) + (pairs // axes,) * (axes - 1)


# ------------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator("cuda")
    g.manual_seed(seed * 1000003 + 13)
    return {"head_norm": _prepare_head_norm, "cache": _prepare_cache, "paged": _prepare_paged}[case["kind"]](case, g)


def _normal(g, *shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _prepare_head_norm(case, g):
    T, Hq, Hk, D, axes = case["T"], case["Hq"], case["Hk"], case["D"], case["axes"]
    H = Hq + Hk

    def rows(dtype):
        if case["fused"]:  # q and k are the first heads of the projection's rows; the key heads' number again belongs to v
            return _normal(g, T, (H + Hk) * D, dtype=DTYPES[dtype])[:, :H * D].unflatten(1, (H, D))
        return _normal(g, T, H, D, dtype=DTYPES[dtype])

    # heads have sizes of their own, an offset, and a few wide channels; weights are near one
    s = {"case": case, "X": rows(case["x"]), "weight": 1 + 0.1 * _normal(g, 2, D, dtype=torch.float32), "positions": None, "freqs": None}
    wide = 1 + 4 * (torch.rand(H, D, generator=g, device="cuda") < 0.02).float()
    s["X"].mul_(wide * torch.exp(_normal(g, H, 1, dtype=torch.float32))).add_(0.25)
    if case["pass"] == "backward":
        s["dY"] = rows(case["y"]).mul_(0.1)
    if axes:
        at = torch.arange(T, device="cuda")
        if axes == 1:    # text somewhere in a long context
            positions = (at + int(torch.randint(0, 65536, (), generator=g, device="cuda")))[:, None]
        elif axes == 2:  # grids of 14 x 14 patches behind one token that stands for the image
            patch = (at % 197 - 1).clamp(min=0)
            positions = torch.stack([patch // 14, patch % 14], 1)
        else:            # frames of 16 x 16
            positions = torch.stack([at // 256, at // 16 % 16, at % 16], 1)
        s["positions"] = positions.to(torch.int32).contiguous()
        s["freqs"] = torch.cat([10000.0 ** (-torch.arange(n, device="cuda", dtype=torch.float32) / max(n, 1)) for n in _sections(case)])
    return s


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _offsets(lengths):
    return torch.tensor([0] + lengths, dtype=torch.int64).cumsum(0).to(torch.int32).cuda()


def _pages(case, g, H, D, filled):
    """Pages for every sequence's tokens, in an order of chance, a page's heads one after another; a few pages more are there,
    and so are what earlier sequences left in them."""
    page, B = case["page"], case["B"]
    width = -(-case["ctx"] // page)
    count = B * width + 3
    table = torch.randperm(count, generator=g, device="cuda")[:B * width].view(B, width).to(torch.int32)
    s = {"case": case, "table": table, "page": page}
    for name in ("K", "V"):
        if filled:
            rows = _normal(g, count, H, page, D)
            rows *= torch.exp2(torch.randint(-1, 2, (count, H, page, 1), generator=g, device="cuda")).to(rows.dtype)
        else:
            rows = torch.zeros(count, H, page, D, dtype=torch.bfloat16, device="cuda")
        scales = None
        if case["format"] == "e4m3":
            rows, scales = _plain_codes(rows)
            scales = scales.transpose(1, 2)
        s[name + "_pages"], s[name + "_scales"] = rows.transpose(1, 2), scales
    return s


def _prepare_cache(case, g):
    H, D = case["H"], case["D"]
    new, tokens = _lengths(case)
    s = _pages(case, g, H, D, case["new"] < case["ctx"])
    s["lengths"] = _ints(tokens)
    if case["pass"] == "read":
        s["first"], s["offsets"], s["tokens"] = None, _offsets(tokens), sum(tokens)
        return s
    # keys and values are part of the joint projection's output, four query heads to each
    row = _normal(g, sum(new), 6 * H * D)
    wide = 1 + 8 * (torch.rand(6 * H * D, generator=g, device="cuda") < 0.02).to(row.dtype)
    s["K"], s["V"] = (t.unflatten(1, (H, D)) for t in row.mul_(wide)[:, 4 * H * D:].split(H * D, 1))
    s["first"], s["offsets"], s["tokens"] = _ints([t - n for n, t in zip(new, tokens)]), _offsets(new), sum(new)
    return s


def _prepare_paged(case, g):
    new, tokens = _lengths(case)
    s = _pages(case, g, case["Hkv"], case["D"], True)
    s["lengths"], s["max_q"], s["max_k"] = _ints(tokens), max(new), max(tokens)
    s["offsets"] = _offsets(new)
    s["Q"] = _normal(g, sum(new), (case["Hq"] + 2 * case["Hkv"]) * case["D"])[:, :case["Hq"] * case["D"]].unflatten(1, (-1, case["D"]))
    s["scale"] = case["D"] ** -0.5
    if case["window"]:  # pages that no token can see any more have been given back
        at = torch.arange(s["table"].shape[1], device="cuda") * case["page"]
        first_seen = s["lengths"][:, None] - _ints(new)[:, None] + 1 - case["window"]
        s["table"] = torch.where((at >= case["sinks"]) & (at + case["page"] <= first_seen), -1, s["table"]).contiguous()
    return s


# ------------------------------------------------------------------------------------------------------
# the operators
# ------------------------------------------------------------------------------------------------------
def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"head_norm": _own_head_norm, "cache": _own_cache, "paged": _own_paged}[kind](s)
    return {"head_norm": _plain_head_norm, "cache": _plain_cache, "paged": _plain_paged}[kind](s)


def _own_head_norm(s):
    import paper_2409_09708_amd as nm
    case = s["case"]
    how = {"heads": case["Hq"], "eps": EPS, "centred": case["centred"], "positions": s["positions"], "freqs": s["freqs"],
           "sections": _sections(case) if case["axes"] else None, "interleaved": case["interleaved"]}
    if case["pass"] == "forward":
        return nm.nm_head_norm(s["X"], s["weight"], out_dtype=DTYPES[case["y"]], **how)
    return nm.nm_head_norm_backward(s["dY"], s["X"], s["weight"], out_dtype=DTYPES[case["x"]], **how)


def _own_cache(s):
    import paper_2409_09708_amd as nm
    scales = {"K_scales": s["K_scales"], "V_scales": s["V_scales"]}
    if s["case"]["pass"] == "write":
        nm.nm_cache_write(s["K"], s["V"], s["K_pages"], s["V_pages"], s["table"], s["lengths"], offsets=s["offsets"], **scales)
    return nm.nm_cache_read(s["K_pages"], s["V_pages"], s["table"], s["lengths"], s["offsets"], tokens=s["tokens"], first=s["first"],
                            **scales)


def _own_paged(s):
    import paper_2409_09708_amd as nm
    return nm.nm_attention_paged(s["Q"], s["K_pages"], s["V_pages"], s["table"], s["lengths"], s["scale"], offsets_q=s["offsets"],
                                 window=s["case"]["window"], sinks=s["case"]["sinks"], K_scales=s["K_scales"], V_scales=s["V_scales"],
                                 max_q=s["max_q"], max_k=s["max_k"], lse=s["case"]["pass"] == "chunk")


def _plain_turn(s, x, back):
    """x's pairs turned by their angles, which are taken in 64 bits: far positions have many turns."""
    case, R = s["case"], s["case"]["R"]
    if not case["axes"]:
        return x
    axis = torch.repeat_interleave(torch.tensor(_sections(case), device="cuda"), output_size=R // 2)
    angle = s["positions"].double()[:, axis] * s["freqs"].double()
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if back:
        sin = -sin
    turned, rest = x[..., :R], x[..., R:]
    if case["interleaved"]:
        a, b = turned[..., 0::2], turned[..., 1::2]
        out = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = turned.chunk(2, -1)
        out = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([out, rest], -1)


def _plain_head_norm(s):
    case, x, Hq = s["case"], s["X"].float(), s["case"]["Hq"]
    w = torch.where(torch.arange(x.shape[1], device="cuda")[:, None] < Hq, s["weight"][0], s["weight"][1])
    if case["centred"]:
        x = x - x.mean(-1, keepdim=True)
    rstd = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
    n = x * rstd
    if case["pass"] == "forward":
        return _plain_turn(s, n * w, False).to(DTYPES[case["y"]])
    dy = _plain_turn(s, s["dY"].float(), True)
    g = dy * w
    dx = g - n * (g * n).mean(-1, keepdim=True)
    if case["centred"]:
        dx = dx - g.mean(-1, keepdim=True)
    dw = dy * n
    return (dx * rstd).to(DTYPES[case["x"]]), torch.stack([dw[:, :Hq].sum((0, 1)), dw[:, Hq:].sum((0, 1))])


def _power(exponent):
    """Two to the given whole numbers, in 32 bits."""
    return (exponent.to(torch.int32) + 127 << 23).view(torch.float32)


def _plain_codes(x):
    """(codes, exponent bytes) of rows of bfloat16: the smallest power of two that leaves no element above 448, the largest
    number of the format; elements over it rounded to four significant bits, or multiples of 2^-9."""
    x = x.float()
    top = torch.where(x.isfinite(), x.abs(), 0.0).amax(-1, keepdim=True)
    mantissa, exponent = torch.frexp(top)
    exponent = torch.where(top == 0, LOWEST, torch.where(mantissa > 0.875, exponent - 8, exponent - 9).clamp(LOWEST, HIGHEST))
    y = torch.where(x.isfinite(), (x * _power(-exponent)).clamp(-448, 448), math.nan)
    step = _power((torch.frexp(y).exponent - 1).clamp(min=-6) - 3)
    y = (y / step).round() * step
    return y.to(E4M3), (exponent + 127).squeeze(-1).to(torch.uint8)


def _bytes(pages):
    return pages.view(torch.uint8) if pages.dtype == E4M3 else pages


def _plain_rows(s, name, entry, slot):
    """Tokens of the pages as they are, in 32 bits."""
    rows = _bytes(s[name + "_pages"])[entry, slot]
    if s[name + "_scales"] is None:
        return rows.float()
    return rows.view(E4M3).float() * _power(s[name + "_scales"][entry, slot].int() - 127)[..., None]


def _places(s, seq, at):
    """Page and slot of token `at` of sequence `seq`."""
    page = s["page"]
    return s["table"][seq, at // page].long(), at % page


def _packed_tokens(s):
    """Sequence of each packed token, and its place in the sequence."""
    rows = torch.arange(s["tokens"], device="cuda")
    seq = torch.searchsorted(s["offsets"][1:].long(), rows, right=True)
    at = rows - s["offsets"].long()[seq]
    return seq, at if s["first"] is None else at + s["first"].long()[seq]


def _plain_cache(s):
    entry, slot = _places(s, *_packed_tokens(s))
    if s["case"]["pass"] == "write":
        for name in ("K", "V"):
            if s[name + "_scales"] is None:
                s[name + "_pages"][entry, slot] = s[name]
            else:
                codes, scales = _plain_codes(s[name])
                _bytes(s[name + "_pages"])[entry, slot] = _bytes(codes)
                s[name + "_scales"][entry, slot] = scales
    return tuple(_plain_rows(s, name, entry, slot).to(torch.bfloat16) for name in ("K", "V"))


def _plain_paged(s):
    case, B, Hkv = s["case"], s["case"]["B"], s["case"]["Hkv"]
    offsets, tokens = s["offsets"].long(), s["lengths"].long()
    new = offsets.diff()
    at_q, at_k = torch.arange(s["max_q"], device="cuda"), torch.arange(s["max_k"], device="cuda")
    rows_q = (offsets[:-1, None] + at_q).clamp(max=s["Q"].shape[0] - 1)
    there_q = at_q < new[:, None]
    position = tokens[:, None] - new[:, None] + at_q
    seen = (at_k <= position[..., None]) & there_q[..., None]
    if case["window"]:
        seen &= (at_k > position[..., None] - case["window"]) | (at_k < case["sinks"])
    entry, slot = _places(s, torch.arange(B, device="cuda")[:, None], at_k[None])
    there_k = (seen.any(1) & (entry >= 0))[..., None, None]
    entry = entry.clamp(min=0)
    K, V = (torch.where(there_k, _plain_rows(s, name, entry, slot.expand_as(entry)), 0.0).transpose(1, 2).contiguous() for name in ("K", "V"))
    Q = torch.where(there_q[..., None, None], s["Q"][rows_q].float(), 0.0).unflatten(2, (Hkv, -1)).permute(0, 2, 3, 1, 4).contiguous()
    group = Q.shape[2]
    S = (Q.flatten(2, 3) @ K.transpose(-1, -2).contiguous()).unflatten(2, (group, -1)) * s["scale"]
    S = torch.where(seen[:, None, None], S, -INFINITY)
    top = S.amax(-1, keepdim=True)
    P = torch.exp(S - torch.where(top == -INFINITY, 0.0, top))
    total = P.sum(-1, keepdim=True)
    O = torch.where(total > 0, (P.flatten(2, 3) @ V).unflatten(2, (group, -1)) / total, 0.0)
    O = O.permute(0, 3, 1, 2, 4).flatten(2, 3)[there_q].to(torch.bfloat16)
    if case["pass"] == "decode":
        return O
    lse = torch.where(total > 0, top + total.log(), -INFINITY)
    return O, lse.permute(0, 3, 1, 2, 4).flatten(2)[there_q].T.contiguous()


# ------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"head_norm": _exact_head_norm, "cache": _exact_cache, "paged": _exact_paged}[case["kind"]](case, s)


def _exact_head_norm(case, s):
    # a pair is a complex number, turned by its angle
    def turn(x, way):
        out, first = x.clone(), 0
        for axis, n in enumerate(_sections(case) if case["axes"] else ()):
            pairs = torch.arange(first, first + n, device="cuda")
            a, b = (2 * pairs, 2 * pairs + 1) if case["interleaved"] else (pairs, pairs + case["R"] // 2)
            angle = torch.outer(s["positions"][:, axis].double(), s["freqs"][pairs].double()) * way
            z = torch.complex(x[..., a], x[..., b]) * torch.polar(torch.ones_like(angle), angle)[:, None]
            out[..., a], out[..., b] = z.real, z.imag
            first += n
        return out

    Hq, D = case["Hq"], case["D"]
    x = s["X"].double()
    which = [0] * Hq + [1] * case["Hk"]
    w = s["weight"].double()[which]
    if case["centred"]:
        var, mean = torch.var_mean(x, -1, correction=0, keepdim=True)
        u, r = x - mean, torch.sqrt(var + EPS)
    else:
        u, r = x, torch.sqrt(torch.einsum("thd,thd->th", x, x)[..., None] / D + EPS)
    if case["pass"] == "forward":
        return turn(u / r * w, 1)
    # u / r: the gradient of 1 / r is -u / (D r^3)
    dy = turn(s["dY"].double(), -1)
    du = dy * w / r - u * torch.einsum("thd,thd->th", dy * w, u)[..., None] / (D * r ** 3)
    if case["centred"]:
        du = du - du.mean(-1, keepdim=True)
    each = torch.einsum("thd,thd->hd", dy, u / r)
    return du, torch.stack([each[:Hq].sum(0), each[Hq:].sum(0)])


def _exact_values(codes, scales):
    """What codes and exponent bytes stand for: e4m3 has a sign, four bits of exponent (bias 7) and three of mantissa."""
    if scales is None:
        return codes.double()
    c = codes.view(torch.uint8).long()
    e, m = c >> 3 & 15, (c & 7).double()
    value = torch.where(e == 0, m * 2.0 ** -9, (8 + m) * torch.exp2(e.double() - 10))
    value = torch.where(c & 127 == 127, math.nan, value) * (1 - 2 * (c >> 7)).double()
    return value * torch.exp2(scales.double()[..., None] - 127)


def _exact_rounded(x):
    """Rows as the 8-bit cache holds them: of all numbers of the format times the row's power of two, the nearest, an even code
    where two are as near."""
    x = x.double()
    top = x.abs().amax(-1, keepdim=True)
    power = torch.ceil(torch.log2(top.clamp(min=2.0 ** -140) / 448))
    power = torch.where(448 * torch.exp2(power - 1) >= top, power - 1, power)  # (a logarithm that was rounded up or down)
    power = torch.where(448 * torch.exp2(power) < top, power + 1, power).clamp(LOWEST, HIGHEST)
    y = x / torch.exp2(power)
    numbers = torch.tensor([m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:-1],
                           dtype=torch.float64, device="cuda")
    above = torch.searchsorted(numbers, y.abs()).clamp(max=len(numbers) - 1)
    below = (above - 1).clamp(min=0)
    up, down = numbers[above] - y.abs(), y.abs() - numbers[below]
    code = torch.where((up < down) | ((up == down) & (above % 2 == 0)), above, below)
    return torch.copysign(numbers[code], y) * torch.exp2(power)


def _exact_cache(case, s):
    if case["pass"] == "write":
        return tuple(s[n].double() if case["format"] == "bf16" else _exact_rounded(s[n]) for n in ("K", "V"))
    outs = []
    for name in ("K", "V"):
        pages, scales = s[name + "_pages"], s[name + "_scales"]
        rows = []
        for b, n in enumerate(_lengths(case)[1]):
            entries = s["table"][b, :-(-n // case["page"])].long()
            codes = (pages.view(torch.uint8) if scales is not None else pages)[entries].flatten(0, 1)[:n]
            rows.append(_exact_values(codes, None if scales is None else scales[entries].flatten(0, 1)[:n]))
        outs.append(torch.cat(rows))
    return tuple(outs)


def _exact_paged(case, s):
    """One sequence and one key head at a time, over the pages that its table names."""
    new, tokens = _lengths(case)
    Hkv, group, page = case["Hkv"], case["Hq"] // case["Hkv"], case["page"]
    O = torch.zeros(s["Q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full((case["Hq"], sum(new)), -INFINITY, dtype=torch.float64, device="cuda")
    q0 = 0
    for b, (L, n) in enumerate(zip(new, tokens)):
        rq = slice(q0, q0 + L)
        q0 += L
        if L == 0:
            continue
        keys = torch.arange(n, device="cuda")
        position = torch.arange(n - L, n, device="cuda")[:, None]
        hidden = keys > position
        if case["window"]:
            hidden |= (keys <= position - case["window"]) & (keys >= case["sinks"])
        keys = keys[~hidden.all(0)]
        hidden = hidden[:, keys]
        entry, slot = s["table"][b, keys // page].long(), keys % page
        for h in range(Hkv):
            hq = slice(h * group, (h + 1) * group)
            k, v = (_exact_values((p.view(torch.uint8) if c is not None else p)[entry, slot, h].contiguous(), None if c is None else c[entry, slot, h])
                    for p, c in ((s["K_pages"], s["K_scales"]), (s["V_pages"], s["V_scales"])))
            q = s["Q"][rq, hq].double().transpose(0, 1).contiguous()
            z = torch.matmul(q, k.T.contiguous()) * s["scale"]
            z.masked_fill_(hidden, -INFINITY)
            lse[hq, rq] = torch.logsumexp(z, -1)
            O[rq, hq] = torch.matmul(torch.softmax(z, -1), v).transpose(0, 1)
    return O if case["pass"] == "decode" else (O, lse)


# ------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------------
def work(case):
    size = {"bf16": 2, "f32": 4}
    if case["kind"] == "head_norm":
        n, x, y = case["T"] * (case["Hq"] + case["Hk"]) * case["D"], size[case["x"]], size[case["y"]]
        small = 4 * case["T"] * case["axes"] + 2 * case["R"] + 8 * case["D"]
        if case["pass"] == "forward":
            return {"bytes": n * (x + y) + small, "flops": 10 * n}
        return {"bytes": n * (2 * x + y) + small + 8 * case["D"], "flops": 18 * n}
    new, tokens = _lengths(case)
    row = case["D"] + 1 if case["format"] == "e4m3" else 2 * case["D"]  # of one head of a token in the cache
    if case["kind"] == "cache":
        n = 2 * case["H"] * (sum(new) if case["pass"] == "write" else sum(tokens))
        if case["pass"] == "read":
            return {"bytes": n * (row + 2 * case["D"]), "flops": n * case["D"]}
        return {"bytes": n * (2 * row + 4 * case["D"]), "flops": 4 * n * case["D"]}  # read, kept, read back
    pairs = keys = 0
    for L, n in zip(new, tokens):
        window, sinks = case["window"] or n, case["sinks"] if case["window"] else 0
        seen = [min(p + 1, window) + max(0, min(sinks, p + 1 - window)) for p in range(n - L, n)]
        pairs += sum(seen)
        if L:
            first = max(0, n - L + 1 - window)
            keys += n - first + min(sinks, first)
    q = 2 * sum(new) * case["Hq"] * case["D"]
    return {"bytes": 2 * q + 2 * keys * case["Hkv"] * row + (4 * sum(new) * case["Hq"] if case["pass"] == "chunk" else 0),
            "flops": 4 * case["D"] * pairs * case["Hq"]}
