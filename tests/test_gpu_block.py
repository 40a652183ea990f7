"""A whole block of sparse linears, norms, rotary positions and attention: its values and gradients against torch's automatic
differentiation in 64 bits on the masked weights, and single tokens against a whole prompt."""
import pytest
import torch

import paper_2409_09708_amd as nm
from paper_2409_09708_amd.block import Cache, Sequences, SparseBlock, finish

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
LEVELS = {"qkv": (2, 4), "proj": (2, 8), "fc1": (1, 4), "fc2": (4, 8)}


def make(C, heads, key_heads, F, causal, seed):
    g = torch.Generator("cuda")
    g.manual_seed(seed)

    def normal(*shape, scale=1.0):
        return torch.randn(shape, generator=g, device="cuda") * scale

    size = C // heads
    weights = {n: normal(o, k, scale=2 * k ** -0.5).to(BF16)
               for n, o, k in (("qkv", (heads + 2 * key_heads) * size, C), ("proj", C, C), ("fc1", F, C), ("fc2", C, F))}
    biases = {n: normal(w.shape[0], scale=0.1) for n, w in weights.items()}
    norms = [(1 + normal(C, scale=0.1), normal(C, scale=0.1)) for _ in range(2)]
    freqs = 100.0 ** (-torch.arange(size // 2, device="cuda") / (size // 2))
    return SparseBlock(weights, LEVELS, norms, heads, key_heads, biases, freqs, (size // 4, size // 4), causal=causal), normal


def definition(block, leaves, branch, stream, lens, positions):
    """The block in 64 bits on masked weights."""
    W, b, norms = leaves
    size, H, Hk = block.size, block.heads, block.key_heads

    def norm(x, p):
        return torch.nn.functional.layer_norm(x, x.shape[-1:], p[0], p[1], block.eps)

    s1 = branch + stream
    qkv = (norm(s1, norms[0]) @ W["qkv"].T + b["qkv"]).unflatten(1, (-1, size))
    pairs = size // 2
    axis = [a for a, n in enumerate(block.sections) for _ in range(n)]
    angle = (positions[:, axis].float() * block.freqs).double()[:, None]
    u, v = qkv[:, :H + Hk, :pairs], qkv[:, :H + Hk, pairs:]
    turned = torch.cat([u * angle.cos() - v * angle.sin(), v * angle.cos() + u * angle.sin()], -1)
    outs, at = [], 0
    for n in lens:
        q, k = turned[at:at + n, :H], turned[at:at + n, H:].repeat_interleave(H // Hk, 1)
        val = qkv[at:at + n, H + Hk:].repeat_interleave(H // Hk, 1)
        z = (q.transpose(0, 1) @ k.permute(1, 2, 0)) * size ** -0.5
        if block.causal:
            z = z.masked_fill(torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1), -float("inf"))
        outs.append((z.softmax(-1) @ val.transpose(0, 1)).transpose(0, 1).flatten(1))
        at += n
    s2 = torch.cat(outs) @ W["proj"].T + b["proj"] + s1
    h = norm(s2, norms[1]) @ W["fc1"].T + b["fc1"]
    return torch.nn.functional.gelu(h) @ W["fc2"].T + b["fc2"], s2


def near(got, want, by, what):
    err = float((got.double() - want).norm() / want.norm())
    assert err <= by, (what, err)


@pytest.mark.parametrize("C,heads,key_heads,F,causal", [(256, 4, 4, 512, False), (256, 8, 2, 320, True)])
def test_training_step(C, heads, key_heads, F, causal):
    block, normal = make(C, heads, key_heads, F, causal, 1)
    lens = [50, 1, 0, 77, 130]
    T = sum(lens)
    offsets = torch.tensor([0] + lens).cumsum(0).to(torch.int32).cuda()
    positions = torch.randint(0, 20, (T, 2), device="cuda", dtype=torch.int32)
    branch, stream, d_branch, d_stream = (normal(T, C).to(BF16) for _ in range(4))
    of = Sequences(offsets, max(lens), positions)
    (out, total), saved = block.forward(branch, stream, of, train=True)
    plain, _ = block.forward(branch, stream, of)
    assert torch.equal(plain[0], out) and torch.equal(plain[1], total)
    (dx, _), grads = block.backward(d_branch, d_stream, saved)

    W = {n: w.double().requires_grad_() for n, w in block.masked.items()}
    b = {n: v.double().requires_grad_() for n, v in block.biases.items()}
    norms = [tuple(p.double().requires_grad_() for p in n) for n in block.norms]
    x, s = branch.double().requires_grad_(), stream.double()
    want = definition(block, (W, b, norms), x, s, lens, positions)
    # every activation is rounded to bfloat16 (2^-8 at most, 2^-9.6 root mean square) on a path of about ten of them; the gradients'
    # path is twice as long
    for got, v, name in zip((out, total), want, ("branch", "stream")):
        near(got, v.detach(), 10 ** 0.5 * 2.0 ** -8, name)
    torch.autograd.backward(want, (d_branch.double(), d_stream.double()))
    by = 20 ** 0.5 * 2.0 ** -8
    near(dx, x.grad, by, "dx")
    for n in W:
        kept = block.masked[n] != 0
        near(grads[n] * kept, W[n].grad * kept, by, n)
        near(grads[n + ".bias"], b[n].grad, by, n + ".bias")
    for i, n in enumerate(("norm1", "norm2")):
        for got, p in zip(grads[n], norms[i]):
            near(got, p.grad, by, n)


def test_single_tokens_give_what_the_prompt_gives():
    block, normal = make(256, 8, 2, 512, True, 2)
    lens, more = [40, 7, 129], 5
    full = [n + more for n in lens]
    T = sum(full)
    branch, stream = normal(T, 256).to(BF16), normal(T, 256).to(BF16)
    positions = torch.cat([torch.arange(n) for n in full])[:, None].repeat(1, 2).to(torch.int32).cuda()
    start = torch.tensor([0] + full).cumsum(0).tolist()
    offsets = torch.tensor(start, dtype=torch.int32).cuda()
    want, _ = block.forward(branch, stream, Sequences(offsets, max(full), positions))
    want = finish(*want, block.norms[0])

    rows = torch.cat([torch.arange(start[i], start[i] + n) for i, n in enumerate(lens)]).cuda()
    cache = Cache.empty(3, 200, 2, 32)
    prompt = torch.tensor([0] + lens).cumsum(0).to(torch.int32).cuda()
    got, _ = block.forward(branch[rows], stream[rows], Sequences(prompt, max(lens), positions[rows].contiguous()), cache=cache)
    near(finish(*got, block.norms[0]), want[rows].double(), 10 ** 0.5 * 2.0 ** -8, "prompt")
    each = torch.arange(4, dtype=torch.int32, device="cuda")
    for t in range(more):
        rows = torch.tensor([start[i] + n + t for i, n in enumerate(lens)]).cuda()
        got = block.step(branch[rows], stream[rows], positions[rows].contiguous(), each, cache, max(lens) + t + 1)
        near(finish(*got, block.norms[0]), want[rows].double(), 10 ** 0.5 * 2.0 ** -8, t)
    assert cache.lengths.tolist() == full
