"""A block with norms of queries and keys, and its tokens in a cache in pages: values and gradients against torch's automatic
differentiation in 64 bits, chunks and single tokens against a whole prompt."""
import pytest
import torch

import paper_2409_09708_amd as nm
from pages_reference import rounded
from paper_2409_09708_amd.block import Cache, PagedCache, Sequences, SparseBlock, finish
from test_gpu_block import BF16, LEVELS, make, near

pytestmark = pytest.mark.gpu
# every activation is rounded to bfloat16 (2^-8 at most) on a path of about a dozen of them; the gradients' path is twice as long
FORWARD, BACKWARD = 12 ** 0.5 * 2.0 ** -8, 24 ** 0.5 * 2.0 ** -8


def normed(C, heads, key_heads, F, seed, centred=False):
    block, normal = make(C, heads, key_heads, F, True, seed)
    block.head_norms, block.head_norms_centred = 1 + normal(2, block.size, scale=0.2), centred
    return block, normal


def definition(block, leaves, branch, stream, lens, positions, window=0, sinks=0):
    W, b, norms, w = leaves
    size, H, Hk = block.size, block.heads, block.key_heads

    def norm(x, p):
        return torch.nn.functional.layer_norm(x, x.shape[-1:], p[0], p[1], block.eps)

    s1 = branch + stream
    qkv = (norm(s1, norms[0]) @ W["qkv"].T + b["qkv"]).unflatten(1, (-1, size))
    qk = qkv[:, :H + Hk]
    if w is not None:
        if block.head_norms_centred:
            qk = qk - qk.mean(-1, keepdim=True)
        qk = qk * (qk.square().mean(-1, keepdim=True) + block.eps).rsqrt()
        qk = torch.cat([qk[:, :H] * w[0], qk[:, H:] * w[1]], 1)
    pairs = size // 2
    axis = [a for a, n in enumerate(block.sections) for _ in range(n)]
    angle = (positions[:, axis].double() * block.freqs.double())[:, None]
    u, v = qk[..., :pairs], qk[..., pairs:]
    turned = torch.cat([u * angle.cos() - v * angle.sin(), v * angle.cos() + u * angle.sin()], -1)
    outs, at = [], 0
    for n in lens:
        q, k = turned[at:at + n, :H], turned[at:at + n, H:].repeat_interleave(H // Hk, 1)
        val = qkv[at:at + n, H + Hk:].repeat_interleave(H // Hk, 1)
        z = (q.transpose(0, 1) @ k.permute(1, 2, 0)) * size ** -0.5
        j = torch.arange(n, device="cuda")
        seen = j <= j[:, None]
        if window:
            seen = seen & ((j > j[:, None] - window) | (j < sinks))
        outs.append((z.masked_fill(~seen, -float("inf")).softmax(-1) @ val.transpose(0, 1)).transpose(0, 1).flatten(1))
        at += n
    s2 = torch.cat(outs) @ W["proj"].T + b["proj"] + s1
    h = norm(s2, norms[1]) @ W["fc1"].T + b["fc1"]
    return torch.nn.functional.gelu(h) @ W["fc2"].T + b["fc2"], s2


def constants(block):
    w = None if block.head_norms is None else block.head_norms.double()
    return ({n: t.double() for n, t in block.masked.items()}, {n: t.double() for n, t in block.biases.items()},
            [tuple(p.double() for p in n) for n in block.norms], w)


def starts(lens):
    return torch.tensor([0] + list(lens)).cumsum(0).to(torch.int32).cuda()


@pytest.mark.parametrize("centred", [False, True])
def test_training_step(centred):
    block, normal = normed(256, 8, 2, 320, 1, centred)
    lens = [50, 1, 0, 77, 130]
    T = sum(lens)
    positions = torch.randint(0, 20, (T, 2), device="cuda", dtype=torch.int32)
    branch, stream, d_branch, d_stream = (normal(T, 256).to(BF16) for _ in range(4))
    of = Sequences(starts(lens), max(lens), positions)
    (out, total), saved = block.forward(branch, stream, of, train=True)
    plain, _ = block.forward(branch, stream, of)
    assert torch.equal(plain[0], out) and torch.equal(plain[1], total)
    (dx, _), grads = block.backward(d_branch, d_stream, saved)

    W, b, norms, w = constants(block)
    leaves = [t.requires_grad_() for t in [*W.values(), *b.values(), *(p for n in norms for p in n), w]]
    x, s = branch.double().requires_grad_(), stream.double()
    want = definition(block, (W, b, norms, w), x, s, lens, positions)
    for got, v, name in zip((out, total), want, ("branch", "stream")):
        near(got, v.detach(), FORWARD, name)
    torch.autograd.backward(want, (d_branch.double(), d_stream.double()))
    assert all(t.grad is not None for t in leaves)
    near(dx, x.grad, BACKWARD, "dx")
    near(grads["head_norms"], w.grad, BACKWARD, "head_norms")
    for n in W:
        kept = block.masked[n] != 0
        near(grads[n] * kept, W[n].grad * kept, BACKWARD, n)


class Rounded(PagedCache):
    """A cache of bfloat16 that keeps what one of 8 bits would."""

    def keep(self, k, v, offsets):
        super().keep(*(rounded(t)[0].to(BF16) for t in (k, v)), offsets)


def run_in_pieces(block, cache, branch, stream, positions, lens, pieces):
    """Sequences a chunk at a time, each from its own place on; rows as in one pass."""
    start = starts(lens).tolist()
    out = torch.empty_like(branch)
    done = [0] * len(lens)
    for counts in pieces:
        rows = torch.cat([torch.arange(start[b] + done[b], start[b] + done[b] + n) for b, n in enumerate(counts)]).cuda()
        done = [d + n for d, n in zip(done, counts)]
        at = (branch[rows], stream[rows], positions[rows].contiguous(), starts(counts), cache)
        out[rows] = finish(*block.step(*at, max(done), max(counts)), block.norms[0])
    assert done == list(lens) and cache.lengths.tolist() == list(lens)
    return out


LENS = [90, 7, 140]
PIECES = [[64, 7, 0], [20, 0, 120], [1, 0, 1], [4, 0, 4], [1, 0, 15]]


@pytest.mark.parametrize("window,sinks", [(0, 0), (30, 4)])
@pytest.mark.parametrize("page", [16, 64])
def test_chunks_and_single_tokens_give_what_the_prompt_gives(page, window, sinks):
    block, normal = normed(256, 8, 2, 512, 2)
    T = sum(LENS)
    branch, stream = normal(T, 256).to(BF16), normal(T, 256).to(BF16)
    positions = torch.cat([torch.arange(n) for n in LENS])[:, None].repeat(1, 2).to(torch.int32).cuda()
    want = definition(block, constants(block), branch.double(), stream.double(), LENS, positions, window, sinks)
    norm = block.norms[0]
    want = torch.nn.functional.layer_norm(want[0] + want[1], (256,), norm[0].double(), norm[1].double(), block.eps)

    cache = PagedCache.empty(3, 200, 2, 32, page, window=window, sinks=sinks)
    near(run_in_pieces(block, cache, branch, stream, positions, LENS, PIECES), want, FORWARD, "pieces")
    whole = PagedCache.empty(3, 200, 2, 32, page, window=window, sinks=sinks)
    got, _ = block.forward(branch, stream, Sequences(starts(LENS), max(LENS), positions), cache=whole)
    near(finish(*got, norm), want, FORWARD, "prompt")
    for ours, other in zip(cache.read(starts(LENS), T), whole.read(starts(LENS), T)):
        near(ours, other.double(), FORWARD, "keys and values")

    eight = PagedCache.empty(3, 200, 2, 32, page, eight_bits=True, window=window, sinks=sinks)
    same = Rounded.empty(3, 200, 2, 32, page, window=window, sinks=sinks)
    a = run_in_pieces(block, eight, branch, stream, positions, LENS, PIECES)
    b = run_in_pieces(block, same, branch, stream, positions, LENS, PIECES)
    near(a, b.double(), FORWARD, "8 bits")
    for x, y in zip(eight.read(starts(LENS), T), same.read(starts(LENS), T)):
        near(x, y.double(), 2.0 ** -8, "what is kept")


def test_both_caches_give_the_same():
    block, normal = make(256, 8, 2, 512, True, 3)
    T = sum(LENS)
    branch, stream = normal(T, 256).to(BF16), normal(T, 256).to(BF16)
    positions = torch.cat([torch.arange(n) for n in LENS])[:, None].repeat(1, 2).to(torch.int32).cuda()
    a = run_in_pieces(block, Cache.empty(3, 200, 2, 32), branch, stream, positions, LENS, PIECES)
    b = run_in_pieces(block, PagedCache.empty(3, 200, 2, 32), branch, stream, positions, LENS, PIECES)
    near(a, b.double(), FORWARD, "caches")


def test_pages_handed_out_as_sequences_grow():
    """A table with pages in any order, given when they are needed and taken back when the window has left them."""
    block, normal = normed(256, 8, 2, 512, 4)
    page, window, sinks, n = 16, 24, 3, 100
    branch, stream = normal(n, 256).to(BF16), normal(n, 256).to(BF16)
    positions = torch.arange(n)[:, None].repeat(1, 2).to(torch.int32).cuda()
    plain = PagedCache.empty(1, n, 2, 32, page, eight_bits=True, window=window, sinks=sinks)
    few = PagedCache.empty(1, n, 2, 32, page, eight_bits=True, window=window, sinks=sinks)
    few.table.fill_(-1)
    free, held = [4, 0, 3, 1], {}  # (four pages for seven)
    one = starts([1])
    for t in range(n):
        if t % page == 0:
            for i in [i for i in held if i * page >= sinks and (i + 1) * page <= t - window + 1]:
                free.append(held.pop(i))
                few.table[0, i] = -1
            held[t // page] = free.pop(0)
            few.table[0, t // page] = held[t // page]
        at = (branch[t:t + 1], stream[t:t + 1], positions[t:t + 1].contiguous(), one)
        for x, y in zip(block.step(*at, few, t + 1), block.step(*at, plain, t + 1)):
            assert torch.equal(x, y), t


def test_refusals():
    block, normal = normed(256, 8, 2, 320, 5)
    x = normal(20, 256).to(BF16)
    positions = torch.zeros(20, 2, dtype=torch.int32, device="cuda")
    of = Sequences(starts([20]), 20, positions)
    cache = PagedCache.empty(1, 19, 2, 32, 16)
    with pytest.raises(ValueError, match="room for 19"):
        block.forward(x, x, of, cache=cache)
    assert cache.lengths.tolist() == [0]
    with pytest.raises(ValueError, match="no backward pass"):
        block.forward(x, x, of, cache=PagedCache.empty(1, 30, 2, 32), train=True)
    block.causal = False
    for call in (lambda: block.forward(x, x, of, cache=PagedCache.empty(1, 30, 2, 32)),
                 lambda: block.step(x[:1], x[:1], positions[:1], starts([1]), PagedCache.empty(1, 30, 2, 32), 1)):
        with pytest.raises(ValueError, match="causal"):
            call()


def test_a_step_captured_and_replayed():
    block, normal = normed(256, 8, 2, 512, 6)
    cache, eager = (PagedCache.empty(2, 700, 2, 32, 16, eight_bits=True) for _ in range(2))
    prompt = normal(650, 256).to(BF16)
    at = torch.arange(650, device="cuda")[:, None].repeat(1, 2).to(torch.int32)
    for c in (cache, eager):
        block.forward(prompt, prompt, Sequences(starts([600, 50]), 600, at), cache=c)
    x, s = normal(2, 256).to(BF16), normal(2, 256).to(BF16)
    positions, each = torch.zeros(2, 2, dtype=torch.int32, device="cuda"), starts([1, 1])
    spare = PagedCache.empty(2, 700, 2, 32, 16, eight_bits=True)
    block.step(x, s, positions, each, spare, 700)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = block.step(x, s, positions, each, cache, 700)
    for t in range(4):
        x.copy_(normal(2, 256))
        positions.fill_(600 + t)
        want = block.step(x, s, positions, each, eager, 700)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, want)), t
        assert torch.equal(cache.lengths, eager.lengths)


def test_head_norms_without_positions_and_with_a_cache_of_rows():
    block, normal = normed(256, 8, 2, 512, 7, centred=True)
    T = sum(LENS)
    branch, stream = normal(T, 256).to(BF16), normal(T, 256).to(BF16)
    positions = torch.zeros(T, 2, dtype=torch.int32, device="cuda")
    want = definition(block, constants(block), branch.double(), stream.double(), LENS, positions)  # (no angle: no turn)
    norm = block.norms[0]
    want = torch.nn.functional.layer_norm(want[0] + want[1], (256,), norm[0].double(), norm[1].double(), block.eps)
    block.freqs = None
    of = Sequences(starts(LENS), max(LENS), positions)
    out, saved = block.forward(branch, stream, of, train=True)
    near(finish(*out, norm), want, FORWARD, "prompt")
    for cache in (Cache, PagedCache):
        near(run_in_pieces(block, cache.empty(3, 200, 2, 32), branch, stream, positions, LENS, PIECES), want, FORWARD, cache.__name__)
    d_branch, d_stream = normal(T, 256).to(BF16), normal(T, 256).to(BF16)
    (dx, _), grads = block.backward(d_branch, d_stream, saved)
    W, b, norms, w = constants(block)
    x, w = branch.double().requires_grad_(), w.requires_grad_()
    block.freqs = torch.zeros(block.size // 2, device="cuda")
    torch.autograd.backward(definition(block, (W, b, norms, w), x, stream.double(), LENS, positions), (d_branch.double(), d_stream.double()))
    near(dx, x.grad, BACKWARD, "dx")
    near(grads["head_norms"], w.grad, BACKWARD, "head_norms")
