"""A pre-norm transformer block whose four linears carry N:M levels (Section 3, "Problem Formulation": qkv, proj, fc1 and fc2 of
a block, one level each), run end to end through the library: layer norm with the residual sum, the sparse linears, norms of queries and
keys with their rotary positions, attention; its training step; and single tokens, or chunks of them, against a cache of keys and values.

The residual stream travels beside the branch that was computed last, so that the sum of the two is part of the next norm:
a block takes (branch, stream) and returns the same pair, and `finish` adds the last branch.  All activations are bfloat16
[tokens, width], sequences packed one after another (offsets as nm_attention takes them).
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Dict, Optional, Sequence, Tuple, Union

from . import binding as nm
from .workloads import Level

LINEARS = ("qkv", "proj", "fc1", "fc2")


@dataclass
class Sequences:
    """Packed sequences: offsets (int32 [count + 1] on the device) and the longest length; positions of their tokens for the
    rotary turn (int32 or float32 [tokens, axes])."""
    offsets: object
    longest: int
    positions: object


class _Room:
    """What both caches know of the room they have: `room` tokens for each sequence, `lengths` on the device, `used` on the host."""

    def expect(self, new: int, offsets) -> None:
        """Up to `new` more tokens of each sequence (offsets: how many of each) are about to be kept: ValueError where a sequence has
        no room for its.  Waits for the device only where what the host knows of the lengths does not settle it."""
        import torch
        if self.used is not None and self.used + new <= self.room:
            self.used += new
        elif not (self.lengths.is_cuda and torch.cuda.is_current_stream_capturing()):  # (a capture computes nothing yet)
            used = int((self.lengths + offsets.diff()).max())
            if used > self.room:
                raise ValueError(f"a sequence of {used} tokens in a cache with room for {self.room} each")
            self.used = used


@dataclass
class Cache(_Room):
    """Keys and values of `count` sequences with room for `room` tokens each ([count * room, key heads, head size]), how many are
    in use (int32 [count]) and where each sequence begins (int32 [count + 1]).  used: what the host knows of the lengths, none is
    above it (None: nothing is known); a caller that raises `lengths` itself sets it.

    Tokens that do not fit are refused before anything is computed.  Where the host cannot know -- a replayed graph -- no row of
    another sequence is written: the lengths count on, and a sequence whose length is above `room` has lost its last tokens, and its
    outputs mean nothing from there on."""
    K: object
    V: object
    lengths: object
    offsets: object
    room: int
    used: Optional[int] = None

    @classmethod
    def empty(cls, count: int, room: int, heads: int, size: int, device="cuda") -> "Cache":
        import torch
        K, V = (torch.zeros((count * room, heads, size), dtype=torch.bfloat16, device=device) for _ in range(2))
        offsets = torch.arange(count + 1, dtype=torch.int32, device=device) * room
        return cls(K, V, torch.zeros(count, dtype=torch.int32, device=device), offsets, room, 0)


@dataclass
class PagedCache(_Room):
    """Keys and values of sequences in pages ([pages, page size, key heads, head size]), in bfloat16 or in 8 bits with the powers of two of
    their rows, as nm_cache_write has them.  Token j of sequence b is in page table[b, j // page size]; a program that hands out pages as
    sequences grow, or takes them back, writes `table` itself (an entry below 0: no page).  window, sinks: a token sees the last `window`
    tokens and the first `sinks` of its sequence (window 0: all of them), so pages in between can be taken back.

    Tokens that do not fit are refused as by `Cache`.  Where the host cannot know -- a replayed graph -- what falls outside the table is
    dropped and the lengths count on: tokens see those before them that were kept."""
    K: object
    V: object
    K_scales: object
    V_scales: object
    table: object
    lengths: object
    room: int
    used: Optional[int] = None
    window: int = 0
    sinks: int = 0

    @classmethod
    def empty(cls, count: int, room: int, heads: int, size: int, page: int = 64, eight_bits: bool = False, window: int = 0, sinks: int = 0,
              device="cuda") -> "PagedCache":
        """Every sequence with pages of its own for `room` tokens, the heads of a page one after another."""
        import torch
        each = -(-room // page)

        def pages(*shape, dtype):
            return torch.zeros((count * each, heads, page, *shape), dtype=dtype, device=device).transpose(1, 2)

        K, V = (pages(size, dtype=torch.float8_e4m3fn if eight_bits else torch.bfloat16) for _ in range(2))
        scales = [pages(dtype=torch.uint8) if eight_bits else None for _ in range(2)]
        table = torch.arange(count * each, dtype=torch.int32, device=device).view(count, each)
        return cls(K, V, *scales, table, torch.zeros(count, dtype=torch.int32, device=device), room, 0, window, sinks)

    def keep(self, k, v, offsets) -> None:
        """New tokens of each sequence (offsets) behind those that are there."""
        self.lengths += offsets.diff()
        nm.nm_cache_write(k, v, self.K, self.V, self.table, self.lengths, offsets, self.K_scales, self.V_scales)

    def read(self, offsets, tokens: int, first=None):
        """(k, v) in bfloat16 of the tokens from `first` on (int32 [count]; None: all), `tokens` rows in all."""
        return nm.nm_cache_read(self.K, self.V, self.table, self.lengths, offsets, tokens, first, self.K_scales, self.V_scales)

    def attend(self, q, offsets, new: int, longest: int):
        """Attention of the tokens that were kept last (offsets; at most `new` of each sequence)."""
        return nm.nm_attention_paged(q, self.K, self.V, self.table, self.lengths, offsets_q=offsets, window=self.window, sinks=self.sinks,
                                     K_scales=self.K_scales, V_scales=self.V_scales, max_q=new, max_k=longest)


class SparseBlock:
    """weights: dense bfloat16 {"qkv": [(heads + 2 key heads) * size, C], "proj": [C, heads * size], "fc1": [F, C], "fc2": [C, F]};
    levels: {name: (N, M)}; norms: (weight, bias) of both norms, float32 [C]; biases: {name: float32 [O]}, any of them missing;
    freqs, sections, interleaved: as nm_rotary takes them (freqs None: no rotary positions); head_norms: weights of the norms of queries and
    keys, float32 [2, head size] (None: they are not normed), which are layer norms where head_norms_centred, else by the root mean
    square."""

    def __init__(self, weights: Dict[str, object], levels: Dict[str, Level], norms: Sequence[Tuple[object, object]], heads: int,
                 key_heads: Optional[int] = None, biases: Optional[Dict[str, object]] = None, freqs=None, sections=None,
                 interleaved: bool = False, causal: bool = False, eps: float = 1e-6, head_norms=None, head_norms_centred: bool = False):
        self.heads, self.key_heads = heads, key_heads or heads
        self.size = weights["proj"].shape[1] // heads
        if weights["qkv"].shape[0] != (heads + 2 * self.key_heads) * self.size:
            raise ValueError("qkv must have (heads + 2 * key heads) * head size rows")
        self.levels, self.norms, self.biases = levels, norms, biases or {}
        self.freqs, self.sections, self.interleaved, self.causal, self.eps = freqs, sections, interleaved, causal, eps
        self.head_norms, self.head_norms_centred = head_norms, head_norms_centred
        self.update(weights)

    def update(self, weights: Dict[str, object]) -> None:
        """Take new dense weights: the mask of each level, the masked dense form and the packed one."""
        self.mask, self.masked, self.packed = {}, {}, {}
        for name in LINEARS:
            W, (N, M) = weights[name], self.levels[name]
            self.masked[name] = W.new_empty(W.shape)
            self.mask[name] = nm.nm_prune(W, N, M, W_masked=self.masked[name])
            self.packed[name] = nm.nm_pack(W, N, M)

    def _linear(self, name: str, x):
        N, M = self.levels[name]
        return nm.nm_linear_forward(*self.packed[name], x.shape[1], N, M, x, bias=self.biases.get(name), out_dtype=x.dtype)

    def _split(self, qkv):
        """(q and k, q, k, v) of the joint projection's rows, as views."""
        heads = qkv.unflatten(1, (-1, self.size))
        turned = self.heads + self.key_heads
        return heads[:, :turned], heads[:, :self.heads], heads[:, self.heads:turned], heads[:, turned:]

    def _turn(self, x, positions, inverse: bool = False) -> None:
        if self.freqs is not None:
            nm.nm_rotary(x, positions, self.freqs, self.sections, self.interleaved, inverse, out=x)

    def _head_norms(self, positions) -> dict:
        turn = dict(positions=positions, freqs=self.freqs, sections=self.sections) if self.freqs is not None else {}
        return dict(weight=self.head_norms, heads=self.heads, eps=self.eps, centred=self.head_norms_centred, interleaved=self.interleaved,
                    **turn)

    def _queries_and_keys(self, turned, positions, train: bool):
        """q and k, normed and turned: in place, but that a backward pass needs what was normed."""
        if self.head_norms is None:
            self._turn(turned, positions)
        else:
            turned = nm.nm_head_norm(turned, out=None if train else turned, **self._head_norms(positions))
        return turned[:, :self.heads], turned[:, self.heads:]

    def _mlp(self, branch, stream, train: bool):
        import torch
        n2 = nm.nm_layer_norm(branch, *self.norms[1], self.eps, residual=stream, train=train, out_dtype=branch.dtype)
        h = self._linear("fc1", n2[0])
        return n2, h, self._linear("fc2", torch.nn.functional.gelu(h))

    def forward(self, branch, stream, of: Sequences, cache: Union[Cache, PagedCache, None] = None, train: bool = False):
        """((branch, stream), what `backward` needs or None).  With an empty cache the keys and values of the sequences are kept in
        it as their first tokens; ValueError where one is longer than the cache's room.  (A cache in pages is read again: what it holds,
        and what its window shows, is what the next tokens will see.)"""
        paged = isinstance(cache, PagedCache)
        if paged and (train or not self.causal):
            raise ValueError("a cache in pages serves causal attention, and no backward pass")
        if cache is not None:
            cache.expect(of.longest, of.offsets)
        n1 = nm.nm_layer_norm(branch, *self.norms[0], self.eps, residual=stream, train=train, out_dtype=branch.dtype)
        qkv = self._linear("qkv", n1[0])
        turned, _, _, v = self._split(qkv)
        q, k = self._queries_and_keys(turned, of.positions, train)
        if paged:
            cache.keep(k, v, of.offsets)
            att = cache.attend(q, of.offsets, of.longest, of.longest if cache.used is None else cache.used)
        else:
            att = nm.nm_attention(q, k, v, self.causal, offsets_q=of.offsets, offsets_k=of.offsets, max_q=of.longest, max_k=of.longest,
                                  lse=train)
        o = att[0] if train else att
        if cache is not None and not paged:
            self._keep(cache, k, v, of.offsets)
        n2, h, out = self._mlp(self._linear("proj", o.flatten(1)), n1[1], train)
        return (out, n2[1]), ((n1, qkv, o, att[1], n2, h, of, q, k) if train else None)

    def _keep(self, cache: Cache, k, v, offsets) -> None:
        import torch
        rows = torch.arange(k.shape[0], device=k.device)
        seq = torch.searchsorted(offsets[1:-1], rows, right=True)
        # (what would go past a sequence's rows goes to the last of them)
        at = torch.minimum(rows + (cache.offsets[:-1] + cache.lengths - offsets[:-1])[seq], (cache.offsets[1:] - 1)[seq])
        cache.K[at], cache.V[at] = k, v
        cache.lengths += offsets.diff()

    def step(self, branch, stream, positions, offsets, cache: Union[Cache, PagedCache], longest: int, new: int = 1):
        """One or a few new tokens per sequence (offsets; at most `new` each) against the cache, which takes their keys and
        values; longest: tokens of the longest sequence, the new ones counted, as far as known.  ValueError, and nothing computed or
        kept, where a sequence has no room for its."""
        if isinstance(cache, PagedCache) and not self.causal:
            raise ValueError("a cache in pages serves causal attention")
        cache.expect(new, offsets)
        n1 = nm.nm_layer_norm(branch, *self.norms[0], self.eps, residual=stream, out_dtype=branch.dtype)
        turned, _, _, v = self._split(self._linear("qkv", n1[0]))
        q, k = self._queries_and_keys(turned, positions, False)
        if isinstance(cache, PagedCache):
            cache.keep(k, v, offsets)
            o = cache.attend(q, offsets, new, longest)
        else:
            self._keep(cache, k, v, offsets)
            o = nm.nm_attention(q, cache.K, cache.V, True, offsets_q=offsets, offsets_k=cache.offsets, lengths_k=cache.lengths, max_q=new,
                                max_k=longest)
        n2, _, out = self._mlp(self._linear("proj", o.flatten(1)), n1[1], False)
        return out, n2[1]

    def backward(self, d_branch, d_stream, saved):
        """((d_branch, d_stream) of the block's inputs, which are the same tensor, and the gradients by name: float32 masked weight
        gradients "qkv" .., bias gradients "qkv.bias" .., "norm1" and "norm2" as (weight, bias), and "head_norms" [2, head size])."""
        import torch
        n1, qkv, o, lse, n2, h, of, q, k = saved
        grads = {}

        def linear(name, dy, x):
            grads[name] = nm.nm_linear_backward_weight(dy, x, mask=self.mask[name])
            if name in self.biases:
                grads[name + ".bias"] = dy.sum(0, dtype=torch.float32)
            return nm.nm_linear_backward_input(self.masked[name], dy, out_dtype=dy.dtype)

        def norm(name, n, dy, d_sum):
            dx, dw, db = nm.nm_layer_norm_backward(dy, n[1], n[2], self.norms[0 if name == "norm1" else 1][0], dS=d_sum, out_dtype=dy.dtype)
            grads[name] = (dw, db)
            return dx

        dh = torch.ops.aten.gelu_backward(linear("fc2", d_branch, torch.nn.functional.gelu(h)), h)
        d_sum = norm("norm2", n2, linear("fc1", dh, n2[0]), d_stream)
        d_o = linear("proj", d_sum, o.flatten(1)).unflatten(1, (-1, self.size))
        raw, _, _, v = self._split(qkv)
        d_qkv = torch.empty_like(qkv)
        d_turned, dq, dk, dv = self._split(d_qkv)
        nm.nm_attention_backward(d_o, q, k, v, o, lse, self.causal, offsets_q=of.offsets, offsets_k=of.offsets, max_q=of.longest,
                                 max_k=of.longest, out=(dq, dk, dv))
        if self.head_norms is None:
            self._turn(d_turned, of.positions, inverse=True)
        else:
            grads["head_norms"] = nm.nm_head_norm_backward(d_turned, raw, out=d_turned, **self._head_norms(of.positions))[1]
        d_in = norm("norm1", n1, linear("qkv", d_qkv, n1[0]), d_sum)
        return (d_in, d_in), grads


def finish(branch, stream, norm, eps: float = 1e-6):
    """The last norm of a model: of the stream with the last branch added."""
    return nm.nm_layer_norm(branch, *norm, eps, residual=stream, out_dtype=branch.dtype)[0]
