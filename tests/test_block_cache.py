"""A block's cache of keys and values: a sequence keeps its tokens in its own rows, up to the last of them, and one more is refused."""
import pytest
import torch

from paper_2409_09708_amd.block import Cache, Sequences, SparseBlock, finish

BF16 = torch.bfloat16


def starts(counts, device="cpu"):
    return torch.tensor([0] + counts).cumsum(0).to(torch.int32).to(device)


def filled(lengths, room, heads=2, size=4):
    """A cache on the CPU whose row r holds the value r + 1 throughout."""
    cache = Cache.empty(len(lengths), room, heads, size, device="cpu")
    for t in (cache.K, cache.V):
        t.copy_((torch.arange(t.shape[0]) + 1)[:, None, None].expand_as(t))
    cache.lengths.copy_(torch.tensor(lengths))
    return cache


def tokens(n, value, heads=2, size=4):
    t = torch.arange(n, dtype=torch.float32)[:, None, None].expand(n, heads, size)
    return (value + t).to(BF16), (-value - t).to(BF16)


def keep(cache, counts, value=200):
    k, v = tokens(sum(counts), value)
    SparseBlock._keep(None, cache, k, v, starts(counts))
    return k, v


@pytest.mark.parametrize("lengths,counts", [([3, 0, 7], [2, 5, 1]), ([7, 8, 0], [1, 0, 8]), ([0, 0, 0], [8, 8, 8]), ([2], [6])])
def test_tokens_go_behind_those_that_are_there(lengths, counts):
    cache = filled(lengths, 8)
    before = cache.K.clone(), cache.V.clone()
    k, v = keep(cache, counts)
    want_k, want_v, at = *before, 0
    for b, (n, new) in enumerate(zip(lengths, counts)):
        want_k[b * 8 + n:b * 8 + n + new], want_v[b * 8 + n:b * 8 + n + new] = k[at:at + new], v[at:at + new]
        at += new
    assert torch.equal(cache.K, want_k) and torch.equal(cache.V, want_v)
    assert cache.lengths.tolist() == [n + new for n, new in zip(lengths, counts)]


@pytest.mark.parametrize("lengths,counts", [([8, 3, 8], [1, 1, 1]), ([7, 0, 6], [4, 2, 5]), ([20, 3, 30], [1, 0, 2])])
def test_a_full_sequence_leaves_its_neighbours_alone(lengths, counts):
    """Lengths that went past the room without the host's knowledge: no row of another sequence is written, nor one past the cache."""
    cache = filled(lengths, 8)
    before = cache.K.clone(), cache.V.clone()
    k, v = keep(cache, counts)
    at = sum(counts[:1])
    for t, old, new in ((cache.K, before[0], k), (cache.V, before[1], v)):
        assert torch.equal(t[:min(lengths[0], 7)], old[:min(lengths[0], 7)])
        assert torch.equal(t[8:8 + lengths[1]], old[8:8 + lengths[1]])
        assert torch.equal(t[8 + lengths[1]:8 + lengths[1] + counts[1]], new[at:at + counts[1]])
        assert torch.equal(t[8 + lengths[1] + counts[1]:16], old[8 + lengths[1] + counts[1]:16])
        assert torch.equal(t[16:16 + min(lengths[2], 7)], old[16:16 + min(lengths[2], 7)])
    assert cache.lengths.tolist() == [n + new for n, new in zip(lengths, counts)]  # (above the room: it shows)


def test_more_than_the_room_is_refused_before_anything_is_kept():
    cache = Cache.empty(3, 8, 2, 4, device="cpu")
    for counts in ([5, 1, 0], [2, 1, 3], [1, 6, 1]):
        cache.expect(max(counts), starts(counts))
        keep(cache, counts)
    assert cache.lengths.tolist() == [8, 8, 4]
    before = cache.K.clone()
    for counts in ([1, 0, 0], [0, 1, 4], [0, 0, 5]):
        with pytest.raises(ValueError, match="room for 8"):
            cache.expect(max(counts), starts(counts))
    assert torch.equal(cache.K, before) and cache.lengths.tolist() == [8, 8, 4]
    cache.expect(4, starts([0, 0, 4]))  # (the others' tokens do not count)
    keep(cache, [0, 0, 4])
    cache.lengths.zero_()               # a caller that starts over
    cache.expect(8, starts([8, 1, 2]))


def test_lengths_that_the_host_does_not_know():
    K, V = torch.zeros(16, 2, 4, dtype=BF16), torch.zeros(16, 2, 4, dtype=BF16)
    cache = Cache(K, V, torch.tensor([8, 2], dtype=torch.int32), torch.tensor([0, 8, 16], dtype=torch.int32), 8)
    with pytest.raises(ValueError, match="room for 8"):
        cache.expect(1, starts([1, 1]))
    cache.expect(1, starts([0, 1]))
    with pytest.raises(ValueError, match="room for 8"):
        Cache.empty(1, 8, 2, 4, device="cpu").expect(9, starts([9]))


@pytest.mark.gpu
def test_steps_up_to_the_last_row_and_one_past_it():
    from test_gpu_block import make, near
    block, normal = make(256, 8, 2, 512, True, 5)
    lens, room = [12, 3, 9], 12
    T = sum(lens)
    branch, stream = normal(T, 256).to(BF16), normal(T, 256).to(BF16)
    positions = torch.cat([torch.arange(n) for n in lens])[:, None].repeat(1, 2).to(torch.int32).cuda()
    want = finish(*block.forward(branch, stream, Sequences(starts(lens, "cuda"), 12, positions))[0], block.norms[0])
    last = starts(lens, "cuda")[1:].long() - 1

    cache = Cache.empty(3, room, 2, 32)
    rows = torch.ones(T, dtype=torch.bool, device="cuda")
    rows[last] = False
    before = [n - 1 for n in lens]
    block.forward(branch[rows], stream[rows], Sequences(starts(before, "cuda"), 11, positions[rows].contiguous()), cache=cache)
    each = starts([1, 1, 1], "cuda")

    def step():
        return finish(*block.step(branch[last], stream[last], positions[last].contiguous(), each, cache, room), block.norms[0])

    near(step(), want[last].double(), 10 ** 0.5 * 2.0 ** -8, "the last row")
    assert cache.lengths.tolist() == lens
    kept = cache.K.clone(), cache.V.clone()
    with pytest.raises(ValueError, match="room for 12"):
        step()
    for of in (starts([1, 0, 0], "cuda"), starts([13, 0, 0], "cuda")):
        n = int(of[1])
        with pytest.raises(ValueError, match="room for 12"):
            block.forward(branch[:n], stream[:n], Sequences(of, n, positions[:n].contiguous()), cache=cache)
    assert cache.lengths.tolist() == lens and torch.equal(cache.K, kept[0]) and torch.equal(cache.V, kept[1])
    cache.used = 0  # (as a replayed graph would go on: the host does not count along)
    step()
    for t, old in zip((cache.K, cache.V), kept):
        assert torch.equal(t[:11], old[:11]) and torch.equal(t[12:15], old[12:15]) and torch.equal(t[24:33], old[24:33])
    assert cache.lengths.tolist() == [13, 4, 10]


@pytest.mark.gpu
def test_one_sequence_on_the_device():
    cache = Cache.empty(1, 6, 2, 4)
    k, v = (t.cuda() for t in tokens(4, 10))
    cache.expect(4, starts([4], "cuda"))
    SparseBlock._keep(None, cache, k, v, starts([4], "cuda"))
    assert torch.equal(cache.K[:4], k) and torch.equal(cache.V[:4], v) and cache.lengths.tolist() == [4]
