"""Scratch memory of attention over a cache in pages: what is dealt to blocks leaves two parts a block, however many sequences and heads there are."""
import pytest

from paper_2409_09708_amd import binding


@pytest.mark.parametrize("head_size", [32, 64, 128])
def test_few_queries(head_size):
    size = binding.load_library().nm_attention_paged_workspace_bytes
    one = size(1, 1, 32, 8, head_size, 1)
    assert 0 < one <= 1024 * 16 * (head_size + 2) * 4 + 512 * 32 + 512  # (sums, maximum and total of 16 columns; what blocks share; rounding)
    for sequences, heads_q, heads_kv, new in ((1, 8, 8, 1), (24, 32, 8, 1), (100, 64, 64, 4), (512, 32, 32, 1), (512, 64, 64, 1), (512, 64, 8, 4)):
        assert size(sequences * new, sequences, heads_q, heads_kv, head_size, new) == one
    assert size(513, 513, 32, 8, head_size, 1) == 0
