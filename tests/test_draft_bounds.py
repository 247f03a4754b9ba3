"""What the binding takes for the bound on a tree's queries (no GPU)."""
import pytest
import torch

import paper_2503_01483_amd as kt


def call(n, words, **kw):
    """A tree call of n rows on the CPU: it ends at the check that comes first."""
    cache = kt.KVCache(4, 64, 2, 64, kt.KT_KV_U4, device="cpu")
    q, lens, pages = torch.zeros(n, 4, 64, dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32), torch.zeros(1, 3, dtype=torch.int32)
    kt.kt_tree_attention(q, cache, pages, lens, torch.zeros(n, words, dtype=torch.int64), q_starts=torch.tensor([0, n], dtype=torch.int32), **kw)


@pytest.mark.parametrize("n,words", [(65, 1), (100, 1), (129, 2)])
def test_more_rows_than_bits_need_a_bound(n, words):
    """One sequence could have all rows, and its drafts behind the last bit would be hidden from every row, themselves included."""
    with pytest.raises(ValueError, match="max_q"):
        call(n, words)


@pytest.mark.parametrize("n,words,kw", [(64, 1, {}), (128, 2, {}), (100, 1, dict(max_q=64)), (65, 1, dict(max_q=3))])
def test_with_a_bound_or_enough_bits_the_call_goes_on(n, words, kw):
    with pytest.raises(ValueError, match="current device"):
        call(n, words, **kw)
