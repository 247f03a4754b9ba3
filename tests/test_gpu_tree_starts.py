"""q_starts of trees that descend, which they may not: calls stay within their memory."""
import numpy as np
import pytest
import torch

import paper_2503_01483_amd as kt
from draft_util import FORMATS, NAMES, ints, random_tree, tree_check, words_of
from serving_util import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("counts", [[4, 3], [40, 30]], ids=["few", "many"])
def test_zeros_behind_the_last_sequence(fmt, counts):
    """Rows of a batch that is not full, left at 0: sequences without queries."""
    b = Batch(fmt, 128, 2, 4, [100, 90, 50, 70], counts + [0, 0], seed=1)
    masks = [random_tree(c, np.random.default_rng(2)) for c in b.counts]
    lse = torch.full((b.n, b.hq), 7.0, device="cuda")
    starts = ints(b.starts[:3] + [0, 0])
    out = kt.kt_tree_attention(b.q.cuda(), b.cache, b.pages, ints(b.lens), words_of(masks, b.n, 1), q_starts=starts, max_q=max(counts), lse=lse)
    tree_check(b, out, lse, masks)


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
def test_sequences_that_share_queries_beyond_what_a_list_holds(fmt):
    """2048 sequences that all have the same 8192 queries, over 65536 tokens each: more key tiles than 32 bits count, over all heads.  Nothing is computed."""
    n, heads, group, hd, n_seq, ldp = 8192, 8, 8, 64, 4096, 1024
    cache = kt.KVCache(4, 64, heads, hd, fmt)
    cache.data.zero_()
    q = torch.zeros(n, heads * group, hd, dtype=torch.bfloat16, device="cuda")
    starts = torch.zeros(n_seq + 1, dtype=torch.int32, device="cuda")
    starts[1::2] = n
    pages, lens = torch.zeros(n_seq, ldp, dtype=torch.int32, device="cuda"), torch.full((n_seq,), 64 * ldp, dtype=torch.int32, device="cuda")
    rows = {kt.KT_KV_BF16: 256}.get(fmt, 128)
    assert n_seq // 2 * (n * group // rows) * (4 + ldp) * heads > 2 ** 32
    out, lse = torch.full_like(q, 3.0), torch.full((n, heads * group), 7.0, device="cuda")
    kt.kt_tree_attention(q, cache, pages, lens, torch.zeros(n, n // 64, dtype=torch.int64, device="cuda"), q_starts=starts, max_q=n, out=out, lse=lse)
    torch.cuda.synchronize()
    assert bool((out == 3).all()) and bool((lse == 7).all())
