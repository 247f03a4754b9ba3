"""As many sequences as a call takes, through the kernels of many rows, whose lists lie beside the tiles in LDS; weights that add up in far pages."""
import numpy as np
import pytest
import torch

import paper_2503_01483_amd as kt
from draft_util import FORMATS, NAMES, ints, words_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("hd", [128, 256])
@pytest.mark.parametrize("max_q", [40, 70])
def test_4096_sequences(fmt, hd, max_q):
    """A bound of more rows than the kernels of few take (trees over bf16: up to 128 and more), for sequences of none to three queries over up to 70 tokens, one of
    `max_q`: chains as kt_paged_attention computes them, weights that add up to the rows."""
    n_seq, group = 4096, 2
    g = torch.Generator().manual_seed(hd + max_q)
    lens = torch.randint(0, 71, (n_seq,), generator=g)
    counts = torch.minimum(lens, torch.randint(0, 4, (n_seq,), generator=g))
    lens[100], counts[100] = 70, max_q
    starts = torch.cat([torch.zeros(1, dtype=torch.long), counts.cumsum(0)])
    n = int(starts[-1])
    pages = torch.randperm(2 * n_seq, generator=g).reshape(n_seq, 2)
    cache = kt.KVCache(2 * n_seq, 64, 1, hd, fmt)
    seq = torch.repeat_interleave(torch.arange(n_seq), lens)
    t = torch.arange(len(seq)) - torch.repeat_interleave(torch.cumsum(lens, 0) - lens, lens)
    slots = (pages[seq, t // 64] * 64 + t % 64).cuda()
    k, v = (torch.randn(len(seq), 1, hd, generator=g).cuda() for _ in range(2))
    kt.kt_kv_append(cache, k, v, slots)
    q = torch.randn(n, group, hd, generator=g).to(torch.bfloat16).cuda()
    lse, want_lse = torch.full((n, group), 7.0, device="cuda"), torch.full((n, group), 9.0, device="cuda")
    more = dict(q_starts=ints(starts), max_q=max_q)
    masks = [np.tril(np.ones((c, c), dtype=bool)) for c in counts.tolist()]
    out = kt.kt_tree_attention(q, cache, ints(pages), ints(lens), words_of(masks, n, 2), lse=lse, **more)
    want = kt.kt_paged_attention(q, cache, ints(pages), ints(lens), lse=want_lse, **more)
    # both round p and the result to bf16 (2^-8 of |v| at most each, of p in fp16 and the values' 1.5 x 2^-11 less); values are within 5.5 of 0
    assert bool(((out.float() - want.float()).abs() <= 4 * 2.0 ** -8 * 5.5).all())
    assert bool(((lse - want_lse).abs() <= 2.0 ** -14).all())
    mass = torch.full((2 * n_seq, 1, 64), 1e30, device="cuda")
    kt.kt_attention_mass(q, cache, ints(pages), ints(lens), lse, mass, decay=0.0, **more)
    per_seq = torch.zeros(n_seq, dtype=torch.float64, device="cuda").index_add_(0, seq.cuda(), mass.reshape(-1)[slots].double())
    rows = counts.cuda() * group
    assert bool(((per_seq - rows).abs() <= 2.0 ** -13 * rows).all())
    untouched = torch.ones(2 * n_seq * 64, dtype=torch.bool, device="cuda")
    untouched[slots] = False
    assert bool((mass.reshape(-1)[untouched] == 1e30).all())


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("count", [9, 70], ids=["few", "many"])
def test_weights_in_far_pages_add_up(fmt, count):
    """Masses of a cache of more than 4 GiB: a weight of one a row, from above and from below."""
    heads, hd, page, t = 8, 256, 1024, 1100
    n_pages = (1 << 32) // (page * heads * {kt.KT_KV_BF16: 1024, kt.KT_KV_U8: 528, kt.KT_KV_U4: 272}[fmt]) + 8
    cache = kt.KVCache(n_pages, page, heads, hd, fmt)
    assert cache.nbytes > 1 << 32
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn(t, heads, hd, generator=g).cuda() for _ in range(2))
    q = torch.randn(count, heads, hd, generator=g).to(torch.bfloat16).cuda()
    table = torch.tensor([n_pages - 1, n_pages - 2], device="cuda")
    at = torch.arange(t, device="cuda")
    kt.kt_kv_append(cache, k, v, table[at // page] * page + at % page)
    pages, lens, starts = table[None].int(), ints([t]), ints([0, count])
    lse = torch.empty(count, heads, device="cuda")
    kt.kt_paged_attention(q, cache, pages, lens, q_starts=starts, max_q=count, lse=lse)
    mass = torch.zeros(n_pages, heads, page, device="cuda")
    kt.kt_attention_mass(q, cache, pages, lens, lse, mass, q_starts=starts, max_q=count)
    sums = mass[table].double().sum((0, 2))
    assert bool(((sums - count).abs() <= 2.0 ** -13 * count).all()) and bool((mass[:-2] == 0).all())
