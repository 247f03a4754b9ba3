"""What scores over a quantised cache may be off by: kt_attention_mass as its documentation bounds it, and sums of whole numbers, which are exact."""
import numpy as np
import pytest
import torch

import draft_util
import paper_2503_01483_amd as kt
from attention_bounds import replace
from draft_util import FORMATS, NAMES, ints, mass_check
from serving_util import TOP, Batch

pytestmark = pytest.mark.gpu

STEPS = {kt.KT_KV_BF16: 0, kt.KT_KV_U8: 255, kt.KT_KV_U4: 31}   # the largest number that a code enters with


def documented(fmt):
    """2^-20 of scale sum |q| (max |k| + STEPS steps), and of the term itself (scale, log2(e) and the exponential: 2^-22 each at most)."""
    return lambda b, q, k, ks, scale: 2.0 ** -20 * (scale * q.abs().sum(-1)[..., None] * (k.abs().amax(1) + STEPS[fmt] * ks) + 1)


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("hd,hkv,group", [(64, 2, 3), (128, 1, 4), (256, 1, 2)])
@pytest.mark.parametrize("counts", [[1, 1], [5, 9], [70, 90]], ids=["tokens", "few", "many"])
def test_weights_within_the_documented_bound(fmt, hd, hkv, group, counts, monkeypatch):
    """Keys of one large feature among small ones: steps are wide, and what a sum loses is far more than 2^-24 of sum |q k|."""
    monkeypatch.setattr(draft_util, "score_error", documented(fmt))
    b = Batch(fmt, hd, hkv, group, [100, 150], counts, seed=hd)
    g = torch.Generator().manual_seed(hd + 1)
    for s, t in enumerate(b.lens):
        k = 0.02 * torch.randn(t, hkv, hd, generator=g)
        k[..., 3] = torch.where(torch.rand(t, hkv, generator=g) < 0.5, 6.0, -6.0)
        replace(b, s, list(range(t)), k=k)
    lse = b.expected()[1].float()
    before = torch.rand(b.cache.n_pages, hkv, b.page, generator=g)
    got = kt.kt_attention_mass(b.q.cuda(), b.cache, b.pages, ints(b.lens), lse.cuda(), before.cuda(), q_starts=ints(b.starts), max_q=max(counts), decay=0.5)
    mass_check(b, got, lse, before, 0.5)


def whole_numbers(fmt, count, tokens, seed):
    """A sequence whose keys are codes times 1/4 and whose queries are whole numbers: 56 large features that cancel between the halves of a head and 8 of a few units in
    each half that are left.  Every sum of q times (16 + code, or code of 8 bits) stays below 2^24, where whole numbers are exact; of q times (128 + code) it does not."""
    rng = np.random.default_rng(seed)
    hkv, group, hd, top = 2, 4, 128, 255 if fmt == kt.KT_KV_U8 else 15
    small = np.arange(0, 64, 8)
    large = np.setdiff1d(np.arange(64), small)
    b = Batch(fmt, hd, hkv, group, [tokens], [count], seed=seed)
    c = rng.integers(0, top + 1, (tokens, hkv, hd))
    c[..., 64 + large] = c[..., large]
    c[..., small], c[..., 64 + small] = (rng.integers(0, 16, (tokens, hkv, 8)) for _ in range(2))
    c[..., [1, 65]], c[..., [2, 66]] = 0, top                       # (minimum 0, step 1/4)
    q = np.zeros((count, hkv * group, hd))
    q[..., large] = 32 * rng.integers(128, 145, (count, hkv * group, 56)) if top == 15 else 4 * rng.integers(120, 140, (count, hkv * group, 56))
    q[..., 64 + large] = -q[..., large]
    q[..., small], q[..., 64 + small] = (rng.choice([-3, -1, 1, 3], (count, hkv * group, 8)) for _ in range(2))
    q = np.concatenate([q, np.zeros((b.n - count, hkv * group, hd))])
    assert np.abs(q).sum(-1).max() * max(STEPS[fmt], top) < 2 ** 24
    if fmt == kt.KT_KV_U4:
        assert (np.abs(q).sum(-1) / 2).min() * 128 > 2 ** 24        # of the first half
    b.q = torch.from_numpy(q).to(torch.bfloat16)
    assert torch.equal(b.q.double(), torch.from_numpy(q))
    k = torch.from_numpy(c / 4).float()
    replace(b, 0, list(range(tokens)), k=k)
    assert torch.equal(b.k[0], k.double()) and (fmt == kt.KT_KV_BF16 or TOP[fmt] == top)
    x = torch.einsum("rhgd,thd->rhgt", torch.from_numpy(q).reshape(-1, hkv, group, hd), torch.from_numpy(c).double())     # whole numbers, in fp64
    return b, x


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("count", [1, 9, 60], ids=["tokens", "few", "many"])
def test_whole_numbers_are_added_exactly_in_weights(fmt, count):
    """x / 4 * scale = x / 16: what is left are the roundings of scale log2(e), of a product, two sums and the exponential, 2^-21 of score, lse and one together."""
    tokens, z = 130, 1.5
    b, x = whole_numbers(fmt, count, tokens, 40 + count)
    lse = torch.full((b.n, b.hq), z, device="cuda")
    mass = torch.zeros(b.cache.n_pages, b.hkv, b.page, device="cuda")
    kt.kt_attention_mass(b.q.cuda(), b.cache, b.pages, ints(b.lens), lse, mass, q_starts=ints(b.starts), max_q=count, scale=0.25)
    seen = torch.arange(tokens)[None] <= tokens - count + torch.arange(count)[:, None]
    p = torch.where(seen[:, None, None], torch.exp(x[:count] / 16 - z), 0.0)
    off = (p * (2.0 ** -21 * (x[:count].abs() / 16 + z + 1) + (count * 4 / 16 + 12) * 2.0 ** -24)).sum((0, 2))       # [hkv, tokens]
    tok = torch.arange(tokens)
    got = mass.cpu().double()[b.pages[0].cpu().long()[tok // b.page], :, tok % b.page].t()
    d = (got - p.sum((0, 2))).abs()
    print(f"off by {float((d / off).max()):.3f} of what it may", flush=True)
    assert bool((d <= off).all())


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("count", [2, 9, 60], ids=["two", "few", "many"])
def test_whole_numbers_are_added_exactly_in_trees(fmt, count):
    """The same scores in lse: their roundings, and those of a sum of up to 130 terms (16 a lane, then in pairs, 2^-19) and of its logarithm (2^-22 of lse and one)."""
    tokens = 130
    b, x = whole_numbers(fmt, count, tokens, 60 + count)
    masks = [np.tril(np.ones((count, count), dtype=bool))]
    lse = torch.empty(b.n, b.hq, device="cuda")
    kt.kt_tree_attention(b.q.cuda(), b.cache, b.pages, ints(b.lens), draft_util.words_of(masks, b.n, 1), q_starts=ints(b.starts), max_q=count, lse=lse, scale=0.25)
    seen = torch.arange(tokens)[None] <= tokens - count + torch.arange(count)[:, None]
    y = torch.where(seen[:, None, None], x[:count] / 16, -torch.inf)
    want = torch.logsumexp(y, -1).reshape(count, -1)
    most = torch.where(seen[:, None, None], x[:count].abs(), 0.0).amax(-1).reshape(count, -1) / 16
    off = 2.0 ** -20 * (most + 1) + 2.0 ** -19 + 2.0 ** -22 * (want.abs() + 1)
    d = (lse.cpu().double()[:count] - want).abs()
    print(f"off by {float((d / off).max()):.3f} of what it may", flush=True)
    assert bool((d <= off).all())
