"""kt_attention_mass: attention weight accumulated a token and key head."""
import math

import pytest
import torch

import paper_2503_01483_amd as kt
from draft_util import FORMATS, NAMES, ints, mass_check, mass_expected
from serving_util import Batch

pytestmark = pytest.mark.gpu


def exact_lse(b):
    return b.expected()[1].float()


def start(b, seed=1, fill=None):
    shape = (b.cache.n_pages, b.hkv, b.page)
    return torch.full(shape, fill) if fill is not None else torch.rand(shape, generator=torch.Generator().manual_seed(seed)) * 3


def call(b, lse, mass, **kw):
    more = {} if b.single else dict(q_starts=ints(b.starts), max_q=max(1, max(b.counts)))
    more.update(kw)
    return kt.kt_attention_mass(b.q.cuda(), b.cache, b.pages, ints(b.lens), lse.cuda(), mass, **more)


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("hd,hkv,group", [(64, 2, 3), (128, 2, 4), (128, 1, 1), (256, 2, 2), (64, 1, 16), (128, 1, 24)])
@pytest.mark.parametrize("lens,counts", [([1, 63, 64, 300], None), ([1, 5, 70, 200], [1, 5, 3, 9]), ([320, 150, 64], [200, 150, 0])], ids=["tokens", "few", "many"])
@pytest.mark.parametrize("decay", [1.0, 0.75])
def test_against_fp64(fmt, hd, hkv, group, lens, counts, decay):
    print(NAMES[fmt], hd, hkv, group, lens, counts, decay, flush=True)
    b = Batch(fmt, hd, hkv, group, lens, counts, seed=hd + group, page=128 if hd == 64 else 64)
    lse, before = exact_lse(b), start(b)
    got = call(b, lse, before.cuda(), decay=decay)
    mass_check(b, got, lse, before, decay)


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("counts", [None, [40, 90]], ids=["tokens", "chunks"])
def test_rows_add_up_to_their_number(fmt, counts):
    """With the lse that attention writes, every row hands out a weight of one."""
    b = Batch(fmt, 128, 2, 4, [130, 100], counts, seed=3)
    lse = torch.empty(b.n, b.hq, device="cuda")
    b.call(lse=lse)
    mass = torch.zeros(b.cache.n_pages, b.hkv, b.page, device="cuda")
    call(b, lse, mass)
    rows = sum(b.counts) * 4
    assert bool(((mass.double().sum((0, 2)) - rows).abs() <= 2.0 ** -14 * rows).all())


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("counts", [None, [7, 64, 1]], ids=["tokens", "chunks"])
def test_what_is_not_read_may_be_anything(fmt, counts):
    """Old masses of the queries' own tokens, and all of them without decay; other places stay as they are."""
    b = Batch(fmt, 64, 2, 4, [90, 64, 1], counts, seed=4)
    lse = exact_lse(b)
    for decay in (0.0, 0.5):
        before = start(b, fill=math.nan)
        if decay:
            for s, t in enumerate(b.lens):
                for j in range(t - b.counts[s]):
                    before[b.pages[s, j // b.page], :, j % b.page] = 0.25 * (j % 5)
        got = call(b, lse, before.cuda(), decay=decay).cpu()
        mass_check(b, got, lse, before, decay)
        written = torch.zeros(got.shape, dtype=torch.bool)
        for s, t in enumerate(b.lens):
            for j in range(t):
                written[b.pages[s, j // b.page], :, j % b.page] = True
        assert torch.equal(torch.isnan(got), ~written)


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
def test_rows_whose_lse_is_not_finite_add_nothing(fmt):
    b = Batch(fmt, 128, 1, 4, [70, 50], [20, 50], seed=5)
    lse, before = exact_lse(b), start(b)
    lse[3, 1], lse[22, 0], lse[40, 3], lse[69] = math.nan, -math.inf, math.inf, math.nan
    mass_check(b, call(b, lse, before.cuda()), lse, before, 1.0)


def test_a_key_of_infinities_reaches_its_own_mass_alone():
    """Rows in front of it and the other keys are as ever, also beside rows that a wave has no query for."""
    b = Batch(kt.KT_KV_BF16, 128, 1, 3, [50], [30], seed=6)
    lse, before = exact_lse(b), start(b)
    want = call(b, lse, before.cuda()).cpu()
    slots = (b.pages[0, 0].long() * b.page + 45)[None]
    k, v = kt.kt_kv_gather(b.cache, slots)
    k[0, 0, 3] = math.inf
    kt.kt_kv_append(b.cache, k, v, slots)
    got = call(b, lse, before.cuda()).cpu()
    at = int(b.pages[0, 0])
    got[at, 0, 45] = want[at, 0, 45]
    assert torch.equal(got, want)


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
def test_long_lists_of_keys_and_rows(fmt):
    """Lengths of many blocks, more sequences than a workgroup has threads, empty ones among them."""
    lens = [(37 * i) % 150 for i in range(300)]
    lens[17] = 2500
    b = Batch(fmt, 64, 1, 2, lens, [min(t, i % 3) for i, t in enumerate(lens)], seed=7)
    lse, before = exact_lse(b), start(b)
    mass_check(b, call(b, lse, before.cuda()), lse, before, 1.0)


@pytest.mark.parametrize("counts", [None, [30, 80]], ids=["tokens", "chunks"])
def test_captured(counts):
    b = Batch(kt.KT_KV_U4, 128, 2, 4, [200, 150], counts, seed=8)
    lse, before = exact_lse(b), start(b)
    q, pages, lens, starts, z = b.q.cuda(), b.pages, ints(b.lens), ints(b.starts), lse.cuda()
    mass = before.cuda()
    more = {} if counts is None else dict(q_starts=starts, max_q=80)
    run = lambda: kt.kt_attention_mass(q, b.cache, pages, lens, z, mass, decay=0.5, **more)  # noqa: E731
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    mass.copy_(before)
    for _ in range(3):
        was = mass.cpu()
        graph.replay()
        torch.cuda.synchronize()
        mass_check(b, mass, lse, was, 0.5)
        again = was.cuda()
        kt.kt_attention_mass(q, b.cache, pages, lens, z, again, decay=0.5, **more)
        assert torch.equal(again, mass)


def test_pages_outside_the_cache_are_passed_over():
    b = Batch(kt.KT_KV_U8, 64, 1, 2, [200], [150], seed=9)
    lse, before = exact_lse(b), start(b)
    want = call(b, lse, before.cuda()).cpu()
    gone = int(b.pages[0, 1])
    b.pages[0, 1] = b.cache.n_pages
    got = call(b, lse, before.cuda()).cpu()
    want[gone] = before[gone]
    assert torch.equal(got, want)


def test_sequences_longer_than_the_bound_on_their_queries():
    """max_q lays the launch out; no row is left out."""
    b = Batch(kt.KT_KV_BF16, 64, 1, 2, [200, 30], [150, 2], seed=10)
    lse, before = exact_lse(b), start(b)
    mass_check(b, call(b, lse, before.cuda(), max_q=2), lse, before, 1.0)


def test_another_scale_and_strided_queries():
    b = Batch(kt.KT_KV_U4, 128, 2, 2, [70], [33], seed=11)
    b.q = (b.q.float() * 0.5).to(torch.bfloat16)
    lse, before = exact_lse(b), start(b)
    wide = torch.zeros(b.n, 3 * b.hq, b.hd, dtype=torch.bfloat16, device="cuda")
    wide[:, b.hq:2 * b.hq] = b.q.cuda()
    got = kt.kt_attention_mass(wide[:, b.hq:2 * b.hq], b.cache, b.pages, ints(b.lens), lse.cuda(), before.cuda(), q_starts=ints(b.starts), max_q=33)
    assert torch.equal(got, call(b, lse, before.cuda()))
    twice = call(b, lse, before.cuda(), scale=2 * b.hd ** -0.5)
    b.q = (b.q.float() * 2).to(torch.bfloat16)
    mass_check(b, twice, lse, before, 1.0)
    assert not torch.equal(twice, got)
    assert mass_expected(b, lse, before, 1.0)[0].shape == got.shape
