"""kt_attention_mass over pages that several sequences of a call name: each token has one owner, whatever the launch's order."""
import copy

import pytest
import torch

import paper_2503_01483_amd as kt
from draft_util import FORMATS, NAMES, ints, mass_expected
from serving_util import Batch

pytestmark = pytest.mark.gpu


def shared(fmt, lens, counts, tables, hd=128, hkv=2, group=4, seed=0):
    """A batch whose sequence s has page `tables[s][i]` of a pool at place i; what the pool holds is what is held of every token."""
    page, most = 64, max(max(t) for t in tables) + 1
    wide = max(len(t) for t in tables)
    b = Batch(fmt, hd, hkv, group, [page * most], None, seed=seed)
    pool = b.pages[0].cpu()
    b.pages = torch.stack([pool[torch.tensor(t + [0] * (wide - len(t)))] for t in tables]).cuda()
    b.lens, b.counts, b.single = list(lens), list(counts), False
    b.k, b.v = ([torch.cat([x[0][page * i:page * i + page] for i in table])[:t] for table, t in zip(tables, lens)] for x in (b.k, b.v))
    b.starts = [0]
    for c in counts:
        b.starts.append(b.starts[-1] + c)
    b.n = b.starts[-1]
    b.q = (torch.randn(b.n, b.hq, hd, generator=torch.Generator().manual_seed(seed + 1)) * 2).to(torch.bfloat16)
    return b


def check(b, decay, single=False):
    lse = b.expected()[1].float()
    before = torch.rand(b.cache.n_pages, b.hkv, b.page, generator=torch.Generator().manual_seed(5)) * 3
    want, tol = before.double(), torch.zeros(before.shape, dtype=torch.float64)
    for s in reversed(range(len(b.lens))):      # the first sequence last: it has the say
        one = copy.copy(b)
        one.lens, one.counts, one.starts, one.k, one.v, one.pages = [b.lens[s]], [b.counts[s]], b.starts[s:s + 2], [b.k[s]], [b.v[s]], b.pages[s:s + 1]
        w, off = mass_expected(one, lse, before, decay)
        tok = torch.arange(b.lens[s])
        at = b.pages[s].cpu().long()[tok // b.page], slice(None), tok % b.page
        want[at], tol[at] = w[at], off[at]
    more = {} if single else dict(q_starts=ints(b.starts), max_q=max(b.counts))
    for _ in range(3):
        got = kt.kt_attention_mass(b.q.cuda(), b.cache, b.pages, ints(b.lens), lse.cuda(), before.cuda(), decay=decay, **more).cpu().double()
        d = (got - want).abs()
        print(f"off by {float((d / tol.clamp_min(1e-300)).max()):.3f} of what it may", flush=True)
        assert bool((d <= tol).all())


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("counts", [[1, 1, 1, 1, 1, 1], [3, 9, 0, 5, 1, 2], [60, 90, 17, 5, 0, 130]], ids=["tokens", "few", "many"])
@pytest.mark.parametrize("decay", [0.0, 0.5, 1.0])
def test_a_prompt_that_sequences_share(fmt, counts, decay):
    """The first sequence has a part of the second page alone; others go on behind it, leave pages out, or share with one behind the first."""
    tables = [[0, 1], [0, 1, 2, 3, 4], [5, 6, 7], [5, 8, 7], [0, 9, 2, 10], [5, 6, 7, 11]]
    lens = [100, 300, 150, 192, 256, 200]
    check(shared(fmt, lens, counts, tables), decay, single=counts == [1] * 6)


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("most", [1, 30], ids=["tokens", "chunks"])
def test_many_sequences_behind_one_page(fmt, most):
    """More sequences than a wave has lanes; the owner changes token by token, an empty sequence and one whose first page is its own among them."""
    n = 150
    lens = [(53 * i) % 151 for i in range(n)]
    tables = [[0, 1 + 2 * i, 2 + 2 * i] for i in range(n)]
    tables[70][0] = 2 * n + 1
    counts = [1 if most == 1 else min(t, i % (most + 1)) for i, t in enumerate(lens)]
    check(shared(fmt, lens, counts, tables, hd=64, hkv=1, group=3, seed=7), 0.5, single=most == 1)


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("most", [1, 30], ids=["tokens", "chunks"])
def test_sharers_far_apart(fmt, most):
    """1100 sequences, few of which share: a page with one hundreds of places in front, the second page alone with nobody."""
    n = 1100
    lens = [(37 * i) % 100 + 20 for i in range(n)]
    tables = [[i % 97 if i % 97 < 3 else 100 + 2 * i, 101 + 2 * i] for i in range(n)]
    counts = [1 if most == 1 else min(t, (7 * i) % 4) for i, t in enumerate(lens)]
    if most > 1:
        counts[1067] = 30
    check(shared(fmt, lens, counts, tables, hd=64, hkv=1, group=3, seed=11), 0.5, single=most == 1)


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
def test_weights_of_a_shared_prompt_choose_the_same_tokens_every_time(fmt):
    b = shared(fmt, [320, 300, 310], [1, 1, 1], [[0, 1, 2, 3, 4], [0, 1, 2, 3, 5], [0, 1, 2, 3, 6]])
    q, lens, lse = b.q.cuda(), ints(b.lens), b.expected()[1].float().cuda()
    lists = []
    for _ in range(5):
        mass = torch.ones(b.cache.n_pages, b.hkv, b.page, device="cuda")
        for _ in range(4):
            kt.kt_attention_mass(q, b.cache, b.pages, lens, lse, mass, decay=0.5)
        lists.append((mass, kt.kt_kv_select(b.cache, mass, b.pages, lens, 100, sink=2, recent=8)[0]))
    assert all(torch.equal(m, lists[0][0]) and torch.equal(k, lists[0][1]) for m, k in lists)
    # 4 steps of fading by a half: what is left of a 1 at the start is 1 / 16, and every query adds at most one a head
    assert bool((lists[0][0][b.pages[0, :4].long()] >= 0.0625).all())
