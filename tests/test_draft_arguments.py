"""Host-side checks of the entry points for drafted tokens and budgets (no GPU): every bad call is refused before anything is enqueued."""
import ctypes

import pytest
import torch

import paper_2503_01483_amd as kt
from paper_2503_01483_amd import binding

FAKE = 0x10000      # never dereferenced: every call below fails its checks
BIG = 1 << 40


def _cache(data=FAKE, n_pages=8, page_size=64, n_heads=2, head_dim=128, fmt=kt.KT_KV_U4):
    return ctypes.byref(binding._CacheDesc(data, n_pages, page_size, n_heads, head_dim, fmt))


BAD_CACHES = [(dict(data=None), 1), (dict(data=FAKE + 8), 2), (dict(page_size=96), 2), (dict(n_heads=0), 2), (dict(n_pages=0), 2), (dict(head_dim=96), 6), (dict(fmt=9), 3)]


def _tree(cache=None, Q=FAKE, ldq=512, dt=1, starts=FAKE, lens=FAKE, pages=FAKE, ldp=4, n_seq=2, n=10, max_q=8, hq=4, tree=FAKE, ldt=1, pp=None, plen=0,
          scale=0.1, O=FAKE, ldo=512, lse=None, ws=FAKE, wsb=BIG):
    return kt.lib().kt_tree_attention(_cache() if cache is None else cache, Q, ldq, dt, starts, lens, pages, ldp, n_seq, n, max_q, hq, tree, ldt, pp, plen, scale, O,
                                      ldo, lse, ws, wsb, None)


@pytest.mark.parametrize("bad,status,text", [
    (dict(tree=None), 1, "tree"), (dict(ldt=0), 2, "ldt"), (dict(max_q=65), 2, "ldt"), (dict(max_q=129, ldt=2), 2, "ldt"), (dict(max_q=(1 << 63) - 1), 2, "ldt"), (dict(max_q=(1 << 62), ldt=1 << 24), 2, "ldt"), (dict(tree=FAKE + 4), 2, "tree"),
    (dict(ldt=(1 << 24) + 1), 2, "ldt"), (dict(Q=None), 1, "null"), (dict(lens=None), 1, "null"), (dict(pages=None), 1, "null"), (dict(O=None), 1, "null"),
    (dict(dt=0), 3, "dtype"), (dict(n_seq=0), 1, "positive"), (dict(n=0), 1, "positive"), (dict(max_q=0), 1, "positive"), (dict(n_seq=4097), 6, "sequences"),
    (dict(starts=None), 1, "q_starts"), (dict(hq=3), 2, "n_q_heads"), (dict(ldq=504), 2, "leading"), (dict(ldo=500), 2, "leading"), (dict(ldp=0), 2, "ldp"),
    (dict(ldp=1 << 25), 2, "ldp"), (dict(plen=5), 1, "prefix"), (dict(scale=0.0), 1, "scale"), (dict(scale=float("nan")), 1, "scale"),
    (dict(ws=None), 4, "workspace"), (dict(wsb=100), 4, "workspace"), (dict(ws=FAKE + 64), 1, "workspace"), (dict(lens=FAKE + 2), 2, "aligned")])
def test_tree_attention_refuses(bad, status, text):
    assert _tree(**bad) == status and text in kt.kt_last_error()


def _mass(cache=None, Q=FAKE, ldq=512, dt=1, starts=FAKE, lens=FAKE, pages=FAKE, ldp=4, n_seq=2, n=10, max_q=8, hq=4, scale=0.1, lse=FAKE, decay=1.0, mass=FAKE):
    return kt.lib().kt_attention_mass(_cache() if cache is None else cache, Q, ldq, dt, starts, lens, pages, ldp, n_seq, n, max_q, hq, scale, lse, decay, mass, None)


@pytest.mark.parametrize("bad,status,text", [
    (dict(Q=None), 1, "null"), (dict(lens=None), 1, "null"), (dict(pages=None), 1, "null"), (dict(lse=None), 1, "null"), (dict(mass=None), 1, "null"),
    (dict(dt=0), 3, "dtype"), (dict(n=0), 1, "positive"), (dict(n=1 << 31), 1, "positive"), (dict(max_q=0), 1, "positive"), (dict(n_seq=0), 1, "n_seq"),
    (dict(n_seq=4097), 6, "sequences"), (dict(starts=None), 1, "q_starts"), (dict(hq=3), 2, "n_q_heads"), (dict(hq=0), 2, "n_q_heads"), (dict(ldq=504), 2, "ldq"),
    (dict(Q=FAKE + 8), 2, "ldq"), (dict(ldp=0), 2, "ldp"), (dict(ldp=1 << 25), 2, "ldp"), (dict(scale=-1.0), 1, "scale"), (dict(scale=float("inf")), 1, "scale"),
    (dict(decay=-0.1), 1, "decay"), (dict(decay=float("nan")), 1, "decay"), (dict(decay=float("inf")), 1, "decay"), (dict(mass=FAKE + 2), 2, "aligned"),
    (dict(n_seq=4096, ldp=1 << 24), 6, "blocks")])
def test_mass_refuses(bad, status, text):
    assert _mass(**bad) == status and text in kt.kt_last_error()


def _select(cache=None, mass=FAKE, lens=FAKE, pages=FAKE, ldp=4, n_seq=2, keep=FAKE, sink=0, recent=0, kept=FAKE, ldk=10, n_kept=FAKE + 64):
    return kt.lib().kt_kv_select(_cache() if cache is None else cache, mass, lens, pages, ldp, n_seq, keep, sink, recent, kept, ldk, n_kept, None)


@pytest.mark.parametrize("bad,status,text", [
    (dict(mass=None), 1, "null"), (dict(lens=None), 1, "null"), (dict(pages=None), 1, "null"), (dict(keep=None), 1, "null"), (dict(kept=None), 1, "null"),
    (dict(n_kept=None), 1, "null"), (dict(n_kept=FAKE), 1, "lens"), (dict(n_seq=0), 1, "n_seq"), (dict(n_seq=4097), 6, "sequences"), (dict(ldp=0), 2, "ldp"),
    (dict(sink=-1), 1, "sink"), (dict(recent=-1), 1, "recent"), (dict(ldk=0), 2, "ldk"), (dict(ldk=(1 << 30) + 1), 2, "ldk"), (dict(kept=FAKE + 1), 2, "aligned")])
def test_select_refuses(bad, status, text):
    assert _select(**bad) == status and text in kt.kt_last_error()


def _compact(cache=None, pages=FAKE, ldp=4, n_seq=2, src=FAKE, lds=10, per_head=0, count=FAKE, first=None, to=None, ldt=0, mass=None):
    return kt.lib().kt_kv_compact(_cache() if cache is None else cache, pages, ldp, n_seq, src, lds, per_head, count, first, to, ldt, mass, None)


@pytest.mark.parametrize("bad,status,text", [
    (dict(pages=None), 1, "null"), (dict(src=None), 1, "null"), (dict(count=None), 1, "null"), (dict(n_seq=0), 1, "n_seq"), (dict(n_seq=4097), 6, "sequences"),
    (dict(ldp=0), 2, "ldp"), (dict(lds=0), 2, "lds"), (dict(lds=(1 << 30) + 1), 2, "lds"), (dict(to=FAKE + 64, ldt=0), 2, "ldt"), (dict(to=FAKE + 64, ldt=1 << 25), 2, "ldt"),
    (dict(to=FAKE, ldt=3), 2, "ldt"), (dict(first=FAKE + 2), 2, "aligned"), (dict(mass=FAKE + 2), 2, "aligned")])
def test_compact_refuses(bad, status, text):
    assert _compact(**bad) == status and text in kt.kt_last_error()


@pytest.mark.parametrize("bad,status", BAD_CACHES)
def test_bad_caches(bad, status):
    for call in (_tree, _mass, _compact):
        assert call(cache=_cache(**bad)) == status, call
    if "data" not in bad:
        assert _select(cache=_cache(**bad)) == status
    for call in (_tree, _mass, _compact, _select):
        assert call(cache=ctypes.POINTER(binding._CacheDesc)()) == 1, call


def test_the_binding_refuses_what_is_not_on_the_current_device():
    cache = kt.KVCache(4, 64, 2, 64, kt.KT_KV_U4, device="cpu")
    q, i, m = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32), torch.zeros(4, 2, 64)
    table = torch.zeros(2, 3, dtype=torch.int32)
    for call in (lambda: kt.kt_tree_attention(q, cache, table, i, torch.zeros(2, 1, dtype=torch.int64)), lambda: kt.kt_attention_mass(q, cache, table, i, torch.zeros(2, 4), m),
                 lambda: kt.kt_kv_select(cache, m, table, i, 5), lambda: kt.kt_kv_compact(cache, table, table, i)):
        with pytest.raises(ValueError, match="current device"):
            call()
    with pytest.raises(ValueError, match="tree"):
        kt.kt_tree_attention(q, cache, table, i, torch.zeros(2, dtype=torch.int64))
