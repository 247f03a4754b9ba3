"""Host-side checks of the serving entry points (no GPU): every bad call is refused before anything is enqueued."""
import ctypes

import pytest
import torch

import paper_2503_01483_amd as kt
from paper_2503_01483_amd import binding

FAKE = 0x10000      # never dereferenced: every call below fails its checks
BIG = 1 << 40


def _cache(data=FAKE, n_pages=8, page_size=64, n_heads=2, head_dim=128, fmt=kt.KT_KV_U4):
    return ctypes.byref(binding._CacheDesc(data, n_pages, page_size, n_heads, head_dim, fmt))


def test_cache_bytes():
    L = kt.lib()
    size = lambda **kw: L.kt_kv_cache_bytes(_cache(**kw))  # noqa: E731
    assert size() == 8 * 2 * (2 * 64 * 64 + 1024)
    assert size(fmt=kt.KT_KV_U8, page_size=256) == 8 * 2 * 4 * (2 * 64 * 128 + 1024)
    assert size(fmt=kt.KT_KV_BF16, head_dim=64) == 8 * 2 * (2 * 64 * 64 * 2)
    assert size(head_dim=256) == 8 * 2 * (2 * 64 * 128 + 1024)
    assert size(n_pages=1 << 24, page_size=1024, n_heads=8) == (1 << 24) * 8 * 16 * 9216         # beyond 32 bits
    assert size(n_pages=1 << 30, page_size=1024, n_heads=8) == 0                                  # beyond 2^47 (2^30 8 16 9216 = 2^50.2)
    assert size(data=None) > 0                                                                     # the address is not looked at
    for bad in (dict(n_pages=0), dict(n_pages=1 << 31), dict(page_size=32), dict(page_size=96), dict(page_size=1 << 17), dict(n_heads=0),
                dict(n_heads=1025), dict(head_dim=96), dict(fmt=3), dict(fmt=-1), dict(n_pages=(1 << 31) - 1, page_size=65536, n_heads=1024)):
        assert size(**bad) == 0, bad
    assert L.kt_kv_cache_bytes(None) == 0


def _norm(L, X=FAKE, ldx=64, res=None, ldres=0, gain=None, n=4, d=64, dt=1, gdt=1, eps=1e-6, clip=1.0, fmt=kt.KT_Q_INT8, ro=None, ldro=0,
          Y=None, ldy=0, codes=FAKE, ldc=64, scales=FAKE):
    return L.kt_add_rmsnorm_quant(X, ldx, res, ldres, gain, n, d, dt, gdt, eps, clip, fmt, ro, ldro, Y, ldy, codes, ldc, scales, None)


@pytest.mark.parametrize("bad,status,text", [
    (dict(X=None), 1, "null"), (dict(codes=None, scales=None), 1, "output"), (dict(n=0), 1, "n must"), (dict(n=1 << 31), 1, "n must"),
    (dict(d=60), 2, "multiple of 8"), (dict(d=0), 2, "multiple of 8"), (dict(d=32776, ldx=32776, ldc=32776), 2, "32768"), (dict(dt=2), 3, "dtype"),
    (dict(gain=FAKE, gdt=7), 3, "gain_dtype"), (dict(fmt=4), 3, "format"), (dict(fmt=kt.KT_Q_NONE), 1, "neither"), (dict(eps=-1.0), 1, "eps"),
    (dict(eps=float("nan")), 1, "eps"), (dict(eps=float("inf")), 1, "eps"), (dict(clip=0.0), 1, "clip"), (dict(clip=1.5), 1, "clip"),
    (dict(clip=float("nan")), 1, "clip"), (dict(ldx=56), 2, "leading"), (dict(ldx=68), 2, "leading"), (dict(X=FAKE + 8), 2, "leading"),
    (dict(res=FAKE, ldres=0), 2, "leading"), (dict(ro=FAKE, ldro=60), 2, "leading"), (dict(Y=FAKE + 2, ldy=64), 2, "leading"),
    (dict(gain=FAKE + 4), 2, "gain"), (dict(codes=FAKE + 4), 2, "codes"), (dict(ldc=60), 2, "ldc"), (dict(ldc=68), 2, "ldc")])
def test_norm_refuses(bad, status, text):
    L = kt.lib()
    assert _norm(L, **bad) == status and text in kt.kt_last_error()


def _append(L, cache=None, Q=FAKE, ldq=512, K=FAKE, ldk=256, V=FAKE, ldv=256, n=3, hq=4, dt=1, slots=FAKE, pos=FAKE, rope=FAKE, n_pos=10, rot=128,
            Qo=FAKE, ldqo=512):
    return L.kt_kv_append(_cache() if cache is None else cache, Q, ldq, K, ldk, V, ldv, n, hq, dt, slots, pos, rope, n_pos, rot, 0, 0, Qo, ldqo, None)


@pytest.mark.parametrize("bad,status,text", [
    (dict(K=None), 1, "null"), (dict(V=None), 1, "null"), (dict(slots=None), 1, "null"), (dict(n=0), 1, "n must"), (dict(dt=5), 3, "dtype"),
    (dict(Q=None), 1, "together"), (dict(Qo=None), 1, "together"), (dict(hq=0), 2, "n_q_heads"), (dict(Q=None, Qo=None), 2, "n_q_heads"),
    (dict(ldq=504), 2, "leading"), (dict(ldk=252), 2, "leading"), (dict(V=FAKE + 4), 2, "leading"), (dict(ldqo=516), 2, "leading"),
    (dict(pos=None), 1, "positions"), (dict(rot=24), 2, "rot_dim"), (dict(rot=144), 2, "rot_dim"), (dict(rot=0), 2, "rot_dim"), (dict(n_pos=0), 1, "n_pos"),
    (dict(rope=FAKE + 4), 2, "rope"), (dict(slots=FAKE + 4), 2, "aligned"), (dict(pos=FAKE + 2), 2, "aligned"),
    (dict(cache=_cache(data=None)), 1, "data"), (dict(cache=_cache(data=FAKE + 8)), 2, "16-byte"), (dict(cache=_cache(head_dim=96)), 6, "head_dim"),
    (dict(cache=_cache(page_size=48)), 2, "page_size"), (dict(cache=_cache(fmt=9)), 3, "format"), (dict(n=(1 << 31) - 1), 6, "too many")])
def test_append_refuses(bad, status, text):
    L = kt.lib()
    assert _append(L, **bad) == status and text in kt.kt_last_error()


def test_gather_refuses():
    L = kt.lib()
    go = lambda slots=FAKE, n=3, K=FAKE, ldk=256, V=FAKE, ldv=256, dt=1, cache=None: L.kt_kv_gather(  # noqa: E731
        _cache() if cache is None else cache, slots, n, K, ldk, V, ldv, dt, None)
    for bad, status in ((dict(slots=None), 1), (dict(K=None, V=None), 1), (dict(n=0), 1), (dict(dt=3), 3), (dict(ldk=248), 2), (dict(V=FAKE + 8), 2),
                        (dict(slots=FAKE + 1), 2), (dict(cache=_cache(n_heads=0)), 2)):
        assert go(**bad) == status, bad


def _attend(L, cache=None, Q=FAKE, ldq=512, dt=1, starts=FAKE, lens=FAKE, pages=FAKE, ldp=4, n_seq=3, n=7, max_q=4, hq=4, pp=None, pl=0, scale=0.1,
            O=FAKE, ldo=512, lse=None, ws=1 << 20, wsb=BIG):
    return L.kt_paged_attention(_cache() if cache is None else cache, Q, ldq, dt, starts, lens, pages, ldp, n_seq, n, max_q, hq, pp, pl, scale, O, ldo,
                                lse, ws, wsb, None)


@pytest.mark.parametrize("bad,status,text", [
    (dict(Q=None), 1, "null"), (dict(lens=None), 1, "null"), (dict(pages=None), 1, "null"), (dict(O=None), 1, "null"), (dict(dt=0), 3, "BF16"),
    (dict(n_seq=0), 1, "positive"), (dict(n=0), 1, "positive"), (dict(max_q=0), 1, "positive"), (dict(n_seq=4097), 6, "4096"),
    (dict(starts=None), 1, "q_starts"), (dict(starts=None, n=3), 1, "q_starts"), (dict(hq=3), 2, "multiple"), (dict(hq=0), 2, "multiple"),
    (dict(ldq=504), 2, "leading"), (dict(Q=FAKE + 8), 2, "leading"), (dict(ldo=511), 2, "leading"), (dict(O=FAKE + 4), 2, "leading"),
    (dict(ldp=0), 2, "ldp"), (dict(ldp=1 << 25), 2, "ldp"), (dict(pl=-1), 1, "prefix_len"), (dict(pl=5), 1, "prefix_len"),
    (dict(pl=(1 << 30) + 1, pp=FAKE), 1, "prefix_len"), (dict(scale=0.0), 1, "scale"), (dict(scale=-1.0), 1, "scale"), (dict(scale=float("nan")), 1, "scale"),
    (dict(scale=float("inf")), 1, "scale"), (dict(ws=None), 4, "workspace"), (dict(wsb=1000), 4, "workspace"), (dict(ws=(1 << 20) + 16), 1, "256-byte"),
    (dict(lens=FAKE + 2), 2, "aligned"), (dict(lse=FAKE + 1), 2, "aligned"), (dict(cache=_cache(fmt=-3)), 3, "format"),
    (dict(n_seq=4096, starts=None, n=4096, max_q=1, ldp=1 << 20), 6, "too many"),
    (dict(n=1 << 28, max_q=1, pl=64, pp=FAKE, wsb=1 << 62), 6, "too many")])
def test_attention_refuses(bad, status, text):
    L = kt.lib()
    assert _attend(L, **bad) == status and text in kt.kt_last_error()


def test_attention_bytes():
    f = kt.lib().kt_paged_attention_bytes
    one = f(1, 32, 128, 0)
    assert 0 < one < 128 << 20 and f(1, 32, 128, 1) > one
    assert f(10000, 32, 128, 0) >= one and f(10000, 32, 128, 4096) > 2 * 10000 * 32 * 128 * 4
    for bad in ((0, 32, 128, 0), (1, 0, 128, 0), (1, 32, 100, 0), (1, 32, 128, -1), (1, 65536, 128, 0), (1, 32, 128, (1 << 30) + 1)):
        assert f(*bad) == 0


def test_the_binding_refuses_operands_that_are_not_on_the_gpu():
    cache = kt.KVCache(2, 64, 1, 64, kt.KT_KV_U4, device="cpu")
    assert cache.data.numel() == 2 * (2 * 64 * 32 + 1024)
    k, slots = torch.zeros(1, 1, 64), torch.zeros(1, dtype=torch.int64)
    for call in (lambda: kt.kt_add_rmsnorm_quant(torch.zeros(1, 64), scales=torch.zeros(1)), lambda: kt.kt_kv_append(cache, k, k, slots),
                 lambda: kt.kt_kv_gather(cache, slots), lambda: kt.kt_paged_attention(k.bfloat16(), cache, slots.int().view(1, 1), slots.int())):
        with pytest.raises(ValueError, match="current device"):
            call()


def test_the_cache_checks_its_sizes_and_data():
    with pytest.raises(kt.KtError, match="page_size"):
        kt.KVCache(2, 100, 1, 64, kt.KT_KV_U4, device="cpu")
    with pytest.raises(kt.KtError, match="head_dim"):
        kt.KVCache(2, 64, 1, 80, kt.KT_KV_U4, device="cpu")
    with pytest.raises(ValueError, match="bytes"):
        kt.KVCache(2, 64, 1, 64, kt.KT_KV_U4, data=torch.zeros(10, dtype=torch.uint8))
    with pytest.raises(ValueError, match="bytes"):
        kt.KVCache(2, 64, 1, 64, kt.KT_KV_U4, data=torch.zeros(2 * 5120, dtype=torch.int8))
