"""kt_kv_append and kt_kv_gather: what the cache holds, bit for bit against elementary fp32 operations."""
import math

import pytest
import torch

import paper_2503_01483_amd as kt
import serving_util as su

pytestmark = pytest.mark.gpu
FMT = [kt.KT_KV_BF16, kt.KT_KV_U8, kt.KT_KV_U4]
IDS = ["bf16", "u8", "u4"]


def _equal(a, b):
    return torch.equal(torch.nan_to_num(a.float(), nan=1e30), torch.nan_to_num(b.float(), nan=1e30))


@pytest.mark.parametrize("fmt", FMT, ids=IDS)
@pytest.mark.parametrize("hd,rot,inter,had", [(64, 64, False, True), (64, 16, True, False), (64, 48, False, False), (128, 128, False, True), (128, 64, True, True),
                                              (128, 0, False, True), (256, 256, False, False), (256, 128, False, True), (256, 256, True, True), (128, 0, False, False)])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_rotated_rows_in_their_slots(fmt, hd, rot, inter, had, dt):
    n, hq, hkv, page, n_pages = 150, 6, 3, 64 if hd == 64 else 128, 7
    g = torch.Generator().manual_seed(hd + rot)
    x = (torch.randn(n, (hq + 2 * hkv) * hd, generator=g) * torch.exp(torch.randn((hq + 2 * hkv) * hd, generator=g))).to(dt)
    slots = torch.randperm(n_pages * page, generator=g)[:n]
    slots[5], slots[77], slots[149] = -1, n_pages * page, -(1 << 40)        # padding, and slots that are not there
    pos = torch.randint(0, 500, (n,), generator=g).to(torch.int32)
    if rot:
        pos[9], pos[10] = -1, 500
    rope = su.rope_table(500, rot) if rot else None
    cache = kt.KVCache(n_pages, page, hkv, hd, fmt)
    cache.data.copy_(torch.randint(0, 256, (cache.data.numel(),), generator=g).to(torch.uint8))
    every = torch.arange(n_pages * page).cuda()
    before = kt.kt_kv_gather(cache, every, dtype=torch.float32)
    xd = x.cuda()
    q, k, v = xd.split([hq * hd, hkv * hd, hkv * hd], 1)
    q_out = torch.full((n, hq, hd), 5.0, dtype=dt, device="cuda")
    kt.kt_kv_append(cache, k, v, slots.cuda(), Q=q, positions=pos.cuda() if rot else None, rope=rope.cuda() if rot else None, interleaved=inter,
                    hadamard=had, Q_out=q_out)
    live = (slots >= 0) & (slots < n_pages * page)
    if rot:
        live &= (pos >= 0) & (pos < 500)
    xf = x.float().reshape(n, hq + 2 * hkv, hd)
    y = su.rotate(xf[:, :hq + hkv], pos.clamp(0, 499), rope, inter, had)
    want_q = torch.where(live[:, None, None], y[:, :hq].to(dt), torch.full((), 5.0, dtype=dt))
    assert torch.equal(q_out.cpu(), want_q)
    K, V = kt.kt_kv_gather(cache, every, dtype=torch.float32)
    for have, was, want in ((K, before[0], su.held(y[:, hq:], fmt)), (V, before[1], su.held(xf[:, hq + hkv:], fmt))):
        full = was.cpu().clone()
        full[slots[live]] = want[live]
        assert _equal(have.cpu(), full)
    # bf16 values: the fp32 ones rounded once; one of the two alone; repeated and absent slots
    some = torch.cat([slots[:20], slots[:3], torch.tensor([-5, n_pages * page + 3])]).cuda()
    Vb = torch.full((25, hkv, hd), 3.0, dtype=torch.bfloat16, device="cuda")
    kt.kt_kv_gather(cache, some, V=Vb)
    there = (some >= 0) & (some < n_pages * page)
    assert _equal(Vb[there].cpu(), V[some[there]].to(torch.bfloat16).cpu()) and bool((Vb[~there] == 3).all())


@pytest.mark.parametrize("fmt", FMT[1:], ids=IDS[1:])
def test_constant_tiny_and_not_finite_rows(fmt):
    n, hd = 8, 128
    k = torch.randn(n, 1, hd, generator=torch.Generator().manual_seed(2))
    k[1] = 2.5
    k[2] = 0.0
    k[3] = 1e-39 * k[3].sign()
    k[4, 0, 3], k[5, 0, 100], k[6, 0, 0] = math.nan, math.inf, -math.inf
    k[7] *= 1e38
    cache = kt.KVCache(1, 64, 1, hd, fmt)
    slots = torch.arange(n).cuda()
    kt.kt_kv_append(cache, k.cuda(), k.flip(0).contiguous().cuda(), slots)
    K, V = kt.kt_kv_gather(cache, slots, dtype=torch.float32)
    assert _equal(K.cpu(), su.held(k, fmt)) and _equal(V.cpu(), su.held(k.flip(0), fmt))
    assert bool((K[1] == 2.5).all()) and bool(torch.isnan(K[4:8]).all())


def test_tokens_one_by_one_hold_what_a_prompt_holds():
    n, hkv, hd = 200, 2, 128
    g = torch.Generator().manual_seed(4)
    k, v = (torch.randn(n, hkv, hd, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    slots = torch.arange(n).cuda() + 17
    for fmt in FMT:
        a, b = (kt.KVCache(4, 64, hkv, hd, fmt) for _ in range(2))
        a.data.zero_(), b.data.zero_()
        kt.kt_kv_append(a, k, v, slots, hadamard=True)
        for i in range(n):
            kt.kt_kv_append(b, k[i:i + 1], v[i:i + 1], slots[i:i + 1], hadamard=True)
        assert torch.equal(a.data, b.data)
