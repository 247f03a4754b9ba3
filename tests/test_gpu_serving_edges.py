"""The serving operators where they can go wrong: what is not seen, odd layouts, far offsets, several calls at once, random calls."""
import math

import pytest
import torch

import paper_2503_01483_amd as kt
import serving_util as su
from serving_util import Batch

pytestmark = pytest.mark.gpu
FMT = [kt.KT_KV_BF16, kt.KT_KV_U8, kt.KT_KV_U4]
IDS = ["bf16", "u8", "u4"]


def _slot(b, seq, t):
    return int(b.pages[seq, t // b.page]) * b.page + t % b.page


@pytest.mark.parametrize("fmt", FMT, ids=IDS)
@pytest.mark.parametrize("hd,group,counts", [(128, 2, [40, 5]), (64, 4, [3, 1]), (256, 1, [70, 2]), (128, 4, [4, 4])])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_tokens_that_a_query_does_not_see_have_no_effect(fmt, hd, group, counts, what):
    """The last token but one of each sequence gets a key or value that is not finite: earlier queries give the same bits."""
    b = Batch(fmt, hd, 2, group, [100, 66], counts, seed=3)
    clean, lse = torch.zeros(b.n, b.hq, hd, dtype=torch.bfloat16, device="cuda"), torch.zeros(b.n, b.hq, device="cuda")
    b.call(out=clean, lse=lse)
    g = torch.Generator().manual_seed(5)
    for which in ("k", "v", "kv"):
        for seq, (length, count) in enumerate(zip(b.lens, b.counts)):
            t = length - 2 if count > 1 else length - 1
            k, v = (torch.randn(1, 2, hd, generator=g) for _ in range(2))
            if "k" in which:
                k[0, :, 3] = what
            if "v" in which:
                v[0, :, hd - 1] = what
            kt.kt_kv_append(b.cache, k.cuda(), v.cuda(), torch.tensor([_slot(b, seq, t)], device="cuda"))
        out, lse2 = torch.zeros_like(clean), torch.zeros_like(lse)
        b.call(out=out, lse=lse2)
        for seq, count in enumerate(b.counts):
            a, e = b.starts[seq], b.starts[seq + 1]
            blind = max(0, count - 2) if count > 1 else 0
            assert torch.equal(out[a:a + blind], clean[a:a + blind]) and torch.equal(lse2[a:a + blind], lse[a:a + blind])
            sees = out[a + blind:e].float()
            if which == "v" and fmt == kt.KT_KV_BF16:       # only the feature of that value
                assert bool(torch.isfinite(sees[..., :hd - 1]).all()) and not bool(torch.isfinite(sees[..., hd - 1]).any())
            elif which == "v":
                assert bool(torch.isnan(sees).all())        # a quantised row is NaN as a whole
            elif what != what or fmt != kt.KT_KV_BF16:
                assert bool(torch.isnan(sees).all())


@pytest.mark.parametrize("fmt", FMT, ids=IDS)
def test_prefix_and_gaps_in_the_rows(fmt):
    b = Batch(fmt, 128, 2, 4, [90, 10, 200], [30, 10, 25], prefix=77, seed=4, pad=11)
    starts = torch.tensor([0, 30, 40, 65], dtype=torch.int32, device="cuda") + 6      # six rows in front belong to nobody
    q = torch.cat([torch.randn(6, b.hq, 128).bfloat16(), b.q[:-6]]).cuda()
    out, lse = torch.full((b.n, b.hq, 128), 3.0, dtype=torch.bfloat16, device="cuda"), torch.full((b.n, b.hq), 3.0, device="cuda")
    b.call(Q=q, q_starts=starts, out=out, lse=lse)
    ref, zref = torch.zeros_like(out), torch.zeros_like(lse)
    b.call(out=ref, lse=zref)
    assert bool((out[:6] == 3).all()) and bool((out[71:] == 3).all()) and bool((lse[:6] == 3).all()) and bool((lse[71:] == 3).all())
    # (row tiles begin at a sequence's first row: the same sums in the same order)
    assert torch.equal(out[6:71], ref[:65]) and torch.equal(lse[6:71], zref[:65])


def test_many_sequences():
    g = torch.Generator().manual_seed(6)
    lens = torch.randint(0, 130, (700,), generator=g).tolist()
    b = Batch(kt.KT_KV_U4, 64, 1, 2, lens, seed=6)
    out, lse = torch.zeros(b.n, b.hq, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(b.n, b.hq, device="cuda")
    b.call(out=out, lse=lse)
    b.check(out, lse)
    counts = [int(torch.randint(0, 12, (1,), generator=g)) for _ in lens]
    c = Batch(kt.KT_KV_U8, 64, 1, 3, lens, [min(a, n) if n else a for a, n in zip(counts, lens)], seed=7)
    out, lse = torch.zeros(c.n, c.hq, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(c.n, c.hq, device="cuda")
    c.call(out=out, lse=lse)
    c.check(out, lse)


@pytest.mark.parametrize("fmt,hd", [(kt.KT_KV_BF16, 256), (kt.KT_KV_U4, 128)])
def test_pages_beyond_four_gigabytes(fmt, hd):
    page, heads = 1024, 4
    per = kt.KVCache(1, page, heads, hd, fmt, device="cpu").data.numel()
    n_pages = (9 << 30) // per
    cache = kt.KVCache(n_pages, page, heads, hd, fmt)
    g = torch.Generator().manual_seed(8)
    n = 1500
    k, v = (torch.randn(n, heads, hd, generator=g).bfloat16() for _ in range(2))
    pages = torch.tensor([[n_pages - 1, n_pages // 2 + 1]], dtype=torch.int32, device="cuda")
    t = torch.arange(n)
    slots = (pages[0].cpu().long()[t // page] * page + t % page).cuda()
    q = torch.randn(n, 2 * heads, hd, generator=g).bfloat16()
    qd = kt.kt_kv_append(cache, k.cuda(), v.cuda(), slots, Q=q.cuda())
    assert torch.equal(qd.cpu(), q)
    K, V = kt.kt_kv_gather(cache, slots, dtype=torch.float32)
    assert torch.equal(K.cpu(), su.held(k.float(), fmt)) and torch.equal(V.cpu(), su.held(v.float(), fmt))
    small = kt.KVCache(3, page, heads, hd, fmt)
    near = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda")
    kt.kt_kv_append(small, k.cuda(), v.cuda(), (near[0].cpu().long()[t // page] * page + t % page).cuda())
    lens, starts = torch.tensor([n], dtype=torch.int32, device="cuda"), torch.tensor([0, n], dtype=torch.int32, device="cuda")
    for kw in (dict(q_starts=starts, max_q=n), dict()):
        rows = qd if kw else qd[-1:].contiguous()
        assert torch.equal(kt.kt_paged_attention(rows, cache, pages, lens, **kw), kt.kt_paged_attention(rows, small, near, lens, **kw))


def test_two_calls_at_once_on_two_streams():
    a, b = Batch(kt.KT_KV_U4, 128, 4, 4, [3000, 50, 700] * 8, seed=9), Batch(kt.KT_KV_BF16, 128, 2, 4, [900, 400], [900, 400], seed=10)
    ra, rb = a.call(), b.call()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    wa, wb = kt.Workspace(), kt.Workspace()
    oa, ob = [torch.zeros_like(ra) for _ in range(4)], [torch.zeros_like(rb) for _ in range(4)]
    torch.cuda.synchronize()
    for i in range(4):
        with torch.cuda.stream(sa):
            a.call(out=oa[i], workspace=wa)
        with torch.cuda.stream(sb):
            b.call(out=ob[i], workspace=wb)
    torch.cuda.synchronize()
    assert all(torch.equal(o, ra) for o in oa) and all(torch.equal(o, rb) for o in ob)


def test_captured_append_norm_and_prompt_replay_like_eager_calls():
    g = torch.Generator().manual_seed(11)
    n, hq, hkv, hd = 70, 4, 2, 128
    qkv = torch.randn(n, (hq + 2 * hkv) * hd, generator=g).bfloat16().cuda()
    rope, pos = su.rope_table(256, hd).cuda(), torch.arange(n, dtype=torch.int32).cuda()
    pages = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda")
    slots = (pages[0].long()[pos.long() // 64] * 64 + pos % 64).contiguous()
    lens, starts = torch.tensor([n], dtype=torch.int32, device="cuda"), torch.tensor([0, n], dtype=torch.int32, device="cuda")

    def state():
        return dict(cache=kt.KVCache(2, 64, hkv, hd, kt.KT_KV_U4), q=torch.empty(n, hq, hd, dtype=torch.bfloat16, device="cuda"), ws=kt.Workspace(),
                    out=torch.zeros(n, hq, hd, dtype=torch.bfloat16, device="cuda"), codes=torch.empty(n, hq * hd, dtype=torch.int8, device="cuda"),
                    scales=torch.empty(n, device="cuda"), stream=torch.zeros(n, hq * hd, dtype=torch.bfloat16, device="cuda"))

    def step(s):
        q, k, v = qkv.split([hq * hd, hkv * hd, hkv * hd], 1)
        kt.kt_kv_append(s["cache"], k, v, slots, Q=q, positions=pos, rope=rope, hadamard=True, Q_out=s["q"])
        kt.kt_paged_attention(s["q"], s["cache"], pages, lens, q_starts=starts, max_q=n, out=s["out"], workspace=s["ws"])
        kt.kt_add_rmsnorm_quant(s["out"].view(n, -1), res=s["stream"], res_out=s["stream"], codes=s["codes"], scales=s["scales"])

    eager, cap = state(), state()
    step(eager), step(cap)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        step(cap)
    for i in range(4):
        qkv.mul_(0.9)
        graph.replay()
        step(eager)
        torch.cuda.synchronize()
        for key in ("q", "out", "codes", "scales", "stream"):
            assert torch.equal(cap[key], eager[key]), (i, key)
        _ = (qkv.float() ** 2).sum().item()


@pytest.mark.parametrize("seed", range(12))
def test_random_calls(seed):
    g = torch.Generator().manual_seed(100 + seed)
    pick = lambda *v: v[int(torch.randint(0, len(v), (1,), generator=g))]  # noqa: E731
    whole = lambda lo, hi: int(torch.randint(lo, hi + 1, (1,), generator=g))  # noqa: E731
    fmt, hd, hkv, group = pick(*FMT), pick(64, 128, 256), pick(1, 2, 3), pick(1, 2, 5, 8)
    lens = [whole(0, 400) for _ in range(whole(1, 6))]
    counts = None if whole(0, 2) == 0 else [whole(0, min(t, pick(1, 5, 90))) if t else whole(0, 2) for t in lens]
    if counts is not None and sum(counts) == 0:
        counts[0] = 1
    prefix = pick(0, 0, 1, 64, 300)
    print(f"seed {seed} fmt {fmt} hd {hd} hkv {hkv} group {group} lens {lens} counts {counts} prefix {prefix}", flush=True)
    b = Batch(fmt, hd, hkv, group, lens, counts, prefix=prefix, page=pick(64, 128), seed=seed, pad=whole(0, 3) if counts else 0)
    out, lse = torch.zeros(b.n, b.hq, hd, dtype=torch.bfloat16, device="cuda"), torch.zeros(b.n, b.hq, device="cuda")
    b.call(out=out, lse=lse)
    b.check(out, lse)
