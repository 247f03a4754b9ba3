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


@pytest.mark.parametrize("fmt", FMT, ids=IDS)
def test_many_tokens_of_little_weight(fmt):
    """One token outweighs each of 2^17 others by 2^25 and has a value of 0; the others' values are 1: together they are 2^-8 of it."""
    hd, n, page, count = 64, (1 << 17) + 1, 1024, 20
    cache = kt.KVCache(n // page + 1, page, 1, hd, fmt)
    k, v = torch.zeros(n, 1, hd), torch.ones(n, 1, hd)
    k[0, 0, 0], v[0] = 1, 0                                    # scores 25 ln 2 and 0, in every format
    slots = torch.arange(n, device="cuda")
    kt.kt_kv_append(cache, k.cuda(), v.cuda(), slots)
    K, V = kt.kt_kv_gather(cache, slots, dtype=torch.float32)
    assert torch.equal(K.cpu(), k) and torch.equal(V.cpu(), v)
    q = torch.zeros(count, 1, hd, dtype=torch.bfloat16)
    q[:, 0, 0] = 1
    pages, lens = torch.arange(n // page + 1, dtype=torch.int32, device="cuda")[None], torch.tensor([n], dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, count], dtype=torch.int32, device="cuda")
    lse = torch.zeros(count, 1, device="cuda")
    out = kt.kt_paged_attention(q.cuda(), cache, pages, lens, q_starts=starts, max_q=count, scale=25 * math.log(2), lse=lse).cpu().double()
    seen = n - count + torch.arange(count, dtype=torch.double)  # others than the first
    mass = seen * 2.0 ** -25
    want = (mass / (1 + mass))[:, None, None].expand_as(out)
    # scale in fp32 times 1 / ln 2: the exponent is off by 2^-22 of 25 at most, p by 2^-18; a token's rounding 2^-31 (16 bits) or 2^-9; the result's 2^-9;
    # 2^13 sums of 16 products, one after the other if the segment is not cut, each cut off to 24 bits: 2^-10
    bound = want * (2.0 ** -18 + 2.0 ** -9 + 2.0 ** -10) * 1.01 + (want * 2.0 ** -9 if fmt == kt.KT_KV_BF16 else n * 2.0 ** -31)
    assert bool(((out - want).abs() <= bound).all()), float(((out - want).abs() / bound).max())
    assert bool(((lse.cpu()[:, 0].double() - (25 * math.log(2) + torch.log1p(mass))).abs() <= 2.0 ** -17).all())


@pytest.mark.parametrize("fmt", FMT, ids=IDS)
def test_values_near_the_end_of_the_range(fmt):
    """Values of 2^124 and of 2^-120, each alone and together."""
    for values in ([2.0 ** 124], [2.0 ** -120], [2.0 ** 124, 2.0 ** -120, 2.0 ** 124], [2.0 ** -120] * 3):
        n, count = len(values), 1
        cache = kt.KVCache(1, 64, 1, 64, fmt)
        v = torch.tensor(values)[:, None, None].expand(n, 1, 64).contiguous()
        kt.kt_kv_append(cache, torch.zeros(n, 1, 64, device="cuda"), v.cuda(), torch.arange(n, device="cuda"))
        for group in (1, 32):                                   # few rows, many
            q, pages, lens = torch.zeros(count, group, 64, dtype=torch.bfloat16), torch.zeros(1, 1, dtype=torch.int32), torch.tensor([n], dtype=torch.int32)
            out = kt.kt_paged_attention(q.cuda(), cache, pages.cuda(), lens.cuda()).cpu().double()
            want = sum(values) / n
            assert bool(((out - want).abs() <= want * (2.0 ** -8 + 2.0 ** -10)).all()), (values, group)


@pytest.mark.parametrize("hd", [64, 256])
def test_as_many_sequences_as_a_call_takes(hd):
    n = 4096
    lens = [(7 * i) % 5 for i in range(n)]
    b = Batch(kt.KT_KV_U8, hd, 1, 1, lens, seed=12, page=64)
    out, lse = torch.zeros(b.n, b.hq, hd, dtype=torch.bfloat16, device="cuda"), torch.zeros(b.n, b.hq, device="cuda")
    b.call(out=out, lse=lse)
    b.check(out, lse)
    wide = Batch(kt.KT_KV_U8, hd, 1, 32, lens, seed=13, page=64)
    out, lse = torch.zeros(wide.n, wide.hq, hd, dtype=torch.bfloat16, device="cuda"), torch.zeros(wide.n, wide.hq, device="cuda")
    wide.call(out=out, lse=lse)
    wide.check(out, lse)


@pytest.mark.parametrize("n,d", [((1 << 22) + 9, 8), ((1 << 20) + 3, 1024)])
def test_norm_of_more_rows_than_a_row_of_workgroups(n, d):
    x = torch.randn(n, d, dtype=torch.bfloat16, device="cuda")
    call = lambda rows: kt.kt_add_rmsnorm_quant(rows, codes=torch.empty(rows.shape, dtype=torch.int8, device="cuda"),  # noqa: E731
                                                scales=torch.empty(rows.shape[0], device="cuda"))
    codes, scales = call(x)
    for rows in (slice(0, 7), slice(n // 2, n // 2 + 9), slice(n - 11, n)):
        want = call(x[rows].clone())
        assert torch.equal(codes[rows], want[0]) and torch.equal(scales[rows], want[1])
    assert bool((codes.abs().amax(1) == 127).all())


@pytest.mark.parametrize("fmt,hd,group,counts", [(kt.KT_KV_U4, 128, 3, [7, 21, 1, 0, 20]), (kt.KT_KV_U8, 64, 1, [64, 17, 33]), (kt.KT_KV_BF16, 64, 32, [1, 1, 1]),
                                                 (kt.KT_KV_U8, 256, 5, [6, 3]), (kt.KT_KV_U4, 256, 64, [1, 1]), (kt.KT_KV_U4, 64, 9, [7, 5])])
@pytest.mark.parametrize("prefix", [0, 130])
def test_a_few_rows_more_than_sixteen(fmt, hd, group, counts, prefix):
    """Rows of one token on both sides of a boundary between row tiles; segments cut between workers; with and without a prefix."""
    for lens in ([max(n, t) for n, t in zip(counts, (300, 64, 1, 0, 1000))], [n + 5000 for n in counts]):
        b = Batch(fmt, hd, 2, group, lens, counts, prefix=prefix, seed=14, pad=2)
        out, lse = torch.zeros(b.n, b.hq, hd, dtype=torch.bfloat16, device="cuda"), torch.zeros(b.n, b.hq, device="cuda")
        b.call(out=out, lse=lse)
        b.check(out, lse)
