"""kt_paged_attention against what its documentation says of each rounding: no more is off, whatever the values' sizes."""
import pytest
import torch

import paper_2503_01483_amd as kt
from attention_bounds import check, expected, replace
import serving_util as su
from serving_util import Batch

pytestmark = pytest.mark.gpu
FMT = [kt.KT_KV_BF16, kt.KT_KV_U8, kt.KT_KV_U4]
IDS = ["bf16", "u8", "u4"]


def run(b, **kw):
    out, lse = torch.zeros(b.n, b.hq, b.hd, dtype=torch.bfloat16, device="cuda"), torch.zeros(b.n, b.hq, device="cuda")
    b.call(out=out, lse=lse, **kw)
    return out, lse


@pytest.mark.parametrize("fmt", FMT, ids=IDS)
@pytest.mark.parametrize("hd,group", [(64, 3), (128, 4), (256, 2)])
def test_every_rounding_is_within_its_bound(fmt, hd, group):
    """Few rows and many, with and without a prefix: values of one size, and values that all lie on one side (their output does not cancel)."""
    for counts in ([2, 1, 7], [70, 33, 5]):
        for prefix in (0, 100):
            b = Batch(fmt, hd, 2, group, [300, 64, 9], counts, prefix=prefix, seed=hd + prefix)
            check(b, *run(b))


@pytest.mark.parametrize("fmt", FMT, ids=IDS)
def test_sums_are_not_biased(fmt):
    """A value that all tokens share comes back as itself: what p is rounded by may go either way, not one.

    256 values (sequences x heads), sixteen to a step of bf16, evenly and none nearer than 2^-12 to the middle of two: rounded to bf16 their errors cancel.
    A row's 130 independent roundings of p (2^-11 each at most, fp16; 2^-8, bf16) move its sum by 2^-15 (2^-12), either way, and so change results of 16896 rows
    by less than 2^-13 in the mean; p cut off to 11 bits is 2^-11.5 too small in the mean, which takes one of sixteen values a step of 2^-7 down: 2^-11."""
    b = Batch(fmt, 64, 8, 1, [130] * 32, [66] * 32, seed=23)
    step = torch.arange(256).reshape(32, 1, 8, 1)
    value = 1 + step.div(16, rounding_mode="floor") * 2.0 ** -7 + (step % 16 + 0.5) * 2.0 ** -11
    for s in range(32):
        replace(b, s, range(130), v=value[s].expand(130, 8, 64).contiguous())
    out, lse = run(b)
    check(b, out, lse)
    want = torch.cat([b.v[s][:1].expand(66, 8, 64) for s in range(32)])
    if fmt != kt.KT_KV_BF16:
        assert torch.equal(want[::66], value[:, 0].expand(32, 8, 64).double())        # (a row of one value is held as its minimum)
    far = float((out.cpu().double() - want).mean().abs())
    assert far < 2.0 ** -13, far


def one_key_a_query(b, seq, tokens, seed):
    """Queries of a sequence that each attend to one token, by 2^-20 or more."""
    g = torch.Generator().manual_seed(seed)
    k = torch.randn(b.lens[seq], b.hkv, b.hd, generator=g)
    replace(b, seq, range(b.lens[seq]), k=k)
    b.q[b.starts[seq]:b.starts[seq + 1]] = (64 / b.hd ** 0.5 * k[tokens]).repeat_interleave(b.hq // b.hkv, 1).to(torch.bfloat16)


@pytest.mark.parametrize("fmt", FMT[1:], ids=IDS[1:])
@pytest.mark.parametrize("hd", [64, 128, 256])
def test_values_of_many_rows_lose_no_more_than_their_bound(fmt, hd):
    """Rows just wider than -1 to 1, where the step's rounding and the middle's are as large as they get; one key a query, so that an output is a
    value, and those near 0 show what their row's step and middle were rounded by.  (s c + b from s and b in fp16 is off by up to 2 x 2^-11.)"""
    n, count, g = 512, 100, torch.Generator().manual_seed(21)
    for tokens in (4 * torch.arange(count), n - count + torch.arange(count)):      # in tiles that all rows see, and in those that they do not
        b = Batch(fmt, hd, 2, 2, [n], [count], seed=21)
        wide = 1 + 0.03 * torch.rand(2, n, 2, 1, generator=g)
        v = torch.rand(n, 2, hd, generator=g) * 0.1 - 0.05
        v[..., :1], v[..., 1:2] = -wide[0], wide[1]
        replace(b, 0, range(n), v=v)
        one_key_a_query(b, 0, tokens, 22)
        check(b, *run(b))


@pytest.mark.parametrize("fmt", FMT, ids=IDS)
@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("prefix", [0, 64])
@pytest.mark.parametrize("group", [3, 65])
def test_large_values_of_next_to_no_weight_take_no_bits_off_others(fmt, hd, prefix, group):
    """64 tokens in front have values 2^e times as large and weights of 2^-70 or less: what follows is as exact as without them, in few rows and many.
    (Lengths and heads for which a workgroup goes through several tiles of a segment in turn.)"""
    g = torch.Generator().manual_seed(31)
    heads, lens = 8, [1500, 100, 1500, 1500, 1400, 1500]
    b = Batch(fmt, hd, heads, group, lens, prefix=prefix, seed=30)
    b.q[..., 0] = 32
    for s, t in enumerate(lens):
        k = torch.randn(t, heads, hd, generator=g)
        k[..., 0] = 0
        replace(b, s, range(t), k=k)
    far = torch.randn(64, heads, hd, generator=g)
    far[..., 0] = -3.5 * hd ** 0.5                       # scores of -112 and a little: 2^-161
    for e in (0, 8, 14, 17, 20, 32, 60, 90):
        for s in [None] if prefix else range(len(lens)):
            replace(b, s, range(64), k=far, v=torch.randn(64, heads, hd, generator=g) * 2.0 ** e)
        print(f"2^{e}", end=" ")
        check(b, *run(b))


@pytest.mark.parametrize("fmt", FMT[1:], ids=IDS[1:])
@pytest.mark.parametrize("lift", [0, 100, -100])
def test_values_that_grow_and_shrink_along_a_sequence(fmt, lift):
    """Every tile of 64 tokens has values and scores of another size: values that rise and fall by 2^30, near the ends of the range too."""
    g = torch.Generator().manual_seed(32)
    hd, heads, t = 128, 8, 1280
    b = Batch(fmt, hd, heads, 65, [t] * 8, seed=33)
    b.q[..., 0] = 8
    for s in range(len(b.lens)):
        k, v = torch.randn(t, heads, hd, generator=g), torch.randn(t, heads, hd, generator=g)
        for tile in range(t // 64):
            at = slice(64 * tile, 64 * tile + 64)
            k[at, :, 0] = 30 * (torch.rand(1, generator=g) - 0.5)
            v[at] *= 2.0 ** (lift + 30 * float(torch.rand(1, generator=g) - 0.5))
        replace(b, s, range(t), k=k, v=v)
    check(b, *run(b))


@pytest.mark.parametrize("fmt", FMT, ids=IDS)
@pytest.mark.parametrize("hd,group,counts,prefix", [(64, 3, [70, 30], 0), (128, 4, [90, 17], 0), (128, 1, [100, 66], 70), (256, 2, [70, 40], 0), (256, 1, [70, 40], 64),
                                                    (64, 2, [5, 3], 0), (128, 4, [9, 4], 30), (256, 8, [2, 2], 0)])
def test_large_values_of_later_tokens_have_no_effect(fmt, hd, group, counts, prefix):
    """A token in the middle of each chunk has values 2^e times as large: queries in front of it give the same bits, the others are as exact as ever."""
    b = Batch(fmt, hd, 2, group, [200, 100], counts, prefix=prefix, seed=40)
    out, lse = run(b)
    check(b, out, lse)
    g = torch.Generator().manual_seed(41)
    for e in (8, 10, 12, 14, 16, 20, 40, 100):
        print(f"2^{e}", end=" ")
        for s, (t, n) in enumerate(zip(b.lens, b.counts)):
            replace(b, s, [t - n + n // 2], v=torch.randn(1, 2, hd, generator=g) * 2.0 ** e)
        now, lse2 = run(b)
        for s, n in enumerate(b.counts):
            rows = slice(b.starts[s], b.starts[s] + n // 2)
            assert torch.equal(now[rows], out[rows]) and torch.equal(lse2[rows], lse[rows])
        check(b, now, lse2)


@pytest.mark.parametrize("fmt", FMT, ids=IDS)
@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("prefix", [0, 200])
def test_sizes_that_differ_within_64_tokens(fmt, hd, prefix):
    """Single tokens with values 2^e times as large, or as small, as their neighbours', of next to no weight or of an ordinary one."""
    g = torch.Generator().manual_seed(42)
    heads, lens, at = 8, [900, 70, 900, 800], [3, 60, 69]
    b = Batch(fmt, hd, heads, 65, lens, prefix=prefix, seed=43)
    b.q[..., 0] = 32
    for s, t in enumerate(lens):
        k = torch.randn(t, heads, hd, generator=g)
        k[..., 0] = 0
        replace(b, s, range(t), k=k)
    for weight in (-3.5 * hd ** 0.5, 0.0):
        far = torch.randn(len(at), heads, hd, generator=g)
        far[..., 0] = weight
        for e in (-40, -9, 5, 7, 12, 20, 40, 100):
            for s in range(len(lens)):
                replace(b, s, at, k=far, v=torch.randn(len(at), heads, hd, generator=g) * 2.0 ** e)
            if prefix:
                replace(b, None, at, k=far, v=torch.randn(len(at), heads, hd, generator=g) * 2.0 ** e)
            print(f"2^{e}", end=" ")
            check(b, *run(b))


@pytest.mark.parametrize("fmt", FMT, ids=IDS)
@pytest.mark.parametrize("hd,group,counts", [(64, 1, 70), (128, 2, 70), (256, 1, 70), (64, 2, 8), (128, 4, 4), (128, 1, 16), (256, 2, 7)])
def test_keys_of_later_tokens_have_no_effect(fmt, hd, group, counts):
    """Later tokens that outweigh all others: queries in front of them give the same bits, also where they share a wave with queries that see them and
    a workgroup goes through several tiles in turn."""
    lens = [1500, 1480, 1500, 1300, 1490, 1500, 1500, 1410]
    b = Batch(fmt, hd, 8, group, lens, [counts] * len(lens), seed=50)
    out, lse = run(b)
    g = torch.Generator().manual_seed(51)
    for size in (3.0, 30.0, 1000.0):
        for s, t in enumerate(lens):
            n = counts // 4
            replace(b, s, range(t - n, t), k=torch.randn(n, 8, hd, generator=g) * size)
        now, lse2 = run(b)
        for s in range(len(lens)):
            rows = slice(b.starts[s], b.starts[s] + counts - counts // 4)
            assert torch.equal(now[rows], out[rows]), f"{int((now[rows] != out[rows]).sum())} values"
            assert torch.equal(lse2[rows], lse[rows])


@pytest.mark.parametrize("fmt", FMT[1:], ids=IDS[1:])
@pytest.mark.parametrize("hd,group", [(64, 3), (128, 4), (128, 1), (256, 2)])
def test_few_rows_keep_sixteen_bits_of_weight_times_step(fmt, hd, group):
    """Rows from 0 up, half of their features 0: the part of the centred codes and that of the middle cancel there, and what p step was rounded by is left.
    One term of 8 bits instead of two (computed here, in 64 bits) would be outside the bound."""
    b = Batch(fmt, hd, 2, group, [500, 130, 64], [1, 2, 5], seed=70)
    g = torch.Generator().manual_seed(71)
    for s, t in enumerate(b.lens):
        v = torch.rand(t, 2, hd, generator=g) * (1 + torch.rand(t, 2, 1, generator=g))
        v[..., ::2] = 0
        replace(b, s, range(t), v=v)
    out, lse = run(b)
    check(b, out, lse)
    _, _, tol, _ = expected(b)
    worst = 0.0
    for row in range(b.n):
        s = next(i for i in range(len(b.lens)) if row < b.starts[i + 1])
        sees = b.lens[s] - b.counts[s] + row - b.starts[s] + 1
        for h in range(b.hq):
            x = b.k[s][:sees, h // group] @ b.q[row, h].double() * hd ** -0.5
            p = torch.exp(x - x.max())
            step = b.v[s][:sees, h // group].amax(1) / su.TOP[fmt]
            lost = ((p * step).to(torch.bfloat16).double() - p * step).sum() * (8 if fmt == kt.KT_KV_U4 else 128) / p.sum()
            worst = max(worst, float(lost.abs() / tol[row, h, 0]))
    assert worst > 4, worst


@pytest.mark.parametrize("fmt", FMT, ids=IDS)
@pytest.mark.parametrize("hd,group,counts", [(64, 1, 100), (128, 2, 90), (256, 1, 70), (128, 4, 3)])
def test_scores_far_beyond_the_exponents_of_values(fmt, hd, group, counts):
    """Scores of 2^27 and more, 2^20 apart: a query's output is the value of its own token, whatever is added to a score on the way."""
    n, g = 200, torch.Generator().manual_seed(80)
    b = Batch(fmt, hd, 2, group, [n], [counts], seed=81)
    k = (torch.randint(0, 2, (n, 2, hd), generator=g) * 2 - 1) * 1024.0             # (held exactly)
    v = torch.randn(n, 2, hd, generator=g) * torch.exp(torch.randn(n, 2, 1, generator=g))
    replace(b, 0, range(n), k=k, v=v)
    own = torch.arange(n - counts, n)
    for at in (own, torch.arange(counts)):                                          # the last token that it sees, and one in front
        b.q[:] = (16 * k[at]).repeat_interleave(group, 1).to(torch.bfloat16)
        out, lse = run(b)
        want = b.v[0][at].repeat_interleave(group, 1)
        most = want.abs().amax(-1, keepdim=True) * (0 if fmt == kt.KT_KV_BF16 else 1)
        # p = 1: the result's rounding, and the value's (p step to 16 bits in few rows; 1.5 x 2^-11 of the row's largest, or of 2^7 times it)
        near = torch.stack([b.v[0][int(i) // 64 * 64:int(i) // 64 * 64 + 64].abs().amax((0, 2)) for i in at]).repeat_interleave(group, 1)[..., None]
        bound = 2.0 ** -8 * want.abs() + 1.5 * 2.0 ** -11 * torch.minimum(128 * most, near)
        assert bool(((out.cpu().double() - want).abs() <= bound).all()), float(((out.cpu().double() - want).abs() / bound).max())
        score = 16 * 1024.0 ** 2 * hd ** 0.5
        assert bool(((lse.cpu().double() / score - 1).abs() <= 2.0 ** -20).all())


@pytest.mark.parametrize("seed", range(24))
def test_random_sizes(seed):
    """Calls of any shape whose tokens' values and keys are of any size."""
    g = torch.Generator().manual_seed(900 + seed)
    pick = lambda *v: v[int(torch.randint(0, len(v), (1,), generator=g))]  # noqa: E731
    whole = lambda lo, hi: int(torch.randint(lo, hi + 1, (1,), generator=g))  # noqa: E731
    fmt, hd, hkv, group = pick(*FMT), pick(64, 128, 256), pick(1, 2, 8), pick(1, 2, 5, 8, 65)
    lens = [whole(0, pick(70, 400, 1500)) for _ in range(whole(1, 6))]
    counts = None if group == 65 else [whole(0, min(t, pick(1, 5, 90))) for t in lens]
    if counts is not None and sum(counts) == 0:
        lens[0], counts[0] = max(lens[0], 1), 1
    prefix, spread, tilt = pick(0, 0, 1, 64, 300), pick(0.0, 1.0, 5.0, 20.0), pick(0.0, 1.0, 10.0)
    print(f"seed {seed} fmt {fmt} hd {hd} hkv {hkv} group {group} lens {lens} counts {counts} prefix {prefix} spread {spread} tilt {tilt}", flush=True)
    b = Batch(fmt, hd, hkv, group, lens, counts, prefix=prefix, page=pick(64, 128), seed=seed, pad=whole(0, 3) if counts else 0)
    for s, t in [*enumerate(lens), (None, prefix)]:
        if t:
            size = torch.exp2(spread * torch.randn(t, 1, 1, generator=g))
            k = torch.randn(t, hkv, hd, generator=g) + tilt * torch.randn(t, hkv, 1, generator=g) / hd ** 0.5
            replace(b, s, range(t), k=k, v=torch.randn(t, hkv, hd, generator=g) * size)
    check(b, *run(b))
