"""kt_paged_attention against fp64 attention over what the cache holds; unwritten cache bytes are NaN patterns throughout."""
import math

import pytest
import torch

import paper_2503_01483_amd as kt
from serving_util import Batch, rope_table

pytestmark = pytest.mark.gpu
FMT = [kt.KT_KV_BF16, kt.KT_KV_U8, kt.KT_KV_U4]
IDS = ["bf16", "u8", "u4"]


def _run(b, **kw):
    lse = torch.full((b.n, b.hq), 9.0, device="cuda")
    out = torch.full((b.n, b.hq, b.hd), 9.0, dtype=torch.bfloat16, device="cuda")
    b.call(out=out, lse=lse, **kw)
    b.check(out, lse, kw.get("scale"))
    assert bool((out[b.starts[-1]:] == 9).all()) and bool((lse[b.starts[-1]:] == 9).all())
    return out, lse


@pytest.mark.parametrize("fmt", FMT, ids=IDS)
@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("hkv,group", [(1, 1), (2, 4), (3, 7), (1, 16), (2, 17)])
def test_single_tokens(fmt, hd, hkv, group):
    _run(Batch(fmt, hd, hkv, group, [1, 2, 63, 64, 65, 127, 0, 200, 129], page=64 if group % 2 else 128, seed=hd + group))


@pytest.mark.parametrize("fmt", FMT, ids=IDS)
@pytest.mark.parametrize("hd,group", [(64, 2), (128, 4), (128, 1), (256, 3)])
def test_chunks_and_prompts(fmt, hd, group):
    _run(Batch(fmt, hd, 2, group, [1, 70, 64, 150, 33, 0, 5], [1, 70, 3, 40, 33, 0, 7], seed=hd, pad=5))


@pytest.mark.parametrize("fmt", FMT, ids=IDS)
@pytest.mark.parametrize("hd", [64, 128, 256])
def test_shared_prefix(fmt, hd):
    _run(Batch(fmt, hd, 2, 4, [1, 100, 0, 64, 33], prefix=130, page=64, seed=hd))
    _run(Batch(fmt, hd, 2, 3, [20, 100, 0, 64], [20, 1, 0, 30], prefix=64, page=128, seed=hd + 1, pad=3))
    _run(Batch(fmt, hd, 1, 2, [0, 5], prefix=1, seed=hd + 2))


@pytest.mark.parametrize("fmt", FMT, ids=IDS)
def test_long_contexts_are_cut_and_joined(fmt):
    b = Batch(fmt, 128, 1, 4, [9001], seed=5, page=256)
    out, lse = _run(b)
    again, lse2 = _run(b)
    assert torch.equal(out, again) and torch.equal(lse, lse2)      # the same bits every time
    _run(Batch(fmt, 64, 2, 2, [3000, 1, 500], prefix=4097, seed=6))
    _run(Batch(fmt, 128, 2, 8, [5000, 4000], [3, 1], seed=7))


@pytest.mark.parametrize("fmt", FMT, ids=IDS)
def test_large_and_small_scores(fmt):
    _run(Batch(fmt, 128, 1, 4, [300], spread=20.0, seed=8))        # one key takes nearly all
    _run(Batch(fmt, 128, 1, 4, [300], spread=1e-3, seed=9))
    _run(Batch(fmt, 128, 1, 4, [100, 40], [100, 40], seed=10), scale=0.7)


@pytest.mark.parametrize("fmt", FMT, ids=IDS)
def test_pages_outside_the_cache_hold_nothing(fmt):
    b = Batch(fmt, 64, 1, 2, [256, 256], seed=11)
    b.pages[0, 1], b.pages[1, 0], b.pages[1, 1], b.pages[1, 2], b.pages[1, 3] = -1, 1 << 30, -7, b.cache.n_pages, -1
    out, lse = torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 2, device="cuda")
    b.call(out=out, lse=lse)
    assert bool((out[1] == 0).all()) and bool(torch.isneginf(lse[1]).all())
    keep = torch.cat([torch.arange(64), torch.arange(128, 256)])
    x = (b.k[0][keep, 0] @ b.q[0].double().t()) / 8
    p = torch.softmax(x, 0)
    o = p.t() @ b.v[0][keep, 0]
    assert bool(((out[0].cpu().double() - o).abs() <= 2.0 ** -8 * (o.abs() + (p.t() @ b.v[0][keep, 0].abs()) + 8 * b.v[0].abs().max() / 7)).all())
    assert torch.allclose(lse[0].cpu().double(), torch.logsumexp(x, 0), atol=1e-4)


def test_lengths_above_the_table_count_as_its_room():
    b = Batch(kt.KT_KV_U4, 64, 1, 2, [128], seed=12)
    ref = b.call()
    many = torch.tensor([1 << 30], dtype=torch.int32, device="cuda")
    assert torch.equal(ref, kt.kt_paged_attention(b.q.cuda(), b.cache, b.pages, many))


def test_strided_queries_outputs_and_a_side_stream():
    b = Batch(kt.KT_KV_U4, 128, 2, 4, [300, 77, 1000], seed=13)
    ref = b.call()
    wide = torch.zeros(3, 2000, dtype=torch.bfloat16, device="cuda")
    wide[:, 8:8 + 1024] = b.q.reshape(3, -1).cuda()
    out = torch.full((3, 1100), 4.0, dtype=torch.bfloat16, device="cuda")
    ws, side = kt.Workspace(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.call(Q=wide[:, 8:8 + 1024].view(3, 8, 128), out=out[:, 4:4 + 1024].view(3, 8, 128), workspace=ws)
    side.synchronize()
    assert torch.equal(out[:, 4:1028].reshape(3, 8, 128), ref) and bool((out[:, :4] == 4).all()) and bool((out[:, 1028:] == 4).all())


def test_a_captured_call_follows_its_lengths_and_pages():
    b = Batch(kt.KT_KV_U8, 128, 2, 4, [700, 64, 1, 333], prefix=100, seed=14)
    lens = torch.tensor(b.lens, dtype=torch.int32, device="cuda")
    q, ws = b.q.cuda(), kt.Workspace()
    out = torch.zeros(4, 8, 128, dtype=torch.bfloat16, device="cuda")
    run = lambda o, w: kt.kt_paged_attention(q, b.cache, b.pages, lens, prefix_pages=b.prefix_pages, prefix_len=100, out=o, workspace=w)  # noqa: E731
    run(out, ws)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        run(out, ws)
    for step in range(4):
        lens.copy_(torch.tensor([700 - 90 * step, 64 - step, step, 333], dtype=torch.int32))
        q.mul_(-1)
        graph.replay()
        eager = torch.zeros_like(out)
        run(eager, None)
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), eager.view(torch.int16)), step     # (a token never written is NaN in both)
        _ = (q.float() ** 2).sum().item()


def test_a_rotated_model_decodes_like_the_plain_one():
    """Norm, append and attention together, token by token behind a prompt: Hadamard-rotated queries and keys give the unrotated
    attention (bf16 cache), and the chunk gives what the tokens gave."""
    g = torch.Generator().manual_seed(15)
    d, hq, hkv, hd, n = 512, 4, 2, 128, 90
    x = torch.randn(n, d, generator=g).to(torch.bfloat16).cuda()
    w = (torch.randn(d, (hq + 2 * hkv) * hd, generator=g) / d ** 0.5).cuda()
    rope = rope_table(256, hd).cuda()
    pages, pos = torch.tensor([[2, 0]], dtype=torch.int32).cuda(), torch.arange(n, dtype=torch.int32).cuda()
    slots = pages[0].long()[pos.long() // 64] * 64 + pos % 64

    def normed(rows):
        y = torch.empty(len(rows), d, dtype=torch.bfloat16, device="cuda")
        kt.kt_add_rmsnorm_quant(x[rows], format=kt.KT_Q_INT8, Y=y)
        return y

    every = torch.arange(n).cuda()
    assert torch.equal(normed(every), torch.cat([normed(every[:60])] + [normed(every[i:i + 1]) for i in range(60, n)]))
    projected = (normed(every).float() @ w).to(torch.bfloat16)     # once: a library product's bits depend on its number of rows

    def layer(cache, rows, had):
        q, k, v = projected[rows].split([hq * hd, hkv * hd, hkv * hd], 1)
        q = kt.kt_kv_append(cache, k, v, slots[rows].contiguous(), Q=q, positions=pos[rows].contiguous(), rope=rope, hadamard=had)
        lens = torch.tensor([int(rows[-1]) + 1], dtype=torch.int32, device="cuda")
        starts = torch.tensor([0, len(rows)], dtype=torch.int32, device="cuda")
        return kt.kt_paged_attention(q.view(-1, hq, hd), cache, pages, lens, q_starts=starts, max_q=len(rows))

    res = {}
    for had in (False, True):
        cache = kt.KVCache(3, 64, hkv, hd, kt.KT_KV_BF16)
        prompt = layer(cache, torch.arange(60).cuda(), had)
        res[had] = torch.cat([prompt] + [layer(cache, torch.arange(i, i + 1).cuda(), had) for i in range(60, n)]).float()
        again = kt.KVCache(3, 64, hkv, hd, kt.KT_KV_BF16)
        whole = layer(again, torch.arange(n).cuda(), had).float()
        assert float((whole - res[had]).norm() / whole.norm()) < 2.0 ** -7
        last = int(pos[-1]) + 1
        assert torch.equal(*(kt.kt_kv_gather(c, slots[:last].contiguous())[0] for c in (cache, again)))
    # rotated queries and keys are rounded to bf16 in another basis: scores move by about 2^-8 of |q| |k| / sqrt(hd) ~ 2^-8 sqrt(hd) / sqrt(hd)
    assert float((res[True] - res[False]).norm() / res[False].norm()) < 2.0 ** -5
