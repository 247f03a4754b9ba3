"""The serving operators' calls: rows that are not finite, outputs and workspaces that the binding makes, streams, padded batches."""
import math

import pytest
import torch

import paper_2503_01483_amd as kt
from serving_util import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 1024, 8192])
def test_rows_without_codes_whose_sum_of_squares_is_not_finite(dt, d):
    """NaN as with codes, not zeros: finite rows beyond fp32's squares, infinities, NaN; the rows beside them as ever."""
    x = torch.randn(6, d, generator=torch.Generator().manual_seed(1))
    x[1] *= 3e37
    x[2, 5], x[3, d - 1], x[4, 0] = math.inf, -math.inf, math.nan
    y = torch.zeros(6, d, dtype=dt, device="cuda")
    kt.kt_add_rmsnorm_quant(x.to(dt).cuda(), format=kt.KT_Q_NONE, Y=y)
    y = y.cpu().double()
    assert bool(torch.isnan(y[1:5]).all())
    for row in (0, 5):
        h = x[row].to(dt).double()
        want = h / torch.sqrt(h.square().mean() + 1e-6)
        assert bool(((y[row] - want).abs() <= (torch.finfo(dt).eps / 2 + 23 * 2.0 ** -24) * want.abs()).all())


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_queries_of_a_padded_batch_are_zeros_where_nothing_was_written(dt):
    """New rows for the queries hold nothing of what the memory held before."""
    n, heads, hd = 300, 4, 128
    cache = kt.KVCache(8, 64, 2, hd, kt.KT_KV_U4)
    q, k, v = (torch.randn(n, h, hd, dtype=dt, device="cuda") for h in (heads, 2, 2))
    slots = torch.arange(n, device="cuda")
    slots[100:] = -1
    slots[50] = 8 * 64
    rope, pos = torch.ones(64, hd, device="cuda"), torch.arange(n, dtype=torch.int32, device="cuda")
    for more, written in ((dict(), [i for i in range(100) if i != 50]), (dict(rope=rope, positions=pos), [i for i in range(64) if i != 50])):
        for _ in range(3):
            torch.full_like(q, math.nan)            # (freed at once: the next tensor of this size lies there)
            out = kt.kt_kv_append(cache, k, v, slots, Q=q, **more)
            keep = torch.zeros(n, dtype=torch.bool, device="cuda")
            keep[written] = True
            assert bool((out[~keep] == 0).all()) and bool((out[keep] != 0).any(-1).all())


@pytest.mark.parametrize("fmt", [kt.KT_KV_BF16, kt.KT_KV_U8, kt.KT_KV_U4], ids=["bf16", "u8", "u4"])
@pytest.mark.parametrize("counts", [[3, 1, 2], [40, 0, 90]])
def test_all_rows_are_computed_without_a_bound_on_the_queries(fmt, counts):
    """q_starts without max_q: as if the bound were the number of rows; none is left out."""
    b = Batch(fmt, 128, 2, 4, [100, 64, 120], counts, seed=60)
    starts = torch.tensor(b.starts, dtype=torch.int32, device="cuda")
    lens = torch.tensor(b.lens, dtype=torch.int32, device="cuda")
    lse = torch.full((b.n, b.hq), 9.0, device="cuda")
    out = kt.kt_paged_attention(b.q.cuda(), b.cache, b.pages, lens, q_starts=starts, lse=lse)
    b.check(out, lse)


def _busy():
    """Keeps the current stream busy for some milliseconds."""
    a = torch.ones(4096, 4096, device="cuda")
    for _ in range(20):
        a = a @ a * 2.0 ** -12
    return a


@pytest.mark.parametrize("handle", [False, True], ids=["stream", "handle"])
def test_a_stream_handed_in_orders_what_the_call_makes_for_itself(handle):
    """Rows that the binding zeroes are zeroed in front of the kernel, on its stream, also while the current one is busy."""
    n, heads, hd = 200, 2, 128
    cache = kt.KVCache(4, 64, heads, hd, kt.KT_KV_U8)
    q, k, v = (torch.randn(n, h, hd, dtype=torch.bfloat16, device="cuda") for h in (4, heads, heads))
    slots = torch.arange(n, device="cuda")
    want_q = kt.kt_kv_append(cache, k, v, slots, Q=q, hadamard=True)
    want = kt.kt_kv_gather(cache, slots)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    stream = side.cuda_stream if handle else side
    for _ in range(3):
        a = _busy()
        K, V = kt.kt_kv_gather(cache, slots, stream=stream)
        qo = kt.kt_kv_append(cache, k, v, slots, Q=q, hadamard=True, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(K, want[0]) and torch.equal(V, want[1]) and torch.equal(qo, want_q)
        del a


def test_a_workspace_made_for_another_stream_stays_its_own(monkeypatch):
    """Attention on a stream that is handed in: outputs and scratch come from that stream's memory, so that nothing of the current stream takes it
    while the kernels run.  (Where tensors are made is looked at: nothing is run into a used workspace.)"""
    b = Batch(kt.KT_KV_U4, 128, 2, 4, [300, 200], [80, 70], seed=61)
    want = b.call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    made = []
    for name in ("empty", "zeros"):
        plain = getattr(torch, name)
        monkeypatch.setattr(torch, name, lambda *a, plain=plain, **kw: made.append(torch.cuda.current_stream().cuda_stream) or plain(*a, **kw))
    lens, starts = torch.tensor(b.lens, dtype=torch.int32).cuda(), torch.tensor(b.starts, dtype=torch.int32).cuda()
    q = b.q.cuda()
    torch.cuda.synchronize()
    out = kt.kt_paged_attention(q, b.cache, b.pages, lens, q_starts=starts, max_q=80, stream=side)
    assert len(made) == 2 and all(s == side.cuda_stream for s in made) and torch.cuda.current_stream() != side
    side.synchronize()
    assert torch.equal(out, want)
    # a workspace of the caller's grows there too
    ws = kt.Workspace()
    del made[:]
    assert torch.equal(kt.kt_paged_attention(q, b.cache, b.pages, lens, q_starts=starts, max_q=80, out=out, workspace=ws, stream=side.cuda_stream), out)
    side.synchronize()
    assert made == [side.cuda_stream] and torch.equal(out, want)


def test_other_calls_on_a_stream_that_is_handed_in():
    """The rotation's calls make their outputs and scratch on that stream too."""
    x, r = torch.randn(1, 700, 512, device="cuda").bfloat16(), torch.eye(512, device="cuda")[None]
    want, had = kt.kt_kurtosis_loss_grad(x, r), kt.kt_hadamard_rows(x[0])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream, torch.cuda.current_stream(), 0):
        a = _busy()
        loss, rows = kt.kt_kurtosis_loss_grad(x, r, stream=stream), kt.kt_hadamard_rows(x[0], stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(loss, want) and torch.equal(rows, had)
        del a
