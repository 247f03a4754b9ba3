"""kt_add_rmsnorm_quant: codes bit for bit against elementary fp32 operations, scales and normed rows against fp64."""
import math

import pytest
import torch

import paper_2503_01483_amd as kt
import serving_util as su

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def _inputs(n, d, dt, seed, pad=0):
    g = torch.Generator().manual_seed(seed)
    wide = torch.exp(0.5 * torch.randn(d, generator=g))
    make = lambda s: (torch.randn(n, d + pad, generator=g) * s).to(dt)  # noqa: E731
    return make(1.0), make(2.0), ((1 + 0.2 * torch.randn(d, generator=g)) * wide)


def _check(x, res, gain, fmt, h_out, y, codes, scales, eps, clip):
    n, d = x.shape
    h, code, t, scale = su.norm(x, res, gain, eps, clip, fmt)
    if h_out is not None:
        assert torch.equal(h_out.cpu(), h.to(x.dtype))
    # the sum of squares: at most 3 roundings a term and log2 of its terms on the way up; then mean, eps, root, reciprocal, product
    rel = (3 + 15 + 5) * 2.0 ** -24
    half = torch.finfo(x.dtype).eps / 2
    if fmt == kt.KT_Q_NONE:
        assert bool(((y.cpu().double() - scale).abs() <= (half + rel) * scale.abs() + 1e-37).all())
        return
    if codes is not None:
        assert torch.equal(codes.cpu().float(), code)
    if scales is not None:
        assert bool(((scales.cpu().double() - scale[:, 0]).abs() <= rel * scale[:, 0]).all())
    if y is not None:
        v = code.double() * scale
        assert bool(((y.cpu().double() - v).abs() <= (half + rel + 2.0 ** -24) * v.abs()).all())


@pytest.mark.parametrize("fmt", [kt.KT_Q_NONE, kt.KT_Q_INT4, kt.KT_Q_INT8, kt.KT_Q_E4M3])
@pytest.mark.parametrize("dt", [BF, F], ids=["bf16", "f32"])
@pytest.mark.parametrize("n,d", [(1, 8), (5, 64), (1, 512), (3, 520), (2, 2048), (7, 2056), (3, 4096), (2, 4104), (2, 8192), (3, 8200), (2, 16384), (1, 16392), (2, 32768)])
def test_codes_scales_and_rows(n, d, dt, fmt):
    x, res, gain = _inputs(n, d, dt, seed=n + d)
    for g_dt in (None, BF, F):
        gain_t = None if g_dt is None else gain.to(g_dt)
        for r in (None, res):
            out = [torch.full((n, d), 7.0, dtype=dt, device="cuda") for _ in range(2)]
            codes = None if fmt == kt.KT_Q_NONE else torch.empty(n, d, dtype=torch.float8_e4m3fn if fmt == kt.KT_Q_E4M3 else torch.int8, device="cuda")
            scales = None if codes is None else torch.empty(n, device="cuda")
            kt.kt_add_rmsnorm_quant(x.cuda(), res=None if r is None else r.cuda(), gain=None if gain_t is None else gain_t.cuda(), eps=1e-5,
                                    clip_ratio=0.98, format=fmt, res_out=out[0], Y=out[1], codes=codes, scales=scales)
            _check(x, r, gain_t, fmt, out[0], out[1], codes, scales, 1e-5, 0.98)


def test_many_rows_strided_and_in_place():
    n, d = 1000, 1032
    x, res, gain = _inputs(n, d, BF, 3, pad=8)
    xd, rd = x.cuda(), res.cuda()
    codes = torch.full((n, d + 24), 99, dtype=torch.int8, device="cuda")
    scales = torch.empty(n, device="cuda")
    gain = gain.to(BF)
    kt.kt_add_rmsnorm_quant(xd[:, :d], res=rd[:, :d], gain=gain.cuda(), clip_ratio=1.0, format=kt.KT_Q_INT8, res_out=rd[:, :d], Y=xd[:, :d],
                            codes=codes[:, :d], scales=scales)
    _check(x[:, :d], res[:, :d], gain, kt.KT_Q_INT8, rd[:, :d], xd[:, :d], codes[:, :d], scales, 1e-6, 1.0)
    assert bool((codes[:, d:] == 99).all())                                  # what lies between the rows is left as it was
    assert torch.equal(xd[:, d:].cpu(), x[:, d:]) and torch.equal(rd[:, d:].cpu(), res[:, d:])


@pytest.mark.parametrize("fmt", [kt.KT_Q_INT4, kt.KT_Q_INT8, kt.KT_Q_E4M3])
def test_rows_of_zeros_tiny_values_and_what_is_not_finite(fmt):
    d = 1024
    x = torch.randn(9, d, generator=torch.Generator().manual_seed(1))
    x[1] = 0.0
    x[2] = 1e-38 * x[2].sign()
    x[3, 5], x[4, 900], x[5, 0] = math.nan, math.inf, -math.inf
    x[6] *= 3e37                                                            # its sum of squares is beyond fp32
    gain = torch.ones(d)
    codes = torch.empty(9, d, dtype=torch.float8_e4m3fn if fmt == kt.KT_Q_E4M3 else torch.int8, device="cuda")
    scales, y = torch.empty(9, device="cuda"), torch.empty(9, d, device="cuda")
    kt.kt_add_rmsnorm_quant(x.cuda(), gain=gain.cuda(), format=fmt, codes=codes, scales=scales, Y=y)
    s, c = scales.cpu(), codes.cpu().float()
    assert s[1] == 0 and s[2] == 0 and bool((c[1:3] == 0).all()) and bool((y[1:3] == 0).all())
    assert bool(torch.isnan(s[3:7]).all()) and bool((c[3:7] == 0).all()) and bool(torch.isnan(y[3:7]).all())
    for row in (0, 7, 8):
        _check(x[row:row + 1], None, gain, fmt, None, y[row:row + 1], codes[row:row + 1], scales[row:row + 1], 1e-6, 1.0)
    gain[17] = math.nan
    kt.kt_add_rmsnorm_quant(x.cuda(), gain=gain.cuda(), format=fmt, codes=codes, scales=scales)
    assert bool(torch.isnan(scales[[0, 3, 7, 8]]).all()) and bool((codes.float()[[0, 7, 8]] == 0).all())
