"""The serving operators' calls: rows that are not finite, outputs and workspaces that the binding makes, streams, padded batches."""
import math

import pytest
import torch

import paper_2503_01483_amd as kt

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
