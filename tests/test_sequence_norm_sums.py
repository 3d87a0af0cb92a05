"""The sums over the rows that the layer norm's gradient gives for its weight and bias, against the bound that follows from how the rows are split."""
import math

import pytest
import torch

from paper_2211_10280_amd import binding as B
from test_sequence_operators import DT, U32, _bytes, _gen, _near

pytestmark = pytest.mark.gpu


def _additions(n, D):
    """Additions in fp32 on the way to a column's sum: the rows of a group of lanes, one after the other, then a workgroup's groups; the workgroups' shares are added in 64 bits."""
    lanes = 8 if D <= 32 else 16 if D <= 320 else 32 if D <= 640 else 64
    groups = 256 // lanes
    return min(256, max(1, math.ceil(n / (groups * 1_536)))) + groups


@pytest.mark.parametrize("n,D,dtype", [(3, 4, "f32"), (40_001, 8, "bf16"), (60_011, 32, "f32"), (60_011, 36, "f32"), (30_007, 300, "f32"), (50_021, 320, "bf16"), (9_001, 324, "f32"), (20_011, 640, "bf16"),
                                       (7_001, 644, "f32"), (12_301, 1_024, "bf16"), (1_700_003, 12, "f32")])
def test_sums_for_weight_and_bias(n, D, dtype):
    g = _gen(n + D)
    x, d = ((torch.randn((n, D), generator=g, device="cuda") + 0.3).to(DT[dtype]) for _ in range(2))
    mean, rstd, dw, db = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    B.tensair_norm(x, D, None, None, torch.empty_like(x), mean, rstd)
    B.tensair_norm_grad(d, x, D, None, mean, rstd, torch.empty_like(x), dw, db, _bytes(B.tensair_norm_workspace_bytes(n, D)))
    y, d = (x.double() - mean.double()[:, None]) * rstd.double()[:, None], d.double()
    k = _additions(n, D)
    # a term is off by 3 (difference, two products), a sum once more at the end
    _near(dw, (d * y).sum(0), (k + 4) * U32 * (d * y).abs().sum(0) + 1e-30, "d_weight")
    _near(db, d.sum(0), (k + 1) * U32 * d.abs().sum(0) + 1e-30, "d_bias")
