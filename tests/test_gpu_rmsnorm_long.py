"""RMS norm of rows so long that a thread adds up thousands of elements, and of
so many long rows that a column does: equal elements, whose roundings all go
the same way. Against closed forms in 64 bits, with the tolerances of
test_gpu_rmsnorm.py: F bounds a row's sum, a column's too."""
import numpy as np
import pytest

from paper_2509_26092_amd import binding as B
from gpu_util import PREC, rounded, torch_dtype
from test_gpu_rmsnorm import EPS, F, PRECS, TINY, U
from test_gpu_rows import empty, ws_of

pytestmark = pytest.mark.gpu


def within(t, ref, bound):
    d = (t.double() - ref).abs().max().item()
    assert d <= bound, (d, bound)


def value(x, prec):
    return float(rounded(np.array([x], np.float32), prec)[0])


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("x", [1.1, 0.83, -1.7])
@pytest.mark.parametrize("D", [(1 << 20) + 3, (1 << 22) + 5, 1 << 24])
def test_a_long_row_of_equal_elements(prec, x, D):
    import torch
    P, v = PREC[prec], value(x, prec)
    h = torch.full((2, D), v, dtype=torch_dtype(prec), device="cuda")
    y, rstd = torch.empty_like(h), empty(2)
    B.rn18op_rmsnorm_fwd(P, h, None, None, None, y, rstd, 2, D, D, 0, 0, D, EPS)
    rs = 1 / np.sqrt(v * v + EPS)
    within(rstd, rs, F * rs)
    within(y, v * rs, (U[prec] + F) * abs(v) * rs + TINY[prec])
    y8, scale = torch.empty((2, D), dtype=torch.uint8, device="cuda"), empty(2)
    B.rn18op_rmsnorm_fwd_q8(P, h, None, None, None, y8, scale, rstd, 2, D, D, 0, 0, D, EPS)
    within(scale, abs(v) * rs / 448, F * abs(v) * rs / 448)
    # dy = 2 in the first half and 1 in the other: dh = rs (dy - xh^2 mean(dy))
    n = D // 2
    dy = torch.ones_like(h)
    dy[:, :n] = 2
    dh, rs32 = torch.empty_like(h), float(np.float32(rs))
    rstd.fill_(rs32)
    B.rn18op_rmsnorm_bwd(P, dy, None, h, None, rstd, dh, None, None, 2, D, D, 0, D, D, 0)
    mean = (D + n) / D * v * rs32
    for part, g in ((dh[:, :n], 2.0), (dh[:, n:], 1.0)):
        ref = rs32 * (g - v * rs32 * mean)
        within(part, ref, U[prec] * abs(ref) + F * rs32 * (g + abs(v * rs32 * mean)) + TINY[prec])


@pytest.mark.parametrize("prec", PRECS)
def test_many_long_rows_of_equal_elements(prec):
    import torch
    R, D, P, v, d, rs = 4000, (1 << 19) + 5, PREC[prec], value(1.1, prec), value(0.83, prec), 0.75
    h = torch.full((R, D), v, dtype=torch_dtype(prec), device="cuda")
    dy = torch.full_like(h, d)
    rstd, dgamma = torch.full((R,), rs, device="cuda"), empty(D)
    B.rn18op_rmsnorm_bwd(P, dy, None, h, None, rstd, dy, None, dgamma, R, D, D, 0, D, D, 0,
                         ws=ws_of(B.rn18op_rmsnorm_bwd_workspace(P, R, D)))
    within(dgamma, R * d * v * rs, F * R * d * v * rs)
