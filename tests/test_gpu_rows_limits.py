"""The row operators at the limits of their arguments."""
import pytest

from paper_2509_26092_amd import binding as B
from test_gpu_rows import TOL, ws_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prec,D", [("bf16", 2 ** 27 + 13), ("fp32", 2 ** 27)])
def test_layernorm_bwd_of_the_widest_rows(prec, D):
    """The launch that joins the parameter gradients takes 32 columns a block
    of 1024: more than 2^27 columns pass what one launch may hold."""
    import torch
    R = 2
    dt = {"bf16": torch.bfloat16, "fp32": torch.float32}[prec]
    x = torch.randn((R, D), device="cuda", dtype=dt)
    dy = torch.randn((R, D), device="cuda", dtype=dt)
    m = x.double().mean(dim=1).float()
    rs = (1.0 / torch.sqrt(((x.double() - m.double()[:, None]) ** 2).mean(dim=1) + 1e-5)).float()
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    ws = ws_of(B.rn18op_layernorm_bwd_workspace(B.PREC_IDS[prec], R, D))
    B.rn18op_layernorm_bwd(B.PREC_IDS[prec], dy, x, None, m, rs, dx, dgamma, dbeta, R, D, D, D, D, ws)
    torch.cuda.synchronize()
    g = dy.double()
    xh = (x.double() - m.double()[:, None]) * rs.double()[:, None]
    assert bool(((dbeta.double() - g.sum(dim=0)).abs() <= TOL * 6).all())
    assert bool(((dgamma.double() - (g * xh).sum(dim=0)).abs() <= TOL * 36).all())
    xh *= (g * xh).sum(dim=1, keepdim=True) / D
    want = rs.double()[:, None] * (g - g.sum(dim=1, keepdim=True) / D - xh)
    assert bool(((dx.double() - want).abs() <= (2.0 ** -8 if prec == "bf16" else 0.0) * want.abs() + TOL * 7).all())
