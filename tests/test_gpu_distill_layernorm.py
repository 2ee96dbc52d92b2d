"""The layer norm of the distillation example on rows of any layout."""
import numpy as np
import pytest

from oracle import rows
from gpu_util import assert_close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("r,d", [(1, 1), (1, 40), (7, 1), (6, 40)])
@pytest.mark.parametrize("layout", ["whole", "every second", "transposed", "slice", "expanded"])
def test_layouts(r, d, layout):
    """fp32, 1e-5 of the largest value as for the operators."""
    import torch
    from paper_2509_26092_amd import distill
    g = torch.Generator(device="cuda").manual_seed(r + d)

    def made():
        if layout == "transposed":
            return torch.randn((d, r), device="cuda", generator=g).t()
        if layout == "expanded":
            return torch.randn((1, d), device="cuda", generator=g).expand(r, d)
        wide = torch.randn((r, 2 * d + 3), device="cuda", generator=g)
        return {"whole": wide[:, :d].contiguous(), "every second": wide[:, :2 * d:2], "slice": wide[:, 3:3 + d]}[layout]

    x, dy = made(), made()
    x64, dy64 = x.cpu().double().numpy(), dy.cpu().double().numpy()
    n = distill.LayerNorm(d)
    n.gamma.normal_(1.0, 0.2, generator=g)
    n.beta.normal_(0.0, 0.2, generator=g)
    y = n.forward(x)
    dx = n.backward(dy)
    gamma = n.gamma.cpu().double().numpy()
    want, mean, rstd = rows.layernorm_forward(x64, gamma, n.beta.cpu().double().numpy(), distill.EPS)
    assert_close(y.cpu().double().numpy(), want, 1e-5, "y")
    want, dgamma, dbeta = rows.layernorm_backward(dy64, x64, gamma, mean, rstd)
    size = np.abs(rstd[:, None] * dy64 * gamma).max()
    assert np.abs(dx.cpu().double().numpy() - want).max() <= 1e-5 * size
    for got, w in ((n.dgamma, dgamma), (n.dbeta, dbeta)):
        assert np.abs(got.cpu().double().numpy() - w).max() <= 1e-5 * max(1.0, np.abs(w).max())
    assert np.array_equal(x.cpu().double().numpy(), x64)


def test_refusals():
    import torch
    from paper_2509_26092_amd import distill
    n = distill.LayerNorm(8)
    with pytest.raises(ValueError):
        n.forward(torch.zeros((2, 9), device="cuda"))
    n.forward(torch.zeros((2, 8), device="cuda"))
    for bad in (torch.zeros((3, 8), device="cuda"), torch.zeros((2, 8), device="cuda", dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            n.backward(bad)
