"""Linear attention of few sequences whose query heads share few key heads, up
to as many as there may be: sets of heads of every size that the blocks are
dealt out by. Tolerances as in test_gpu_linattn.py."""
import pytest

from paper_2509_26092_amd import binding as B
from gpu_util import PREC
from test_gpu_linattn import Case
from test_gpu_rows import ws_of

pytestmark = pytest.mark.gpu

PRECS = ["fp32", "bf16", "fp16"]


# (B, T, H, Hk, Dk, Dv, lengths)
SHARED = [(1, 300, 32, 1, 32, 24, None), (1, 45, 128, 1, 16, 72, None), (2, 100, 30, 2, 24, 40, [100, 63]),
          (1, 70, 31, 1, 16, 16, None), (3, 40, 45, 3, 20, 130, [0, 40, 1]), (1, 33, 64, 2, 130, 16, None),
          (1, 420, 12, 2, 64, 64, [401])]


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("i", range(len(SHARED)))
def test_heads_over_few_key_heads(prec, i):
    *sizes, lengths = SHARED[i]
    c = Case(prec, *sizes, lengths, True)
    c.check_fwd()
    c.check_bwd()


def test_all_heads_over_one_key_head():
    """2^20 query heads over one key head, one token, the widest rows: what the
    header admits, and nothing that a launch cannot take. Small integers, whose
    products and sums are exact."""
    import torch
    H, Dk, Dv, P = 1 << 20, 1, 256, PREC["bf16"]
    sizes = (1, 1, H, 1, Dk, Dv)
    small = lambda *s: torch.randint(-3, 4, s, device="cuda", dtype=torch.int8).to(torch.bfloat16)
    q, k, v, do, g = small(H, Dk), small(1, Dk), small(1, Dv), small(H, Dv), torch.zeros(H, device="cuda")
    o = torch.full_like(do, 7)
    k[:] = 2
    B.rn18op_linattn_fwd(P, q, k, v, g, None, None, o, None, *sizes, H * Dk, Dk, Dv, H * Dv, 1.0,
                         ws_of(B.rn18op_linattn_fwd_workspace(P, *sizes)))
    assert torch.equal(o, q * k * v)
    del o
    dq, dk, dv = (torch.full_like(x, 7) for x in (q, k, v))
    ws = ws_of(B.rn18op_linattn_bwd_workspace(P, *sizes))
    B.rn18op_linattn_bwd(P, q, k, v, do, g, None, None, None, dq, dk, dv, None, *sizes, H * Dk, Dk, Dv, H * Dv, H * Dk,
                         Dk, Dv, 1.0, ws)
    dots = torch.zeros((H, 1), dtype=torch.float64, device="cuda")
    sums = torch.zeros((1, Dv), dtype=torch.float64, device="cuda")
    for a in range(0, H, H // 8):
        part = do[a:a + H // 8].double()
        dots[a:a + H // 8] = (part * v.double()).sum(1, keepdim=True)
        sums += (part * q[a:a + H // 8].double()).sum(0, keepdim=True)
    assert torch.equal(dq, (dots * k.double()).to(torch.bfloat16))
    assert torch.equal(dk, (dots * q.double()).sum(0, keepdim=True).to(torch.bfloat16))
    assert torch.equal(dv, (sums * k.double()).to(torch.bfloat16))


@pytest.mark.parametrize("G", [4096, 1 << 17])
@pytest.mark.parametrize("q,do", [(1.1, 0.83), (0.7, 1.3)])
@pytest.mark.parametrize("D", [8, 5])
def test_equal_gradients_of_many_heads(G, q, do, D):
    """Heads that share a key head and give it equal gradients, whose roundings
    all go the same way: dk = G q (dO . v), dv = G dO (q . k), of terms of one
    sign. fp32: a term is off by (2 D + 4) 2^-24 at most, the sum by 2^-23."""
    import torch
    full = lambda *s: torch.full(s[:-1], float(s[-1]), device="cuda")
    sizes = (1, 1, G, 1, D, D)
    qd, kd, vd, dod = full(G, D, q), full(1, D, 0.9), full(1, D, 1.7), full(G, D, do)
    dq, dk, dv = torch.empty_like(qd), torch.empty_like(kd), torch.empty_like(vd)
    ws = ws_of(B.rn18op_linattn_bwd_workspace(PREC["fp32"], *sizes))
    B.rn18op_linattn_bwd(PREC["fp32"], qd, kd, vd, dod, torch.zeros(G, device="cuda"), None, None, None, dq, dk, dv, None,
                         *sizes, G * D, D, D, G * D, G * D, D, D, 1.0, ws)
    first = lambda t: t.double().flatten()[0].item()
    a, b, k, v = first(qd), first(dod), first(kd), first(vd)
    for got, ref in ((dk, G * a * D * b * v), (dv, G * b * D * a * k)):
        assert (got.double() - ref).abs().max().item() <= (2 * D + 6) * 2.0 ** -24 * ref
