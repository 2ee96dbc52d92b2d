"""Arguments that the row operators refuse on the host, before anything is
launched (fake pointers, no GPU)."""
import ctypes
import os

import pytest

from paper_2509_26092_amd import binding as B

P = ctypes.c_void_p
A, A1, A2 = P(1 << 20), P((1 << 20) + 1), P((1 << 20) + 2)
Q = P(1 << 24)
NAN, INF = float("nan"), float("inf")

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="library not built")


def fwd(prec=B.RN18_BF16, x=A, gamma=None, beta=None, y=Q, mean=None, rstd=None, R=4, D=8, ldx=8, ldy=8, eps=1e-5):
    return B.lib().rn18op_layernorm_fwd(prec, x, gamma, beta, y, mean, rstd, R, D, ldx, ldy, eps, None)


def bwd(prec=B.RN18_BF16, dy=A, x=A, gamma=None, mean=A, rstd=A, dx=Q, dgamma=A, dbeta=A, R=4, D=8, lddy=8, ldx=8,
        lddx=8, ws=A, ws_bytes=1 << 30):
    return B.lib().rn18op_layernorm_bwd(prec, dy, x, gamma, mean, rstd, dx, dgamma, dbeta, R, D, lddy, ldx, lddx, ws,
                                        ws_bytes, None)


def topk(prec=B.RN18_BF16, z=A, vals=A, idx=A, R=4, C=8, ldz=8, K=2, ws=A, ws_bytes=1 << 30):
    return B.lib().rn18op_topk_logits(prec, z, vals, idx, R, C, ldz, K, ws, ws_bytes, None)


def distill(prec=B.RN18_BF16, z=A, t_vals=A, t_idx=A, labels=None, weight=None, dz=Q, row_loss=A, loss=None, R=4, C=8,
            ldz=8, lddz=8, K=2, temperature=2.0, alpha=0.5, scale=1.0, ws=A, ws_bytes=1 << 30):
    return B.lib().rn18op_distill_loss(prec, z, t_vals, t_idx, labels, weight, dz, row_loss, loss, R, C, ldz, lddz, K,
                                       temperature, alpha, scale, ws, ws_bytes, None)


BIG = 1 << 46

CASES = [
    (fwd, dict(prec=3)), (fwd, dict(R=-1)), (fwd, dict(D=0)), (fwd, dict(ldx=7)), (fwd, dict(ldy=7)),
    (fwd, dict(x=None)), (fwd, dict(y=None)), (fwd, dict(x=A1)), (fwd, dict(y=A1)),
    (fwd, dict(prec=B.RN18_FP32, x=A2)), (fwd, dict(gamma=A2)), (fwd, dict(beta=A1)), (fwd, dict(mean=A2)),
    (fwd, dict(rstd=A2)), (fwd, dict(eps=-1.0)), (fwd, dict(eps=NAN)), (fwd, dict(eps=INF)),
    (fwd, dict(R=BIG, ldx=BIG, ldy=BIG)), (fwd, dict(ldx=BIG)), (fwd, dict(y=A, ldy=9)),
    (bwd, dict(prec=-1)), (bwd, dict(R=-1)), (bwd, dict(D=-5)), (bwd, dict(lddy=7)), (bwd, dict(ldx=7)),
    (bwd, dict(lddx=7)), (bwd, dict(dy=None)), (bwd, dict(x=None)), (bwd, dict(dx=None)), (bwd, dict(mean=None)),
    (bwd, dict(rstd=None)), (bwd, dict(dy=A1)), (bwd, dict(x=A1)), (bwd, dict(dx=A1)), (bwd, dict(dgamma=A2)),
    (bwd, dict(dbeta=A2)), (bwd, dict(dx=A, lddx=9)), (bwd, dict(lddy=BIG)),
    (topk, dict(prec=9)), (topk, dict(R=-1)), (topk, dict(C=0)), (topk, dict(K=0)), (topk, dict(K=9)),
    (topk, dict(C=1000, ldz=1000, K=257)), (topk, dict(ldz=7)), (topk, dict(z=None)), (topk, dict(vals=None)),
    (topk, dict(idx=None)), (topk, dict(z=A1)), (topk, dict(vals=A2)), (topk, dict(idx=A2)), (topk, dict(ldz=BIG)),
    (distill, dict(prec=7)), (distill, dict(R=-1)), (distill, dict(C=0)), (distill, dict(K=-1)),
    (distill, dict(K=257)), (distill, dict(ldz=7)), (distill, dict(lddz=7)), (distill, dict(z=None)),
    (distill, dict(t_vals=None)), (distill, dict(t_idx=None)), (distill, dict(row_loss=None)), (distill, dict(z=A1)),
    (distill, dict(dz=A1)), (distill, dict(t_vals=A2)), (distill, dict(t_idx=A2)), (distill, dict(labels=A2)),
    (distill, dict(weight=A2)), (distill, dict(row_loss=A2)), (distill, dict(loss=A2)), (distill, dict(dz=A, lddz=9)),
    (distill, dict(temperature=0.0)), (distill, dict(temperature=-1.0)), (distill, dict(temperature=NAN)),
    (distill, dict(temperature=INF)), (distill, dict(temperature=1e-45)), (distill, dict(alpha=-0.1)),
    (distill, dict(alpha=1.1)), (distill, dict(alpha=NAN)), (distill, dict(scale=INF)), (distill, dict(scale=NAN)),
    (distill, dict(ldz=BIG)),
]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_refused_on_the_host(i):
    f, kw = CASES[i]
    assert f(**kw) == B.RN18_EINVAL, (f.__name__, kw)
    assert B.rn18_last_error()


def test_workspace_sizes_of_bad_shapes_are_zero():
    assert B.rn18op_layernorm_bwd_workspace(B.RN18_FP32, 4, 0) == 0
    assert B.rn18op_topk_logits_workspace(B.RN18_FP32, 4, 8, 9) == 0
    assert B.rn18op_distill_loss_workspace(5, 4, 8, 2) == 0


@pytest.mark.parametrize("f,need,kw", [
    (bwd, lambda R, W: B.rn18op_layernorm_bwd_workspace(B.RN18_BF16, R, W), lambda R, W: dict(D=W, lddy=W, ldx=W, lddx=W)),
    (topk, lambda R, W: B.rn18op_topk_logits_workspace(B.RN18_BF16, R, W, 2), lambda R, W: dict(C=W, ldz=W)),
    (distill, lambda R, W: B.rn18op_distill_loss_workspace(B.RN18_BF16, R, W, 2), lambda R, W: dict(C=W, ldz=W, lddz=W)),
])
@pytest.mark.parametrize("R,W", [(5000, 64), (3, 40000), (1, 131072)])
def test_workspaces_too_small_or_missing_are_refused(f, need, kw, R, W):
    n = need(R, W)
    if n == 0:
        return
    assert f(R=R, ws=A, ws_bytes=n - 1, **kw(R, W)) == B.RN18_ENOMEM
    assert f(R=R, ws=None, ws_bytes=n, **kw(R, W)) == B.RN18_EINVAL
    assert f(R=R, ws=P((1 << 20) + 4), ws_bytes=n, **kw(R, W)) == B.RN18_EINVAL


@pytest.mark.parametrize("W", [2 ** 30 + 1, 2 ** 31 - 1])
def test_rows_of_more_than_2_30_elements_are_refused(W):
    """A lane's position past the last chunk would pass 2^31 in the kernels."""
    big = (1 << 62)
    assert fwd(R=1, D=W, ldx=W, ldy=W) == B.RN18_EINVAL
    assert bwd(R=1, D=W, lddy=W, ldx=W, lddx=W, ws_bytes=big) == B.RN18_EINVAL
    assert topk(R=1, C=W, ldz=W, ws_bytes=big) == B.RN18_EINVAL
    assert distill(R=1, C=W, ldz=W, lddz=W, ws_bytes=big) == B.RN18_EINVAL
    assert B.rn18op_layernorm_bwd_workspace(B.RN18_BF16, 1, W) == 0
    assert B.rn18op_topk_logits_workspace(B.RN18_BF16, 1, W, 4) == 0
    assert B.rn18op_distill_loss_workspace(B.RN18_BF16, 1, W, 4) == 0
