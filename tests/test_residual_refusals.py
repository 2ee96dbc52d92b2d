"""Arguments that dropout, RMS norm and linear attention refuse on the host,
before anything is launched (fake pointers, no GPU)."""
import ctypes
import os

import pytest

from paper_2509_26092_amd import binding as B

P = ctypes.c_void_p
A, A1, A2, A4 = P(1 << 20), P((1 << 20) + 1), P((1 << 20) + 2), P((1 << 20) + 4)
Q, W, Z = P(1 << 24), P(1 << 25), P(1 << 26)
NAN, INF, BIG = float("nan"), float("inf"), 1 << 46

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="library not built")


def drop(prec=B.RN18_BF16, x=A, res=None, y=Q, R=4, D=8, ldx=8, ldres=8, ldy=8, p=0.1, step_add=None):
    return B.lib().rn18op_dropout(prec, x, res, y, R, D, ldx, ldres, ldy, p, 1, 2, step_add, None)


def fwd(prec=B.RN18_BF16, x=A, res=None, gamma=None, h=Q, y=W, rstd=None, R=4, D=8, ldx=8, ldres=8, ldh=8, ldy=8,
        eps=1e-5, p=0.1, step_add=None):
    return B.lib().rn18op_rmsnorm_fwd(prec, x, res, gamma, h, y, rstd, R, D, ldx, ldres, ldh, ldy, eps, p, 1, 2,
                                      step_add, None)


def q8(prec=B.RN18_BF16, x=A, res=None, gamma=None, h=Q, y8=W, scale=Z, rstd=None, R=4, D=8, ldx=8, ldres=8, ldh=8,
       ldy8=8, eps=1e-5, p=0.1, step_add=None):
    return B.lib().rn18op_rmsnorm_fwd_q8(prec, x, res, gamma, h, y8, scale, rstd, R, D, ldx, ldres, ldh, ldy8, eps, p,
                                         1, 2, step_add, None)


def bwd(prec=B.RN18_BF16, dy=A, dr=None, h=A, gamma=None, rstd=A, dh=Q, dx=W, dgamma=A, R=4, D=8, lddy=8, lddr=8, ldh=8,
        lddh=8, lddx=8, p=0.1, step_add=None, ws=Z, ws_bytes=1 << 30):
    return B.lib().rn18op_rmsnorm_bwd(prec, dy, dr, h, gamma, rstd, dh, dx, dgamma, R, D, lddy, lddr, ldh, lddh, lddx,
                                      p, 1, 2, step_add, ws, ws_bytes, None)


def la(prec=B.RN18_BF16, q=A, k=A, v=A, g=A, lengths=None, s0=None, o=Q, sT=None, B_=2, T=4, H=2, Hk=1, Dk=8, Dv=4,
       ldq=16, ldk=8, ldv=4, ldo=8, scale=1.0, ws=Z, ws_bytes=1 << 40):
    return B.lib().rn18op_linattn_fwd(prec, q, k, v, g, lengths, s0, o, sT, B_, T, H, Hk, Dk, Dv, ldq, ldk, ldv, ldo,
                                      scale, ws, ws_bytes, None)


def lab(prec=B.RN18_BF16, q=A, k=A, v=A, do=A, g=A, lengths=None, s0=None, dsT=None, dq=Q, dk=W, dv=Z, ds0=None, B_=2,
        T=4, H=2, Hk=1, Dk=8, Dv=4, ldq=16, ldk=8, ldv=4, lddo=8, lddq=16, lddk=8, lddv=4, scale=1.0, ws=P(1 << 27),
        ws_bytes=1 << 40):
    return B.lib().rn18op_linattn_bwd(prec, q, k, v, do, g, lengths, s0, dsT, dq, dk, dv, ds0, B_, T, H, Hk, Dk, Dv,
                                      ldq, ldk, ldv, lddo, lddq, lddk, lddv, scale, ws, ws_bytes, None)


def step(prec=B.RN18_BF16, q=A, k=A, v=A, g=A, s=A, o=Q, new=W, B_=2, H=2, Hk=1, Dk=8, Dv=4, ldq=16, ldk=8, ldv=4,
         ldo=8, scale=1.0):
    return B.lib().rn18op_linattn_step(prec, q, k, v, g, s, o, new, B_, H, Hk, Dk, Dv, ldq, ldk, ldv, ldo, scale, None)


RATES = [dict(p=1.0), dict(p=-0.1), dict(p=NAN), dict(p=INF), dict(step_add=A4)]
HEADS = [dict(prec=3), dict(H=0), dict(Hk=0), dict(H=3, Hk=2), dict(Dk=0), dict(Dv=0), dict(Dk=257),
         dict(Dv=257), dict(B_=-1), dict(ldq=15), dict(ldk=7), dict(ldv=3), dict(q=None),
         dict(k=None), dict(v=None), dict(g=None), dict(q=A1), dict(k=A1), dict(v=A1), dict(g=A2), dict(scale=NAN),
         dict(scale=INF), dict(ldq=BIG), dict(B_=1 << 20)]
CASES = [(drop, c) for c in RATES + [dict(prec=3), dict(R=-1), dict(D=0), dict(ldx=7), dict(ldy=7), dict(x=None),
                                     dict(y=None), dict(x=A1), dict(y=A1), dict(res=A1), dict(res=Z, ldres=7),
                                     dict(y=A, ldy=9), dict(res=Q, ldres=9), dict(ldx=BIG), dict(D=(1 << 30) + 1)]]
CASES += [(fwd, c) for c in RATES + [dict(prec=-1), dict(R=-1), dict(D=0), dict(ldx=7), dict(ldh=7), dict(ldy=7),
                                     dict(x=None), dict(y=None), dict(h=None), dict(h=None, p=0.0, res=A), dict(h=W),
                                     dict(gamma=A2), dict(rstd=A1), dict(eps=-1.0), dict(eps=NAN), dict(eps=INF),
                                     dict(h=A, ldh=9), dict(y=A, ldy=9), dict(res=Q, ldres=9), dict(ldy=BIG)]]
CASES += [(q8, c) for c in RATES + [dict(prec=-1), dict(ldy8=7), dict(y8=None), dict(scale=None), dict(scale=A2),
                                    dict(y8=A), dict(y8=Q), dict(y8=Z, res=Z), dict(h=None), dict(ldy8=BIG),
                                    dict(x=A1), dict(eps=-1.0), dict(R=-2), dict(D=0)]]
CASES += [(bwd, c) for c in RATES + [dict(prec=4), dict(R=-1), dict(D=0), dict(lddy=7), dict(ldh=7), dict(lddh=7),
                                     dict(lddx=7), dict(dr=Z, lddr=7), dict(dy=None), dict(h=None), dict(rstd=None),
                                     dict(dh=None, dx=None), dict(dh=Q, dx=Q), dict(dgamma=A2), dict(gamma=A1),
                                     dict(dh=A, lddh=9), dict(dx=A, lddx=9), dict(dr=Q, lddr=9), dict(ws=A4),
                                     dict(ws=None), dict(dy=A1), dict(dh=A1)]]
CASES += [(la, c) for c in HEADS + [dict(o=None), dict(ldo=7), dict(o=A), dict(o=A1), dict(T=-1), dict(T=(1 << 26) + 1),
                                    dict(lengths=A2), dict(s0=A2), dict(sT=A1), dict(B_=1 << 18, T=1 << 13)]]
CASES += [(lab, c) for c in HEADS + [dict(do=None), dict(dq=None), dict(dk=None), dict(dv=None), dict(lddo=7),
                                     dict(lddq=15), dict(lddk=7), dict(lddv=3), dict(dq=A), dict(dk=A), dict(dv=A),
                                     dict(dq=W), dict(dk=Z), dict(dsT=A2), dict(ds0=A1), dict(s0=P(64), ds0=P(64)),
                                     dict(T=-1), dict(lengths=A1)]]
CASES += [(step, c) for c in HEADS + [dict(o=None), dict(ldo=7), dict(o=A), dict(s=None), dict(new=None), dict(s=A2),
                                      dict(new=A1)]]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_refused_on_the_host(i):
    f, kw = CASES[i]
    assert f(**kw) == B.RN18_EINVAL, (f.__name__, kw)
    assert B.rn18_last_error()


def test_workspaces_too_small_or_missing_are_refused():
    assert B.rn18op_rmsnorm_bwd_workspace(B.RN18_BF16, 5, 0) == 0
    assert B.rn18op_linattn_fwd_workspace(B.RN18_BF16, 1, 5, 3, 2, 8, 8) == 0
    assert B.rn18op_linattn_bwd_workspace(B.RN18_BF16, 1, 5, 2, 2, 8, 300) == 0
    n = B.rn18op_rmsnorm_bwd_workspace(B.RN18_BF16, 5000, 64)
    assert n and bwd(R=5000, D=64, lddy=64, ldh=64, lddh=64, lddx=64, ws_bytes=n - 1) == B.RN18_ENOMEM
    for T in (4, 5000):
        kw = dict(T=T, Dk=64, Dv=64, ldq=128, ldk=64, ldv=64)
        n = B.rn18op_linattn_bwd_workspace(B.RN18_BF16, 2, T, 2, 1, 64, 64)
        assert n and lab(lddo=128, lddq=128, lddk=64, lddv=64, ws_bytes=n - 1, **kw) == B.RN18_ENOMEM
        assert lab(lddo=128, lddq=128, lddk=64, lddv=64, ws=None, **kw) == B.RN18_EINVAL
        n = B.rn18op_linattn_fwd_workspace(B.RN18_BF16, 2, T, 2, 1, 64, 64)
        if n:
            assert la(ldo=128, ws_bytes=n - 1, **kw) == B.RN18_ENOMEM
            assert la(ldo=128, ws=A4, **kw) == B.RN18_EINVAL


def test_the_binding_refuses_arrays_of_other_types_and_sizes():
    import torch
    f32, i64 = torch.zeros(8), torch.zeros(8, dtype=torch.int64)
    x = torch.zeros((4, 8), dtype=torch.bfloat16)
    for bad in (dict(gamma=torch.zeros(7)), dict(gamma=torch.zeros(8).half()), dict(rstd=torch.zeros(3)),
                dict(step_add=torch.zeros(1, dtype=torch.int32))):
        kw = dict(gamma=f32, rstd=torch.zeros(4), step_add=None)
        kw.update(bad)
        with pytest.raises(B.Rn18Error):
            B.rn18op_rmsnorm_fwd(B.RN18_BF16, x, None, kw["gamma"], x, x, kw["rstd"], 4, 8, 8, 8, 8, 8,
                                 step_add=kw["step_add"], stream=None)
    for bad in (dict(g=torch.zeros(1)), dict(g=i64), dict(lengths=i64), dict(lengths=torch.zeros(1, dtype=torch.int32)),
                dict(s0=torch.zeros(127)), dict(sT=torch.zeros(128).half())):
        kw = dict(g=torch.zeros(2), lengths=None, s0=None, sT=None)
        kw.update(bad)
        with pytest.raises(B.Rn18Error):
            B.rn18op_linattn_fwd(B.RN18_BF16, x, x, x, kw["g"], kw["lengths"], kw["s0"], x, kw["sT"], 2, 4, 2, 1, 8, 4,
                                 16, 8, 4, 8, 1.0)


def test_the_student_refuses_dropout_that_nothing_would_take():
    from paper_2509_26092_amd import distill
    with pytest.raises(ValueError, match="without residual blocks"):
        distill.TokenStudent(20, dropout=0.1)
    for kw in ({"blocks": 1}, {"dropout": 0.1}):
        with pytest.raises(ValueError, match="token student"):
            distill.run("resnet", **kw)
