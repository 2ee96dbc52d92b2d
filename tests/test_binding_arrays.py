"""Arrays that the binding refuses: types, sizes and places that the library
would misread or read beyond. Host tensors and a stand-in for the library;
nothing is launched."""
import types

import pytest

from paper_2509_26092_amd import binding as B


@pytest.fixture
def calls(monkeypatch):
    """The names of the library's functions that were called."""
    names = []

    class Lib:
        def __getattr__(self, name):
            return lambda *a: names.append(name) or 0

    monkeypatch.setattr(B, "_lib", Lib())
    monkeypatch.setattr(B, "_stream", lambda s=None: 0)
    return names


def refused(f, **kw):
    with pytest.raises(B.Rn18Error) as e:
        f(**kw)
    assert e.value.code == B.RN18_EINVAL, kw


def test_row_operators_refuse_other_types(calls):
    import torch
    R, C, K = 4, 9, 3
    z, v, i = torch.zeros(R, C), torch.zeros(R, K), torch.zeros(R, K, dtype=torch.int32)
    g, r, y = torch.zeros(C), torch.zeros(R), torch.zeros(R, dtype=torch.int32)
    half = torch.bfloat16

    def fwd(gamma=g, beta=g):
        return B.rn18op_layernorm_fwd(B.RN18_FP32, z, gamma, beta, z, r, r, R, C, C, C)

    def bwd(gamma=g, dgamma=g, dbeta=g):
        return B.rn18op_layernorm_bwd(B.RN18_FP32, z, z, gamma, r, r, z, dgamma, dbeta, R, C, C, C, C, r)

    def topk(vals=v, idx=i):
        return B.rn18op_topk_logits(B.RN18_FP32, z, vals, idx, R, C, C, K)

    def distill(t_vals=v, t_idx=i, labels=y, row_weight=r):
        return B.rn18op_distill_loss(B.RN18_FP32, z, t_vals, t_idx, labels, row_weight, z, r, r, R, C, C, C, K, 2.0, 0.5,
                                     1.0)

    bad = [(fwd, "gamma", g.to(half)), (fwd, "beta", g.double()), (bwd, "gamma", g.to(half)),
           (bwd, "dgamma", g.to(half)), (bwd, "dbeta", g.double()), (topk, "vals", v.to(half)),
           (topk, "idx", i.long()), (distill, "t_vals", v.to(half)), (distill, "t_vals", v.double()),
           (distill, "t_vals", v[:3]), (distill, "t_vals", torch.zeros(R, 2 * K)[:, ::2]),
           (distill, "t_idx", i.long()), (distill, "t_idx", i[:, :2]), (distill, "t_idx", i[:1].expand(R, K)),
           (distill, "labels", y.long()), (distill, "labels", y[:3]), (distill, "labels", y[:1].expand(R)),
           (distill, "row_weight", r.to(half)), (distill, "row_weight", r[:3])]
    for f, name, t in bad:
        refused(f, **{name: t})
    assert not calls
    for f, absent in ((fwd, ("gamma", "beta")), (bwd, ("gamma", "dgamma", "dbeta")), (topk, ()),
                      (distill, ("labels", "row_weight"))):
        assert f() == B.RN18_OK and f(**{name: None for name in absent}) == B.RN18_OK
    assert len(calls) == 8


def worker(classes=10):
    """A Worker's method without its context."""
    w = types.SimpleNamespace(ctx=None, _ensure=lambda N, H, W: None)
    w.step = lambda **kw: B.Worker.train_step_distill(w, **kw)
    return w


def test_worker_refuses_lists_of_another_batch_or_type(calls):
    import torch
    N, K = 4, 3
    v, i = torch.zeros(N, K), torch.zeros(N, K, dtype=torch.int32)
    y, st = torch.zeros(N, dtype=torch.int32), torch.zeros(8)
    good = dict(state=st, images=torch.zeros(N, 3, 16, 16), labels=y, t_vals=v, t_idx=i, temperature=2.0, alpha=0.5,
                lr=0.1)
    w = worker()
    for bad in (dict(t_idx=i.long()), dict(t_vals=v.double()), dict(t_vals=v.to(torch.bfloat16)), dict(t_vals=v[:3]),
                dict(t_idx=i[:3]), dict(t_idx=i[:, :2]), dict(t_vals=v[:, :2]), dict(t_vals=v[0]),
                dict(t_idx=i[:1].expand(N, K)), dict(t_vals=torch.zeros(K, N).t()), dict(labels=y.long()),
                dict(labels=y[:3]), dict(labels=y[:1].expand(N)), dict(labels=torch.zeros(N, 1, dtype=torch.int32)),
                dict(t_vals=v.to("meta")), dict(t_idx=i.to("meta")), dict(labels=y.to("meta"))):
        refused(w.step, **dict(good, **bad))
    assert not calls
    assert w.step(**good) == B.RN18_OK and w.step(**dict(good, labels=None, alpha=1.0)) == B.RN18_OK
    assert calls == ["rn18_train_step_distill"] * 2
