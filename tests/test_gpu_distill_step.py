"""GPU parity of the training step with a teacher (rn18_train_step_distill)
against the fp64 oracle's step, whose loss is replaced by the oracle's
distillation loss: the whole comparison of the plain step (loss, every
gradient, update and running statistic) at its tolerances."""
import numpy as np
import pytest

from oracle import net, rows
from paper_2509_26092_amd import binding as B
from paper_2509_26092_amd import inputs
from gpu_util import gpu_train_step, make_state
from test_gpu_step import LR, _run_parity

pytestmark = pytest.mark.gpu


def teacher(N, C, K, seed, short=False):
    """A teacher's list of K distinct classes a row, in no order; short: some
    entries left out, one row without any."""
    rng = np.random.default_rng(seed)
    idx = np.stack([rng.permutation(C)[:K] for _ in range(N)]).astype(np.int32)
    vals = (rng.standard_normal((N, K)) * 2.0).astype(np.float32)
    if short:
        idx[rng.random((N, K)) < 0.3] = -1
        vals[rng.random((N, K)) < 0.1] = -np.inf
        idx[N - 1] = -1
    return vals, idx


def step_with(vals, idx, temperature, alpha, labels="given"):
    """A Worker whose train_step is the one with this teacher; labels: those
    of the caller, or others (None too)."""
    import torch

    class Student(B.Worker):
        def train_step(self, state, images, y, lr, loss=None):
            lab = y if isinstance(labels, str) else None if labels is None else torch.from_numpy(labels).cuda()
            return self.train_step_distill(state, images, lab, torch.from_numpy(vals).cuda(),
                                           torch.from_numpy(idx).cuda(), temperature, alpha, lr, loss)

    return Student


@pytest.mark.parametrize("arch,classes,prec,N,H,K,T,alpha,short",
                         [("tiny", 10, "fp32", 8, 16, 4, 4.0, 0.9, False),
                          ("tiny", 10, "fp32", 5, 16, 10, 2.0, 0.5, True),
                          ("tiny", 70000, "fp32", 3, 16, 20, 2.0, 0.7, True),
                          ("cifar", 100, "fp32", 4, 32, 10, 4.0, 0.9, False),
                          ("tiny", 10, "fp16", 6, 16, 3, 3.0, 0.6, True),
                          ("tiny", 10, "bf16", 6, 16, 3, 1.5, 1.0, False),
                          ("imagenet", 1000, "bf16", 2, 64, 10, 4.0, 0.9, False)])
def test_step_parity(monkeypatch, arch, classes, prec, N, H, K, T, alpha, short):
    vals, idx = teacher(N, classes, K, N + classes, short)
    labels = inputs.labels(3, N, classes)
    if short:
        labels[0] = -1
    if alpha == 1.0:
        labels = None

    def loss(z, _):
        _, mean, dz = rows.distill(z, vals, idx, labels, None, T, alpha, 1.0 / N)
        return mean, dz

    monkeypatch.setattr(net.ops, "softmax_ce", loss)
    monkeypatch.setattr(B, "Worker", step_with(vals, idx, T, alpha, labels))
    _run_parity(arch, classes, prec, N, H, 310)


def test_step_parity_with_dropout(monkeypatch):
    N, C, K = 8, 10, 4
    vals, idx = teacher(N, C, K, 1)
    y = inputs.labels(3, N, C)

    def loss(z, _):
        _, mean, dz = rows.distill(z, vals, idx, y, None, 2.0, 0.5, 1.0 / N)
        return mean, dz

    monkeypatch.setattr(net.ops, "softmax_ce", loss)
    monkeypatch.setattr(B, "Worker", step_with(vals, idx, 2.0, 0.5, y))
    _run_parity("tiny", C, "fp32", N, 16, 311, dropout=(0.2, 7, 3))


@pytest.mark.parametrize("arch,classes,N,H", [("tiny", 10, 8, 16), ("cifar", 100, 16, 32)])
def test_a_teacher_without_weight_gives_the_plain_step(arch, classes, N, H):
    """alpha = 0: the label's cross-entropy alone. Both losses are fp32 sums
    of the same terms in different orders, 1e-5 of a tensor's largest."""
    L, st = make_state(arch, classes, 312)
    x, y = inputs.images(5, N, H, H), inputs.labels(5, N, classes)
    a, _, la, sa = gpu_train_step(arch, classes, "fp32", st, x, y, LR)
    w = step_with(*teacher(N, classes, 4, 2), 3.0, 0.0)(arch, classes, "fp32")
    b, _, lb, sb = gpu_train_step(arch, classes, "fp32", st, x, y, LR, worker=w)
    w.close()
    assert sa == sb == B.RN18_OK and abs(la[0] - lb[0]) <= 1e-5 * abs(la[0])
    for key in L.off:
        ta, tb = L.get(a, key), L.get(b, key)
        assert np.abs(ta - tb).max() <= 1e-5 * max(np.abs(ta).max(), 1e-3), key


def sticky(vals, idx, labels, alpha=0.5):
    N, C = len(idx), 10
    _, st = make_state("tiny", C, 313)
    w = step_with(vals, idx, 2.0, alpha, labels)("tiny", C, "fp32")
    status = gpu_train_step("tiny", C, "fp32", st, inputs.images(6, N, 16, 16), inputs.labels(6, N, C), 0.0,
                            worker=w)[3]
    w.close()
    return status


def test_bad_labels_classes_and_values_set_the_sticky_error():
    N = 4
    vals, idx = teacher(N, 10, 3, 4)
    y = inputs.labels(6, N, 10)
    assert sticky(vals, idx, y) == B.RN18_OK
    for bad, want in ((10, B.RN18_ELABEL), (-2, B.RN18_ELABEL), (-1, B.RN18_OK)):
        i, lab = idx.copy(), y.copy()
        i[2, 1] = lab[1] = bad
        assert sticky(vals, i, y) == want and sticky(vals, idx, lab) == want
    v = vals.copy()
    v[1, 1] = np.nan
    assert sticky(v, idx, y) == B.RN18_ENONFINITE


def test_host_side_errors():
    import torch
    w = B.Worker("tiny", 10, "fp32")
    st = torch.zeros(w.n_state, device="cuda")
    x = torch.zeros((2, 3, 16, 16), device="cuda")
    y = torch.zeros(2, dtype=torch.int32, device="cuda")
    v, i = torch.zeros((2, 3), device="cuda"), torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    good = dict(state=st, images=x, labels=y, t_vals=v, t_idx=i, K=3, temperature=2.0, alpha=0.5, N=2, H=16, W=16,
                lr=0.1)
    nan = float("nan")
    for bad in (dict(state=None), dict(images=None), dict(labels=None), dict(t_vals=None), dict(t_idx=None), dict(K=0),
                dict(K=257), dict(temperature=0.0), dict(temperature=nan), dict(alpha=-0.1), dict(alpha=1.5),
                dict(alpha=nan), dict(N=0), dict(lr=nan)):
        with pytest.raises(B.Rn18Error) as e:
            B.rn18_train_step_distill(w.ctx, **dict(good, **bad))
        assert e.value.code == B.RN18_EINVAL, bad
    assert w.sync_status() == B.RN18_OK
    w.close()
