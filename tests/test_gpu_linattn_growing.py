"""Linear attention's heads that grow, g above 0, beyond what one factor of a
chunk or a segment holds in fp32: a state of zeros stays zeros, and one of
small values is right as long as it and the results are in fp32's range.

Tolerances are those of test_gpu_linattn.py and, for the powers, 4 roundings
(the decay's logarithm in base 2, its product with the tokens, the power, the
state's product with it) of 2^-24 for each unit of the sequence's whole growth
L = g times the tokens that a nonzero state passes. Below fp32's normal
numbers 1e-37."""
import numpy as np
import pytest

from oracle import linattn
from paper_2509_26092_amd import binding as B
from gpu_util import PREC, rounded
from test_gpu_linattn import Case, acc, near_stored
from test_gpu_rmsnorm import U, near
from test_gpu_rows import f64, mat, out, vec

pytestmark = pytest.mark.gpu

PRECS = ["fp32", "bf16", "fp16"]
L = {"fp32": 130.0, "bf16": 130.0, "fp16": 80.0}          # of a head's whole growth
SIZE = {"fp32": 1e-12, "bf16": 1e-12, "fp16": 1e-3}        # of k and v, or of q and dO
SCALE = {"fp32": 0.37, "bf16": 0.37, "fp16": 2.0 ** -90}   # fp16: results in its range


class Growing(Case):
    """Heads of decays g whose k and v are zeros up to the last tokens, and
    whose q and dO (`back`) are zeros from the first ones on, so that a nonzero
    state or gradient of one grows by exp(L) at most."""

    def __init__(self, prec, T, length, g, D, back, state):
        H = len(g)
        super().__init__(prec, 1, T, H, H, D, D, [length], False)
        self.g = np.array(g, np.float32)
        self.gd = vec(self.g)
        self.scale = SCALE[prec]
        for h in range(H):
            n = max(1, min(length, int(L[prec] / g[h])))
            for name in ("k", "v"):
                a = self.np[name][0, :length, h]
                a[:length - n] = 0
                a[length - n:] *= SIZE[prec]
            if back:
                for name in ("q", "do"):
                    a = self.np[name][0, :length, h]
                    a[n:] = 0
                    a[:n] *= SIZE[prec]
        for name, a in self.np.items():
            a[:, :length] = rounded(a[:, :length], prec)
            self.dev[name] = mat(a.reshape(T, -1), prec)[0]
        if state:
            self.s0 = np.zeros((1, H, D, D), np.float32)
            self.dsT = np.zeros((1, H, D, D), np.float32)

    def check(self, back, limit=True):
        """limit False: what is not finite need not be right."""
        prec, on, a = self.prec, self.inside(), self.np
        lens = on.sum(axis=1)
        tol = acc(prec, self.sizes[1]) + 4 * L[prec] * 2.0 ** -24
        names = ("q", "k", "v", "do") if back else ("q", "k", "v")
        zeros = lambda s, f: None if s is None else f(s)
        if back:
            outs, last = self.bwd()
            got = [self.rows(outs[n][0], self.sizes[4]) for n in ("dq", "dk", "dv")]
            ref, size = (linattn.backward(*[f(a[n]) for n in names], self.g, lens, zeros(self.s0, f),
                                          zeros(self.dsT, f), self.scale) for f in (np.array, np.abs))
        else:
            o, _, last = self.fwd()
            got = [self.rows(o, self.sizes[5])]
            ref, size = (linattn.forward(*[f(a[n]) for n in names], self.g, lens, zeros(self.s0, f), self.scale)[:2]
                         for f in (np.array, np.abs))
        assert all(r.max() < 1e37 for r in size)
        assert any(np.abs(r).max() > 0 for r in ref)
        if not limit:
            got = [np.where(np.isfinite(x), x, r) for x, r in zip(got, ref)]
            last = np.where(np.isfinite(f64(last)), f64(last), ref[-1])
        else:
            last = f64(last)
        for x, r, s in zip(got, ref, size):
            near_stored(x[on], r[on], U[prec] * np.abs(r[on]) + tol * s[on] +
                        (2.0 ** -25 if prec == "fp16" else 1e-37), prec, names)
        near(last.reshape(ref[-1].shape), ref[-1], tol * size[-1] + 1e-37, "state")


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("state", [False, True])
def test_growth_over_a_segment(prec, back, state):
    """384 tokens in segments, over each of which the heads grow by exp(96) and exp(320)."""
    c = Growing(prec, 384, 300, [0.75, 2.5], 64, back, state)
    assert B.rn18op_linattn_fwd_workspace(PREC[prec], *c.sizes) > 0
    c.check(back)


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("T,length", [(20, 20), (60, 60), (100, 97), (500, 500)])
@pytest.mark.parametrize("state", [False, True])
def test_growth_over_a_chunk(prec, back, T, length, state):
    """Up to the limit of a chunk's powers, exp(80) over 32 tokens."""
    Growing(prec, T, length, [2.5, 2.2, 1.0, 0.5, 0.1], 40, back, state).check(back)


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("T,length", [(20, 20), (60, 60), (100, 97), (500, 500)])
@pytest.mark.parametrize("state", [False, True])
def test_growth_beyond_the_limit(prec, back, T, length, state):
    """Heads that grow by more than fp32's range within 32 tokens: what is finite
    is right."""
    Growing(prec, T, length, [3.0, 4.5, 11.0, 30.0, 70.0], 40, back, state).check(back, limit=False)


@pytest.mark.parametrize("prec", PRECS)
def test_growing_single_tokens(prec):
    """Zeros stay zeros, and a small state grows."""
    g, D = np.array([3.0, 60.0, 88.0], np.float32), 24
    H, P = len(g), PREC[prec]
    s = np.zeros((1, H, D, D), np.float32)
    s[:, :, :, 5] = 1e-20
    z = vec(s)
    zero = mat(np.zeros((1, H * D)), prec)[0]
    o, _ = out(1, H * D, prec)
    B.rn18op_linattn_step(P, zero, zero, zero, vec(g), z, o, z, 1, H, H, D, D, H * D, H * D, H * D, H * D, 1.0)
    ref = s.astype(np.float64) * np.exp(g.astype(np.float64))[None, :, None, None]
    near(f64(z).reshape(ref.shape), ref, 4 * 89 * 2.0 ** -24 * ref, "state")
    assert (o == 0).all()
