"""NaN and infinities in linear attention's operands and states, forward and
backward, in calls that are cut into segments (the sums and what joins them see
them too) and in calls that are not.

What a value of token t reaches, by the formulas: o of the token (q), from it
on (k), from it on in its column (v); dq from it on in its column (k), from it
on (v), of the token (dO); dk up to it in its column (q), of the token (v), up
to it (dO); dv up to it (q), of the token (k), up to it in its column (dO).
There every result is NaN or infinite, and everything else keeps its value: in
other heads and sequences bit by bit, in its own within the bounds of
test_gpu_linattn.py, twice, since terms may be added up in another order."""
import numpy as np
import pytest

from oracle import linattn
from gpu_util import PREC
from paper_2509_26092_amd import binding as B
from test_gpu_linattn import Case, acc
from test_gpu_rmsnorm import TINY, U, near
from test_gpu_rows import f64, vec

pytestmark = pytest.mark.gpu

PRECS = ["fp32", "bf16", "fp16"]
D = {"q": 40, "k": 40, "v": 24, "do": 24}
COL = 3
# of each result, whom an operand's value reaches: tokens after ("on"), before ("to") or its own ("at"), all columns or one
REACH = {"o": {"q": ("at", False), "k": ("on", False), "v": ("on", True)},
         "dq": {"k": ("on", True), "v": ("on", False), "do": ("at", False)},
         "dk": {"q": ("to", True), "v": ("at", False), "do": ("to", False)},
         "dv": {"q": ("to", False), "k": ("at", False), "do": ("to", True)}}


class Both:
    """The results of one call each way, their bounds, and whether it is cut."""

    def __init__(self, prec, T):
        self.c = c = Case(prec, 2, T, 2, 2, D["k"], D["v"], None, True)
        self.prec, self.T = prec, T
        size = {n: np.abs(c.np[n]) for n in c.np}
        both = [np.abs(c.s0), np.abs(c.dsT)]
        ao, asT, _ = linattn.forward(size["q"], size["k"], size["v"], c.g, None, both[0], c.scale)
        aq, ak, av, as0 = linattn.backward(size["q"], size["k"], size["v"], size["do"], c.g, None, *both, c.scale)
        self.size = {"o": ao, "dq": aq, "dk": ak, "dv": av, "sT": asT, "ds0": as0}

    def run(self):
        c = self.c
        o, _, sT = c.fwd()
        outs, ds0 = c.bwd()
        width = {"o": D["v"], "dq": D["q"], "dk": D["k"], "dv": D["v"]}
        got = {n: c.rows(t, width[n]).copy() for n, t in (("o", o), *((n, outs[n][0]) for n in outs))}
        got["sT"], got["ds0"] = f64(sT).reshape(c.s0.shape), f64(ds0).reshape(c.s0.shape)
        return got

    def check(self, clean, got, reached):
        """reached: per result the elements of sequence 0, head 1 that are not
        finite (None: some of them may be)."""
        for n, g in got.items():
            own = (0, 1) if n in ("sT", "ds0") else (0, slice(None), 1)
            other = np.ones(g.shape, bool)
            other[own] = False
            assert np.array_equal(g[other], clean[n][other]), n
            r = reached.get(n, False)
            if r is None:
                continue
            mask = np.zeros(g[own].shape, bool)
            mask |= r
            assert not np.isfinite(g[own][mask]).any(), (n, "should not be finite")
            ref, size = clean[n][own][~mask], self.size[n][own][~mask]
            u = 0 if n in ("sT", "ds0") else U[self.prec]
            near(g[own][~mask], ref, 2 * (u * np.abs(ref) * (1 + u) + acc(self.prec, self.T) * size + TINY[self.prec]),
                 n)


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("T,tokens", [(100, (37, 64)), (2500, (0, 159, 160, 1003, 2499))])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_a_tokens_values(prec, T, tokens, value):
    both = Both(prec, T)
    c = both.c
    assert (B.rn18op_linattn_fwd_workspace(PREC[prec], *c.sizes) > 0) == (T > 2000)
    clean = both.run()
    at = np.arange(T)[:, None]
    for t in tokens:
        for what in ("q", "k", "v", "do"):
            x = c.dev[what].view(2, T, 2, -1)
            kept = x[0, t, 1, COL].clone()
            x[0, t, 1, COL] = value
            reached = {}
            for n, whom in REACH.items():
                if what in whom:
                    which, one = whom[what]
                    rows = {"at": at == t, "on": at >= t, "to": at <= t}[which]
                    reached[n] = rows & ((np.arange(both.size[n].shape[3]) == COL) | (not one))[None, :]
            # the states: a column of v's or dO's, a row of k's or q's
            m, n = np.arange(D["k"])[:, None] == COL, np.arange(D["v"])[None, :] == COL
            reached["sT"] = {"k": None, "v": np.broadcast_to(n, (D["k"], D["v"]))}.get(what, False)
            reached["ds0"] = {"q": None, "do": np.broadcast_to(n, (D["k"], D["v"]))}.get(what, False)
            both.check(clean, both.run(), reached)
            x[0, t, 1, COL] = kept
    got = both.run()
    assert all(np.array_equal(got[n], clean[n]) for n in got)


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("T", [100, 2500])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_a_states_values(prec, T, value):
    """An element (m, n) of s0 reaches column n of o and sT, column m of dq;
    one of dsT column m of dk, column n of dv and itself in ds0."""
    both = Both(prec, T)
    c = both.c
    clean = both.run()
    m, n = 5, COL
    col = lambda w, i: np.broadcast_to(np.arange(w)[None, :] == i, (T, w))
    for name in ("s0", "dsT"):
        a = getattr(c, name)
        kept, a[0, 1, m, n] = a[0, 1, m, n], value
        one = np.zeros((D["k"], D["v"]), bool)
        one[m, n] = True
        if name == "s0":
            reached = {"o": col(D["v"], n), "dq": col(D["k"], m), "sT": one}
        else:
            reached = {"dk": col(D["k"], m), "dv": col(D["v"], n), "ds0": one}
        both.check(clean, both.run(), reached)
        a[0, 1, m, n] = kept
