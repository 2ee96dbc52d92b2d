"""GPU parity of linear attention with the fp64 oracle, through the C ABI:
every storage type, sizes from one to the largest, shared heads, ragged
lengths, states, strides, misaligned rows, decays of every kind.

Tolerances, element by element. A is the same result of the operands' absolute
values (every term of its sums with its decay), which bounds what rounding in
the terms and in the additions can do: fp32 additions number at most 256 (a
product's depth) + 64 (a chunk) + T / 32 (chunks one after another, and the
powers' own roundings), 2^-24 each, and operands kept in 8-bit parts lose at
most 2^-16 each, of which a result sees three. Stored in 16 bits it is off by
U of itself more."""
import numpy as np
import pytest

from oracle import linattn
from paper_2509_26092_amd import binding as B
from gpu_util import PREC, rounded
from test_gpu_rmsnorm import TINY, U, near
from test_gpu_rows import f64, gaps_kept, mat, out, vec, ws_of

pytestmark = pytest.mark.gpu

PRECS = ["fp32", "bf16", "fp16"]


def acc(prec, T):
    return (320 + T / 32) * 2.0 ** -24 + (0 if prec == "fp32" else 3 * 2.0 ** -16)


def near_stored(got, ref, bound, prec, name):
    """near, where what rounds beyond fp16's largest number is stored as an
    infinity: from 65520 on, half a step above it."""
    beyond = (prec == "fp16") & (np.abs(ref) + bound >= 65520) & np.isinf(got) & (np.sign(got) == np.sign(ref))
    near(np.where(beyond, ref, got), ref, bound, name)


def decays(H, kind="mixed"):
    with np.errstate(divide="ignore"):
        return np.log1p(-np.exp2(-np.arange(1, H + 1, dtype=np.float64))).astype(np.float32) if kind == "mixed" else \
            np.array({"ends": [-np.inf, 0.0, -80.0, -1e-4], "growing": [0.01, -0.5, 0.1, 1e-5]}[kind] * H,
                     np.float32)[:H]


def ints(a):
    import torch
    return None if a is None else torch.tensor(a, dtype=torch.int32, device="cuda")


class Case:
    """Inputs of one call on the device, rows behind a sequence NaN, and the
    oracle's results."""

    def __init__(self, prec, B_, T, H, Hk, Dk, Dv, lengths=None, state=True, pad=0, off=0, kind="mixed", size=1.0):
        import torch
        rng = np.random.default_rng(T * 31 + Dk + Dv)
        self.prec, self.sizes, self.lengths, self.pad, self.off = prec, (B_, T, H, Hk, Dk, Dv), lengths, pad, off
        self.g = decays(H, kind)
        shapes = {"q": (H, Dk), "k": (Hk, Dk), "v": (Hk, Dv), "do": (H, Dv)}
        self.np = {n: rounded(size * rng.standard_normal((B_, T) + s), prec) for n, s in shapes.items()}
        if lengths is not None:
            for b, n in enumerate(lengths):
                for a in self.np.values():
                    a[b, max(0, min(n, T)):] = np.nan
        f32 = lambda *s: rng.standard_normal(s).astype(np.float32)
        self.s0, self.dsT = (f32(B_, H, Dk, Dv), f32(B_, H, Dk, Dv)) if state else (None, None)
        self.scale = 0.37
        self.dev = {n: mat(a.reshape(B_ * T, -1), prec, pad, off)[0] if B_ * T else torch.empty(0, device="cuda")
                    for n, a in self.np.items()}
        self.gd = vec(self.g)
        self.lens = ints(lengths)

    def ld(self, n):
        return self.np[n].shape[2] * self.np[n].shape[3] + self.pad

    def state(self, a):
        return None if a is None else vec(a)

    def fwd(self, s0=None, sT=None):
        B_, T, H, Hk, Dk, Dv = self.sizes
        P = PREC[self.prec]
        o, buf = out(B_ * T, H * Dv, self.prec, self.pad, self.off)
        sT = vec(np.full((B_, H, Dk, Dv), 5.0)) if sT is None else sT
        s0 = self.state(self.s0) if s0 is None else s0
        ws = ws_of(B.rn18op_linattn_fwd_workspace(P, *self.sizes))
        d = self.dev
        B.rn18op_linattn_fwd(P, d["q"], d["k"], d["v"], self.gd, self.lens, s0, o, sT, *self.sizes, self.ld("q"),
                             self.ld("k"), self.ld("v"), H * Dv + self.pad, self.scale, ws)
        return o, buf, sT

    def bwd(self, ds0=None, dsT=None):
        B_, T, H, Hk, Dk, Dv = self.sizes
        P, d = PREC[self.prec], self.dev
        outs = {n: out(B_ * T, w, self.prec, self.pad, self.off) for n, w in
                (("dq", H * Dk), ("dk", Hk * Dk), ("dv", Hk * Dv))}
        ds0 = vec(np.full((B_, H, Dk, Dv), 5.0)) if ds0 is None else ds0
        ws = ws_of(B.rn18op_linattn_bwd_workspace(P, *self.sizes))
        B.rn18op_linattn_bwd(P, d["q"], d["k"], d["v"], d["do"], self.gd, self.lens, self.state(self.s0),
                             self.state(self.dsT) if dsT is None else dsT, outs["dq"][0], outs["dk"][0], outs["dv"][0],
                             ds0, *self.sizes, self.ld("q"), self.ld("k"), self.ld("v"), self.ld("do"),
                             H * Dk + self.pad, Hk * Dk + self.pad, Hk * Dv + self.pad, self.scale, ws)
        return outs, ds0

    def inside(self):
        B_, T = self.sizes[:2]
        n = np.full(B_, T) if self.lengths is None else np.clip(self.lengths, 0, T)
        return np.arange(T)[None, :] < n[:, None]

    def rows(self, t, width):
        B_, T = self.sizes[:2]
        return f64(t).reshape(B_, T, -1, width)

    def check_fwd(self):
        o, buf, sT = self.fwd()
        on, a, tol = self.inside(), self.np, acc(self.prec, self.sizes[1])
        lens = on.sum(axis=1)
        args = lambda f: [f(a[n]) for n in "qkv"]
        ro, rs, _ = linattn.forward(*args(lambda x: x), self.g, lens, self.s0, self.scale)
        ao, As, _ = linattn.forward(*args(np.abs), self.g, lens, None if self.s0 is None else np.abs(self.s0),
                                    self.scale)
        got = self.rows(o, self.sizes[5])
        near_stored(got[on], ro[on], U[self.prec] * np.abs(ro[on]) + tol * ao[on] + TINY[self.prec], self.prec, "o")
        assert np.all(got[~on] == 7.0) and gaps_kept(o, buf)
        near(f64(sT).reshape(rs.shape), rs, tol * As + 1e-37, "sT")

    def check_bwd(self):
        outs, ds0 = self.bwd()
        on, a, tol = self.inside(), self.np, acc(self.prec, self.sizes[1])
        lens = on.sum(axis=1)
        f = lambda g: linattn.backward(*[g(a[n]) for n in ("q", "k", "v", "do")], self.g, lens,
                                       None if self.s0 is None else g(self.s0),
                                       None if self.dsT is None else g(self.dsT), self.scale)
        ref, size = f(lambda x: x), f(np.abs)
        for n, r, s, w in zip(("dq", "dk", "dv"), ref, size, (self.sizes[4], self.sizes[4], self.sizes[5])):
            got = self.rows(outs[n][0], w)
            near_stored(got[on], r[on], U[self.prec] * np.abs(r[on]) + tol * s[on] + TINY[self.prec], self.prec, n)
            assert np.all(got[~on] == 7.0) and gaps_kept(*outs[n]), n
        near(f64(ds0).reshape(ref[3].shape), ref[3], tol * size[3] + 1e-37, "ds0")


# (B, T, H, Hk, Dk, Dv, lengths, states, pad, offset)
CASES = [(1, 1, 1, 1, 1, 1, None, True, 0, 0), (2, 1, 3, 1, 5, 7, None, False, 0, 0), (1, 5, 2, 2, 16, 16, None, True, 0, 0),
         (1, 63, 2, 2, 64, 64, None, False, 0, 0), (1, 64, 2, 2, 64, 64, None, True, 0, 0),
         (2, 65, 2, 1, 64, 64, [65, 64], True, 0, 0), (3, 129, 4, 2, 32, 96, [129, 0, 1], True, 3, 1),
         (2, 200, 2, 1, 100, 36, [200, 77], True, 5, 2), (1, 130, 2, 2, 256, 256, None, True, 0, 0),
         (1, 257, 1, 1, 128, 200, None, False, 0, 0), (4, 77, 4, 4, 17, 33, [500, -3, 77, 32], True, 1, 3),
         (2, 196, 8, 8, 64, 64, None, False, 0, 0), (1, 500, 4, 1, 128, 128, None, True, 8, 8),
         (2, 33, 2, 2, 250, 3, [31, 33], True, 0, 0), (1, 40, 1, 1, 3, 250, None, True, 0, 0),
         (2, 130, 2, 2, 129, 65, [130, 100], True, 0, 0), (1, 200, 2, 2, 64, 200, None, True, 0, 0),
         (1, 70, 1, 1, 200, 130, None, True, 1, 0), (70, 40, 2, 2, 16, 16, None, False, 0, 0)]


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("i", range(len(CASES)))
def test_forward(prec, i):
    B_, T, H, Hk, Dk, Dv, lengths, state, pad, off = CASES[i]
    Case(prec, B_, T, H, Hk, Dk, Dv, lengths, state, pad, off).check_fwd()


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("i", range(len(CASES)))
def test_backward(prec, i):
    B_, T, H, Hk, Dk, Dv, lengths, state, pad, off = CASES[i]
    Case(prec, B_, T, H, Hk, Dk, Dv, lengths, state, pad, off).check_bwd()


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("T,lengths", [(150, None), (150, [149, 3])])
def test_decays_at_their_ends(prec, T, lengths):
    """A head without memory, one without decay, one that underflows, a slow one."""
    c = Case(prec, 2, T, 4, 2, 24, 40, lengths, True, kind="ends")
    c.check_fwd()
    c.check_bwd()


@pytest.mark.parametrize("prec", PRECS)
def test_growing_heads(prec):
    """exp(0.1 * 150) = 3e6, in one segment and in several; and a head whose
    state loses more than a chunk keeps, whose small rest counts."""
    for T in (150, 500):
        c = Case(prec, 1, T, 4, 4, 24, 40, None, True, kind="growing", size=0.01 if T > 200 else 1.0)
        if T > 200:
            c.g = np.minimum(c.g, 0.02).astype(np.float32)
            c.gd = vec(c.g)
        if prec == "fp16":
            c.scale *= 2.0 ** -20
        c.check_fwd()
        c.check_bwd()


@pytest.mark.parametrize("prec,T,Dk,Dv", [("bf16", 3001, 64, 64), ("fp32", 2500, 40, 24), ("fp16", 2049, 128, 16),
                                          ("bf16", 4100, 128, 128), ("bf16", 2100, 16, 160)])
@pytest.mark.parametrize("lengths", [None, "short"])
def test_long_sequences(prec, T, Dk, Dv, lengths):
    """Long enough that a call's few heads are cut along the sequence."""
    c = Case(prec, 2, T, 2, 1, Dk, Dv, None if lengths is None else [T, T // 2 + 1], True)
    c.check_fwd()
    c.check_bwd()


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("size", [1e-5, 30.0])
def test_small_and_large_values(prec, size):
    """Sums beyond fp16's range and operands below its normal numbers."""
    c = Case(prec, 1, 300, 2, 2, 64, 48, None, False, size=size)
    c.scale = 1e-3 if size > 1 else 1e5
    c.check_fwd()
    if prec != "fp16" or size < 1:
        c.check_bwd()


@pytest.mark.parametrize("prec", PRECS)
def test_no_tokens_and_no_sequences(prec):
    import torch
    c = Case(prec, 2, 0, 2, 1, 8, 8)
    _, _, sT = c.fwd()
    _, ds0 = c.bwd()
    assert np.array_equal(f64(sT).reshape(c.s0.shape), c.s0) and np.array_equal(f64(ds0).reshape(c.s0.shape), c.dsT)
    c = Case(prec, 2, 0, 2, 1, 8, 8, state=False)
    assert (c.fwd()[2] == 0).all() and (c.bwd()[1] == 0).all()
    P = PREC[prec]
    g = vec(decays(2))
    B.rn18op_linattn_fwd(P, None, None, None, g, None, None, None, None, 0, 5, 2, 1, 8, 8, 16, 8, 8, 16, 1.0)
    B.rn18op_linattn_step(P, None, None, None, g, None, None, None, 0, 2, 1, 8, 8, 16, 8, 8, 16, 1.0)
    torch.cuda.synchronize()


@pytest.mark.parametrize("T", [70, 2500])
def test_states_in_place_and_not_wanted(T):
    c = Case("bf16", 2, T, 2, 2, 64, 48, [T, T - 9], True)
    o, _, sT = c.fwd()
    s = vec(c.s0)
    o2, _, _ = c.fwd(s, s)
    import torch
    assert torch.equal(o, o2) and torch.equal(s, sT)
    outs, ds0 = c.bwd()
    s = vec(c.dsT)
    outs2, _ = c.bwd(s, s)
    assert torch.equal(s, ds0) and all(torch.equal(outs[n][0], outs2[n][0]) for n in outs)


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("B_,H,Hk,Dk,Dv,pad,off", [(1, 1, 1, 1, 1, 0, 0), (1, 8, 8, 64, 64, 0, 0), (5, 4, 2, 96, 100, 3, 1),
                                                   (3, 2, 1, 256, 256, 0, 0), (2, 3, 3, 7, 250, 0, 5),
                                                   (2, 2, 2, 250, 6, 1, 0), (40, 16, 16, 128, 128, 0, 0),
                                                   (2, 2, 2, 33, 13, 0, 0), (95, 2, 2, 40, 200, 0, 3),
                                                   (300, 2, 1, 20, 130, 0, 0)])
def test_step(prec, B_, H, Hk, Dk, Dv, pad, off):
    """Against the oracle's one token, into another state and in place."""
    import torch
    c = Case(prec, B_, 1, H, Hk, Dk, Dv, None, True, pad, off)
    P, d = PREC[prec], c.dev
    s0, new = vec(c.s0), vec(np.full(c.s0.shape, 3.0))
    o, buf = out(B_, H * Dv, prec, pad, off)
    call = lambda a, b, to: B.rn18op_linattn_step(P, d["q"], d["k"], d["v"], c.gd, a, to, b, B_, H, Hk, Dk, Dv,
                                                  c.ld("q"), c.ld("k"), c.ld("v"), H * Dv + pad, c.scale)
    call(s0, new, o)
    args = lambda f: [f(c.np[n]) for n in "qkv"]
    ro, rs, _ = linattn.forward(*args(lambda x: x), c.g, None, c.s0, c.scale)
    ao, As, _ = linattn.forward(*args(np.abs), c.g, None, np.abs(c.s0), c.scale)
    tol = acc("fp32", 1)
    near(c.rows(o, Dv), ro, U[prec] * np.abs(ro) + tol * ao + TINY[prec], "o")
    near(f64(new).reshape(rs.shape), rs, tol * As + 1e-37, "state")
    assert gaps_kept(o, buf)
    o2, _ = out(B_, H * Dv, prec, pad, off)
    call(s0, s0, o2)
    assert torch.equal(s0, new) and torch.equal(o, o2)


def test_prompt_then_single_tokens():
    """A prompt's state carried on token by token gives the whole sequence's
    outputs (each path within its own bound of the oracle)."""
    import torch
    c = Case("bf16", 2, 90, 4, 2, 64, 48, None, True)
    B_, T, H, Hk, Dk, Dv = c.sizes
    P, d = PREC["bf16"], c.dev
    cut = 70
    part = {n: d[n].view(B_, T, -1)[:, :cut].reshape(B_ * cut, -1).contiguous() for n in "qkv"}
    o = torch.empty((B_ * cut, H * Dv), dtype=torch.bfloat16, device="cuda")
    s = vec(c.s0)
    sizes = (B_, cut, H, Hk, Dk, Dv)
    B.rn18op_linattn_fwd(P, part["q"], part["k"], part["v"], c.gd, None, s, o, s, *sizes, H * Dk, Hk * Dk, Hk * Dv,
                         H * Dv, c.scale, ws_of(B.rn18op_linattn_fwd_workspace(P, *sizes)))
    outs = [o.view(B_, cut, H * Dv)]
    for t in range(cut, T):
        tok = {n: d[n].view(B_, T, -1)[:, t].contiguous() for n in "qkv"}
        y = torch.empty((B_, H * Dv), dtype=torch.bfloat16, device="cuda")
        B.rn18op_linattn_step(P, tok["q"], tok["k"], tok["v"], c.gd, s, y, s, B_, H, Hk, Dk, Dv, H * Dk, Hk * Dk,
                              Hk * Dv, H * Dv, c.scale)
        outs.append(y[:, None])
    got = f64(torch.cat(outs, dim=1)).reshape(B_, T, H, Dv)
    args = lambda f: [f(c.np[n]) for n in "qkv"]
    ro, rs, _ = linattn.forward(*args(lambda x: x), c.g, None, c.s0, c.scale)
    ao, As, _ = linattn.forward(*args(np.abs), c.g, None, np.abs(c.s0), c.scale)
    near(got, ro, U["bf16"] * np.abs(ro) + acc("bf16", T) * ao, "o")
    near(f64(s).reshape(rs.shape), rs, acc("bf16", T) * As, "state")


def test_parts_of_one_buffer():
    """q, k, v beside each other in the rows of one product's output."""
    import torch
    B_, T, H, Hk, Dk, Dv = 2, 100, 4, 2, 32, 48
    c = Case("bf16", B_, T, H, Hk, Dk, Dv, None, False)
    w = H * Dk + Hk * Dk + Hk * Dv
    buf = torch.cat([c.dev[n] for n in "qkv"], dim=1).contiguous()
    q, k, v = buf[:, :H * Dk], buf[:, H * Dk:(H + Hk) * Dk], buf[:, (H + Hk) * Dk:]
    o = torch.empty((B_ * T, H * Dv), dtype=torch.bfloat16, device="cuda")
    ws = ws_of(B.rn18op_linattn_fwd_workspace(PREC["bf16"], *c.sizes))
    B.rn18op_linattn_fwd(PREC["bf16"], q, k, v, c.gd, None, None, o, None, *c.sizes, w, w, w, H * Dv, c.scale, ws)
    assert torch.equal(o, c.fwd()[0])


def test_same_bits_twice_on_streams_and_replayed():
    """Two calls at once on two streams, with a workspace each, and replays of
    a captured forward and backward pass, give the eager call's bits."""
    import torch
    c = Case("bf16", 1, 2500, 2, 1, 64, 64, None, True)
    o, _, sT = c.fwd()
    outs, ds0 = c.bwd()
    torch.cuda.synchronize()
    want = [o.clone(), sT.clone(), ds0.clone()] + [outs[n][0].clone() for n in outs]
    got = []
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        with torch.cuda.stream(s):
            a, _, b = c.fwd()
            d, e = c.bwd()
            got.append([a, b, e] + [d[n][0] for n in d])
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for g in got for x, y in zip(g, want))
    B_, T, H, Hk, Dk, Dv = c.sizes
    P, d = PREC["bf16"], c.dev
    s0, dsT = vec(c.s0), vec(c.dsT)
    ws = ws_of(B.rn18op_linattn_fwd_workspace(P, *c.sizes))
    wb = ws_of(B.rn18op_linattn_bwd_workspace(P, *c.sizes))
    new = [torch.empty_like(x) for x in want]
    graph, s = torch.cuda.CUDAGraph(), streams[0]
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        B.rn18op_linattn_fwd(P, d["q"], d["k"], d["v"], c.gd, None, s0, new[0], new[1], *c.sizes, H * Dk, Hk * Dk,
                             Hk * Dv, H * Dv, c.scale, ws)
        B.rn18op_linattn_bwd(P, d["q"], d["k"], d["v"], d["do"], c.gd, None, s0, dsT, new[3], new[4], new[5], new[2],
                             *c.sizes, H * Dk, Hk * Dk, Hk * Dv, H * Dv, H * Dk, Hk * Dk, Hk * Dv, c.scale, wb)
    for _ in range(3):
        for x in new:
            x.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(new, want))


def test_offsets_beyond_32_bits():
    """Token rows 2^30 elements apart: the last one beyond 2^32 bytes."""
    import torch
    T, D, ld = 4, 32, (1 << 30) + 8
    buf = torch.zeros(3 * ld + D, dtype=torch.bfloat16, device="cuda")
    q = torch.as_strided(buf, (T, D), (ld, 1), 0)
    q.copy_(torch.randn((T, D), device="cuda"))
    a, g, P = q.contiguous(), vec(decays(1)), PREC["bf16"]
    o, o2 = torch.empty_like(a), torch.empty_like(a)
    sizes = (1, T, 1, 1, D, D)
    ws = ws_of(B.rn18op_linattn_fwd_workspace(P, *sizes))
    B.rn18op_linattn_fwd(P, q, q, q, g, None, None, o, None, *sizes, ld, ld, ld, D, 1.0, ws)
    B.rn18op_linattn_fwd(P, a, a, a, g, None, None, o2, None, *sizes, D, D, D, D, 1.0, ws)
    assert torch.equal(o, o2)


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("what", ["q", "k", "v"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_what_a_token_holds_reaches_no_earlier_one(prec, what, value):
    """A NaN or an infinity of token 37, in a chunk with earlier tokens: those
    keep their outputs; from there on the head's are not finite (q: that token's alone)."""
    import torch
    c = Case(prec, 2, 100, 2, 2, 32, 48, None, True)
    clean = c.fwd()[0].view(2, 100, 2, 48)
    t = c.dev[what].view(2, 100, 2, -1)
    t[0, 37, 1, 3] = value
    o = c.fwd()[0].view(2, 100, 2, 48)
    assert torch.equal(o[1], clean[1]) and torch.equal(o[0, :, 0], clean[0, :, 0])
    # in the chunk of the token, terms may be added up in another order: both
    # results are within the bound of the exact one, so within two of each other
    args = [np.abs(c.np[n]) for n in "qkv"]
    size = linattn.forward(*args, c.g, None, np.abs(c.s0), c.scale)[0][0, :, 1]
    ref = f64(clean[0, :, 1])
    two = 2 * (U[prec] * np.abs(ref) * (1 + U[prec]) + acc(prec, 100) * size)
    near(f64(o[0, :37, 1]), ref[:37], two[:37], "o")
    bad = ~torch.isfinite(o[0, :, 1])
    if what == "q":
        assert bad[37].all() and torch.equal(o[0, 38:, 1], clean[0, 38:, 1])
    elif what == "k":
        assert bad[37:].all()
    else:
        assert bad[37:, 3].all()
        others = [n for n in range(48) if n != 3]
        near(f64(o[0, :, 1])[:, others], ref[:, others], two[:, others], "other columns")


def test_as_many_heads_as_there_may_be():
    """2^20 query heads over 2^19 key heads, one token: rows of 2^28 elements.
    Small integers, whose products and sums are exact."""
    import torch
    H, Hk, Dk, Dv, P = 1 << 20, 1 << 19, 256, 1, PREC["bf16"]
    sizes = (1, 1, H, Hk, Dk, Dv)
    small = lambda n, w: torch.randint(-3, 4, (n, w), device="cuda", dtype=torch.int8).to(torch.bfloat16)
    q, k, v, do = small(H, Dk), small(Hk, Dk), small(Hk, Dv), small(H, Dv)
    g = torch.zeros(H, device="cuda")
    dq, dk, dv = (torch.full_like(x, 7) for x in (q, k, v))
    ws = ws_of(B.rn18op_linattn_bwd_workspace(P, *sizes))
    B.rn18op_linattn_bwd(P, q, k, v, do, g, None, None, None, dq, dk, dv, None, *sizes, H * Dk, Hk * Dk, Hk * Dv,
                         H * Dv, H * Dk, Hk * Dk, Hk * Dv, 1.0, ws)
    shared = lambda x: x.view(Hk, 2, 1)
    assert torch.equal(dq.view(Hk, 2, Dk), shared(do) * v.view(Hk, 1, 1) * k.view(Hk, 1, Dk))
    assert torch.equal(dk, (q.view(Hk, 2, Dk) * (shared(do) * v.view(Hk, 1, 1))).sum(1))
    dots = (q.view(Hk, 2, Dk).float() * k.view(Hk, 1, Dk).float()).sum(2, keepdim=True)
    assert torch.equal(dv, (dots * shared(do).float()).sum(1).to(torch.bfloat16))
