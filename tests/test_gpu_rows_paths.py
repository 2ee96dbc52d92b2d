"""GPU parity of the row operators at the sizes where the choice of kernel
changes hands: enough rows that a block works on several sets of them (the
next rows loaded ahead, sums over the rows kept between them), every number of
lanes and chunks that a row can take, and lists that no room of a block holds.

The layer norms are compared with the definition in 64 bits on the same GPU
(elementary operations), top logits and distillation with the fp64 oracle.
Tolerances are those of test_gpu_rows: U, the unit roundoff of the stored
type, plus TOL = 1e-5 of the largest value for fp32 arithmetic."""
import math

import numpy as np
import pytest

from oracle import rows
from paper_2509_26092_amd import binding as B
from gpu_util import PREC, rounded, torch_dtype
from test_gpu_rows import (EPS, PRECS, TOL, U, check_topk, distill_inputs, empty, f64, gaps_kept, loss_bound, mat,
                           out, run_distill, ws_of)

pytestmark = pytest.mark.gpu


def rand_rows(R, D, prec, pad, off, scale, shift, seed):
    """Random rows made on the GPU, `pad` elements apart, `off` elements into
    their buffer."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((off + R * (D + pad) + 64,), float("nan"), dtype=torch_dtype(prec), device="cuda")
    v = torch.as_strided(buf, (R, D), (D + pad, 1), off)
    v.copy_(torch.randn((R, D), generator=g, device="cuda") * scale + shift)
    return v


def blank(R, D, prec, pad, off):
    import torch
    buf = torch.full((off + R * (D + pad) + 64,), -3.0, dtype=torch_dtype(prec), device="cuda")
    return torch.as_strided(buf, (R, D), (D + pad, 1), off), buf


# (rows, width, pad, offset, in place): more rows than the launch's blocks take at once
FWD = [(40000, 64, 0, 0, False), (300000, 64, 0, 0, True), (2200000, 8, 0, 0, False), (33000, 509, 3, 1, False),
       (17000, 2050, 0, 0, True), (4300, 4101, 0, 0, False), (2200, 8205, 5, 3, True), (1100, 16405, 1, 0, False)]


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("R,D,pad,off,in_place", FWD)
def test_layernorm_fwd_many_rows(prec, R, D, pad, off, in_place):
    import torch
    x = rand_rows(R, D, prec, pad, off, 1.5, 0.4, R + D)
    gamma, beta = torch.randn(D, device="cuda"), torch.randn(D, device="cuda")
    x64 = x.double()
    m = x64.sum(dim=1) / D
    x64 -= m[:, None]
    rs = 1.0 / torch.sqrt((x64 * x64).sum(dim=1) / D + EPS)
    want = x64 * rs[:, None] * gamma.double() + beta.double()
    y, buf = (x, None) if in_place else blank(R, D, prec, 2 * pad, off)
    mean, rstd = empty(R), empty(R)
    B.rn18op_layernorm_fwd(PREC[prec], x, gamma, beta, y, mean, rstd, R, D, x.stride(0), y.stride(0), EPS)
    torch.cuda.synchronize()
    err = (y.double() - want).abs()
    assert bool((err <= (U[prec] + TOL) * want.abs().max()).all()), err.max().item()
    assert bool(((mean.double() - m).abs() <= TOL * m.abs().max()).all())
    assert bool(((rstd.double() - rs).abs() <= TOL * rs.max()).all())
    assert in_place or gaps_kept(y, buf)


# (rows, width, pad, offset, what dx replaces)
BWD = [(300000, 5, 0, 1, None), (400000, 8, 0, 0, None), (200000, 16, 0, 0, "dy"), (120000, 32, 0, 0, "x"),
       (60000, 64, 0, 0, None), (31000, 136, 0, 0, "dy"), (16000, 255, 1, 1, None), (5000, 509, 3, 1, None),
       (2500, 1000, 0, 0, "x"), (1300, 2050, 0, 0, None), (1300, 3001, 0, 0, None), (1300, 4101, 7, 0, "dy"),
       (1300, 6001, 0, 0, None), (1300, 8000, 0, 0, "x"), (600, 8205, 3, 1, None), (600, 12001, 0, 0, "dy"),
       (600, 16380, 0, 0, "x"), (100, 17001, 0, 0, None)]


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("R,D,pad,off,place", BWD)
def test_layernorm_bwd_many_rows(prec, R, D, pad, off, place):
    """The sums over the rows as in test_gpu_rows.check_param_grads: chains of
    at most R additions in fp32, whose roundings add up to about R 2^-24 times
    a term's root mean square, four times that, and the terms' own."""
    import torch
    x = rand_rows(R, D, prec, pad, off, 1.5, 0.4, R + D)
    dy = rand_rows(R, D, prec, pad, off, 0.7, 0.0, R + D + 1)
    gamma = torch.randn(D, device="cuda")
    x64, g64 = x.double(), dy.double()
    m = (x64.sum(dim=1) / D).float()
    rs = (1.0 / torch.sqrt(((x64 - m.double()[:, None]) ** 2).sum(dim=1) / D + EPS)).float()
    xh = (x64 - m.double()[:, None]) * rs.double()[:, None]
    sums = [(g64 * xh, "dgamma"), (g64, "dbeta")]
    sums = [(t.sum(dim=0), torch.sqrt((t * t).sum(dim=0) / R), name) for t, name in sums]
    g64 = g64 * gamma.double()
    want = rs.double()[:, None] * (g64 - g64.sum(dim=1, keepdim=True) / D - xh * (g64 * xh).sum(dim=1, keepdim=True) / D)
    size = (rs.double()[:, None] * g64).abs().max()
    dx, buf = (dy if place == "dy" else x, None) if place else blank(R, D, prec, 2 * pad, off)
    got = [empty(D), empty(D)]
    ws = ws_of(B.rn18op_layernorm_bwd_workspace(PREC[prec], R, D))
    B.rn18op_layernorm_bwd(PREC[prec], dy, x, gamma, m, rs, dx, got[0], got[1], R, D, dy.stride(0), x.stride(0),
                           dx.stride(0), ws)
    torch.cuda.synchronize()
    err = (dx.double() - want).abs()
    # fp16 below 2^-14 rounds to a multiple of 2^-24
    tiny = 2.0 ** -25 if prec == "fp16" else 0.0
    assert bool((err <= U[prec] * want.abs() + TOL * size + tiny).all()), (err.max() / size).item()
    for v, (s, rms, name) in zip(got, sums):
        bound = 4 * R * 2.0 ** -24 * rms + 16 * math.sqrt(R) * 2.0 ** -24 * (rms + rms.max())
        assert bool(((v.double() - s).abs() <= bound).all()), name
    assert place or gaps_kept(dx, buf)


# ---------------------------------------------------------------- top logits
def special_rows(C, K, prec, seed):
    """Random, equal, masked but some, few distinct values, with NaN and
    infinities, one run of large values."""
    rng = np.random.default_rng(seed)
    z = rounded(rng.standard_normal((6, C)) * 2.5, prec)
    z[1] = 1.0
    z[2] = -np.inf
    z[2, rng.integers(0, C, max(1, K // 2))] = 1.0
    z[3] = rng.integers(0, 3, C)
    z[4, rng.integers(0, C, 3)] = np.nan
    z[4, rng.integers(0, C, 3)] = np.inf
    z[5, C // 3:C // 3 + min(K + 5, C // 2)] += 16.0
    z[5] = rounded(z[5], prec)
    return z


@pytest.mark.parametrize("prec,C,K,pad,off",
                         [("bf16", 400, 5, 0, 0), ("fp16", 511, 40, 1, 3), ("fp32", 256 + 3, 7, 0, 1),
                          ("bf16", 2000, 100, 0, 0), ("fp16", 2040, 256, 5, 1), ("fp32", 1024 - 1, 65, 0, 0),
                          ("bf16", 4000, 100, 0, 0), ("fp16", 4090, 200, 1, 1), ("fp32", 2000, 130, 0, 0),
                          ("bf16", 8000, 70, 0, 0), ("fp32", 300001, 256, 1, 1), ("bf16", 600001, 256, 0, 1),
                          ("fp16", 1048577, 200, 0, 0)])
def test_topk_lanes_and_lists(prec, C, K, pad, off):
    """A wave a row with one chunk a lane, blocks with one and two chunks a
    lane, and rows too long for a block's registers with lists too long for
    parts."""
    check_topk(special_rows(C, K, prec, C + K), prec, K, pad, off)


def test_topk_workspace_of_rows_in_parts():
    """Rows of more than 2^14 chunks need room for every part's list, except
    where the lists of all parts pass what one block joins."""
    for prec, C in ((B.RN18_BF16, 131080), (B.RN18_FP32, 65540)):
        n = B.rn18op_topk_logits_workspace(prec, 3, C, 64)
        assert n >= 3 * 2 * 64 * 8 and n % (3 * 64 * 8) == 0
    assert B.rn18op_topk_logits_workspace(B.RN18_FP32, 2, 300001, 256) == 0


# ---------------------------------------------------------------- distillation
@pytest.mark.parametrize("prec,R,C,K,T,alpha,masked,pad,off",
                         [("bf16", 70, 50001, 32, 1.5, 0.5, True, 3, 0), ("fp16", 70, 50001, 32, 1.5, 0.5, True, 3, 1),
                          ("fp32", 66, 20001, 64, 2.0, 1.0, True, 1, 0), ("bf16", 65, 131071, 64, 2.0, 0.6, True, 1, 1),
                          ("fp16", 65, 131064, 20, 2.0, 1.0, False, 0, 0), ("fp32", 65, 40001, 20, 4.0, 0.5, True, 0, 1),
                          ("bf16", 1100, 500, 100, 2.0, 0.5, True, 1, 1), ("fp32", 1100, 255, 100, 2.0, 1.0, True, 0, 0),
                          ("bf16", 1100, 2000, 20, 2.0, 0.5, True, 0, 0), ("fp32", 1030, 1000, 200, 2.0, 0.5, True, 1, 0),
                          ("fp16", 1100, 4000, 64, 4.0, 0.9, True, 3, 1), ("fp32", 1030, 2000, 33, 2.0, 1.0, False, 0, 0),
                          ("bf16", 300, 7001, 65, 2.0, 0.5, True, 1, 0), ("fp16", 300, 20001, 33, 2.0, 0.5, True, 1, 0),
                          ("bf16", 2100, 250, 61, 2.0, 0.6, True, 1, 1), ("fp16", 2100, 255, 62, 2.0, 0.6, True, 0, 0),
                          ("fp32", 2100, 127, 63, 2.0, 1.0, True, 1, 0), ("bf16", 2100, 100, 64, 2.0, 0.6, True, 3, 1),
                          ("fp32", 2100, 63, 64, 2.0, 0.6, True, 0, 0), ("bf16", 2100, 500, 38, 3.0, 0.5, True, 1, 0),
                          ("fp32", 2100, 250, 17, 3.0, 0.5, True, 0, 1)])
def test_distill_lanes_and_chunks(prec, R, C, K, T, alpha, masked, pad, off):
    """Rows whole in a block of 512 or 1024 lanes, in a wave with one to
    eight chunks a lane, and in sixteen lanes with lists of up to 64: several
    rounds of entries a lane, and 1 to 3 places beside the last ones."""
    import torch
    z, t_vals, t_idx, labels, weight = distill_inputs(prec, R, C, K, masked, seed=11)
    scale = (1024.0 if prec == "fp16" else 1.0) / R
    zd, _ = mat(z, prec, pad, off)
    dzd, dzbuf = out(R, C, prec, 2 * pad, off)
    row, loss = run_distill(zd, prec, t_vals, t_idx, labels, weight, K, T, alpha, scale, R, C, C + pad, dzd,
                            C + 2 * pad)
    row_o, loss_o, dz_o = rows.distill(z, t_vals, t_idx, labels, weight, T, alpha, scale)
    tol = loss_bound(z, t_vals, weight, T, alpha)
    assert np.abs(row - row_o).max() <= tol
    assert abs(loss - loss_o) <= scale * R * tol + 2.0 ** -23 * abs(loss_o)
    # an fp16 gradient below 2^-14 rounds to a multiple of 2^-24
    assert np.abs(f64(dzd) - dz_o).max() <= (U[prec] + TOL) * np.abs(dz_o).max() + \
        (2.0 ** -25 if prec == "fp16" else 0.0) + scale * T * TOL
    assert gaps_kept(dzd, dzbuf)
    if weight is not None:
        assert not f64(dzd)[weight == 0.0].any()
    row2, _ = run_distill(zd, prec, t_vals, t_idx, labels, weight, K, T, alpha, scale, R, C, C + pad, zd, C + pad,
                          want_loss=False)
    assert torch.equal(dzd, zd) and np.array_equal(row, row2)      # in place of z, bit for bit


# ---------------------------------------------------------------- every kernel
# 16-byte chunks of a row: one width for each number of lanes and of chunks a lane
@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("chunks", [1, 2, 3, 7, 15, 31, 60, 120, 180, 250, 500, 700, 1000, 1400, 2000, 2900, 4000])
def test_layernorm_every_width(prec, chunks):
    """Few rows, and for rows within a wave as many as take two rows a lane
    at once; whole chunks, and a tail beside them."""
    vw = 4 if prec == "fp32" else 8
    lanes = min(64, 1 << (chunks - 1).bit_length())
    for R in [37] + ([256 * (256 // lanes) * 4 + 3] if chunks <= 64 else []):
        for D in (chunks * vw, chunks * vw + 3):
            test_layernorm_fwd_many_rows(prec, R, D, 0, 0, False)
            test_layernorm_bwd_many_rows(prec, R, D, 0, 0, None)


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("alpha", [1.0, 0.5])
@pytest.mark.parametrize("R,chunks", [(2050, 15), (2050, 30), (2050, 60), (1030, 60), (1030, 120), (1030, 250),
                                      (1030, 500), (300, 200), (300, 400), (300, 1000), (140, 2000), (66, 4000),
                                      (66, 8000), (66, 16000)])
def test_distill_every_width(prec, alpha, R, chunks):
    """Sixteen lanes, a wave and blocks of 256 to 1024 lanes, with the
    labels' term and without (a list of 70 keeps 60 chunks in a wave)."""
    vw = 4 if prec == "fp32" else 8
    test_distill_lanes_and_chunks(prec, R, chunks * vw + 1, 70 if (R, chunks) == (1030, 60) else 9, 2.0, alpha, True, 1,
                                  0)
