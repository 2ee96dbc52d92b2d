"""The row operators at the limits of their arguments."""
import numpy as np
import pytest

from oracle import rows
from paper_2509_26092_amd import binding as B
from test_gpu_rows import TOL, distill_inputs, f64, mat, out, run_distill, ws_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prec,D", [("bf16", 2 ** 27 + 13), ("fp32", 2 ** 27)])
def test_layernorm_bwd_of_the_widest_rows(prec, D):
    """The launch that joins the parameter gradients takes 32 columns a block
    of 1024: more than 2^27 columns pass what one launch may hold."""
    import torch
    R = 2
    dt = {"bf16": torch.bfloat16, "fp32": torch.float32}[prec]
    x = torch.randn((R, D), device="cuda", dtype=dt)
    dy = torch.randn((R, D), device="cuda", dtype=dt)
    m = x.double().mean(dim=1).float()
    rs = (1.0 / torch.sqrt(((x.double() - m.double()[:, None]) ** 2).mean(dim=1) + 1e-5)).float()
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    ws = ws_of(B.rn18op_layernorm_bwd_workspace(B.PREC_IDS[prec], R, D))
    B.rn18op_layernorm_bwd(B.PREC_IDS[prec], dy, x, None, m, rs, dx, dgamma, dbeta, R, D, D, D, D, ws)
    torch.cuda.synchronize()
    g = dy.double()
    xh = (x.double() - m.double()[:, None]) * rs.double()[:, None]
    assert bool(((dbeta.double() - g.sum(dim=0)).abs() <= TOL * 6).all())
    assert bool(((dgamma.double() - (g * xh).sum(dim=0)).abs() <= TOL * 36).all())
    xh *= (g * xh).sum(dim=1, keepdim=True) / D
    want = rs.double()[:, None] * (g - g.sum(dim=1, keepdim=True) / D - xh)
    assert bool(((dx.double() - want).abs() <= (2.0 ** -8 if prec == "bf16" else 0.0) * want.abs() + TOL * 7).all())

LOW = -3.4028234663852886e38


# (rows, classes): sixteen lanes, a wave or a block a row, whole blocks of up
# to 1024 lanes, and rows in parts
@pytest.mark.parametrize("R,C", [(2100, 100), (1100, 1000), (8, 10), (8, 1000), (8, 33000), (70, 50001), (8, 200000)])
@pytest.mark.parametrize("T", [0.5, 2.0 ** -50, 2.0 ** 70])
def test_distill_teacher_values_of_the_whole_range(R, C, T):
    """Teacher's values whose quotient by the temperature passes fp32's range:
    a row of the lowest value throughout (equal shares), the lowest and the
    highest beside others. Logits are small multiples of T where T is tiny
    and of 1 elsewhere, so every loss and gradient is an ordinary number up to
    the factors T^2 and T, which `scale` takes back for the gradient. Soft
    terms of T = 2^70 are log(C / K) T^2, beyond fp32: infinite."""
    rng = np.random.default_rng(R + C)
    K = 4
    z = rng.integers(-3, 4, (R, C)).astype(np.float64) * min(T, 1.0)
    t_idx = np.stack([rng.permutation(C)[:K] for _ in range(R)]).astype(np.int32)
    t_vals = rng.integers(-3, 4, (R, K)).astype(np.float32) * np.float32(min(T, 1.0))
    t_vals[0] = LOW
    t_vals[1] = [LOW, 1.0, 1.0, LOW]
    t_vals[2] = [-LOW, -LOW, 1.0, 0.0]
    t_vals[3] = [2.0 ** 100, 2.0 ** 100, 0.0, LOW]
    t_vals[4, 0] = -np.inf
    scale = 1.0 / T
    zd, _ = mat(z, "fp32")
    dzd, _ = out(R, C, "fp32")
    row, _ = run_distill(zd, "fp32", t_vals, t_idx, None, None, K, T, 1.0, scale, R, C, C, dzd, C)
    row_o, _, dz_o = rows.distill(zd.cpu().numpy(), t_vals, t_idx, None, None, T, 1.0, scale)
    assert np.isfinite(f64(dzd)).all() and np.abs(f64(dzd) - dz_o).max() <= TOL * np.abs(dz_o).max()
    if T > 1e19:
        assert (row == np.inf).all() and (row_o > 3.5e38).all()
    else:
        assert np.abs(row / T ** 2 - row_o / T ** 2).max() <= TOL * np.abs(row_o / T ** 2).max()


def test_distill_of_one_class_at_a_high_temperature():
    """One class: nothing to learn, a loss of 0 at every temperature."""
    zd, _ = mat(np.array([[3.0], [-2.0]]), "fp32")
    dzd, _ = out(2, 1, "fp32")
    for T in (1.0, 1e15, 1e25, 1e38):
        row, loss = run_distill(zd, "fp32", np.ones((2, 1), np.float32), np.zeros((2, 1), np.int32), None, None, 1, T,
                                1.0, 1.0 / T, 2, 1, 1, dzd, 1)
        assert not row.any() and loss == 0.0 and not f64(dzd).any()


@pytest.mark.parametrize("classes", [10, 70000])
def test_step_flags_bad_labels_that_no_term_reads(classes):
    """alpha = 1: the labels have no part in the loss, and one that is
    neither a class nor -1 is still reported."""
    import torch
    N = 4
    w = B.Worker("tiny", classes, "fp32")
    state = torch.zeros(w.n_state, device="cuda")
    B.rn18_destroy(B.rn18_init(w.cfg, 3, state))
    x = torch.randn((N, 3, 16, 16), device="cuda")
    vals = torch.randn((N, 3), device="cuda")
    idx = torch.arange(3 * N, device="cuda", dtype=torch.int32).view(N, 3) % classes
    for bad, want in ((0, B.RN18_OK), (-1, B.RN18_OK), (classes, B.RN18_ELABEL), (-2, B.RN18_ELABEL)):
        y = torch.zeros(N, device="cuda", dtype=torch.int32)
        y[N - 1] = bad
        for alpha in (1.0, 0.5):
            w.train_step_distill(state, x, y, vals, idx, 2.0, alpha, 0.0)
            assert w.sync_status() == want, (bad, alpha)
    w.train_step_distill(state, x, None, vals, idx, 2.0, 1.0, 0.0)
    assert w.sync_status() == B.RN18_OK
    w.close()


def test_workspace_of_a_step_does_not_grow_by_rows_in_parts():
    """Rows of more than 65,536 fp32 classes are joined from parts in a step
    with a teacher. Their room is memory that the backward pass needs anyway:
    the workspace grows by the same amount a class below and above. (Sizes
    where no other buffer changes its kind.)"""
    ctx = {c: B.Worker("tiny", c, "fp32") for c in range(65408, 65665, 64)}
    n = {c: B.rn18_workspace_bytes(w.ctx, 100, 16, 16) for c, w in ctx.items()}
    step = n[65472] - n[65408]
    assert step > 0
    for c in (65472, 65536, 65600):
        assert n[c + 64] - n[c] == step, c


def test_status_names_the_teachers_list():
    """A class of the teacher's list outside [0, C) sets the same status as
    such a label: its text names both."""
    import torch
    w = B.Worker("tiny", 10, "fp32")
    state = torch.zeros(w.n_state, device="cuda")
    B.rn18_destroy(B.rn18_init(w.cfg, 3, state))
    idx = torch.tensor([[1, 10], [2, 3]], device="cuda", dtype=torch.int32)
    w.train_step_distill(state, torch.randn((2, 3, 16, 16), device="cuda"), None, torch.randn((2, 2), device="cuda"),
                         idx, 2.0, 1.0, 0.0)
    assert w.sync_status() == B.RN18_ELABEL
    assert "label" in B.rn18_last_error() and "teacher" in B.rn18_last_error()
    w.close()


@pytest.mark.parametrize("R,C", [(2100, 100), (8, 10), (8, 1000), (8, 33000), (70, 50001), (8, 200000)])
@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_distill_teacher_without_a_number(R, C, bad):
    """A teacher's NaN or +inf: its row's loss and the gradient of the classes
    that the row lists are NaN; the other classes' gradient, which needs the
    student's logits alone, and every other row are as without it."""
    K = 5
    z, t_vals, t_idx, labels, _ = distill_inputs("fp32", R, C, K, False, seed=4)
    t_vals[1, 2] = bad
    zd, _ = mat(z, "fp32")
    dzd, _ = out(R, C, "fp32")
    row, loss = run_distill(zd, "fp32", t_vals, t_idx, labels, None, K, 2.0, 0.5, 1.0, R, C, C, dzd, C)
    with np.errstate(all="ignore"):
        row_o, _, dz_o = rows.distill(z, t_vals, t_idx, labels, None, 2.0, 0.5, 1.0)
    dz = f64(dzd)
    listed = np.zeros((R, C), bool)
    listed[1, t_idx[1]] = True
    assert np.array_equal(np.isnan(dz), listed) and np.array_equal(np.isnan(dz_o), listed)
    assert np.abs(dz - dz_o)[~listed].max() <= TOL * np.abs(dz_o[~listed]).max()
    good = np.arange(R) != 1
    assert np.isnan(row[1]) and np.isnan(loss) and np.allclose(row[good], row_o[good], rtol=1e-5, atol=1e-5)


@pytest.mark.parametrize("D", [3, 64, 1001, 8192, 33000])
def test_layernorm_beyond_the_sums_range(D):
    """Squares beyond fp32's range: rstd 0 and rows of beta. Sums beyond it:
    NaN. The rows beside them are as ever."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(D)
    x = torch.randn((4, D), device="cuda", generator=g)
    x[1, 0], x[1, 1] = 1e20, -1e20
    x[2, :2] = 3e38
    beta = torch.randn(D, device="cuda", generator=g)
    y, mean, rstd = torch.empty_like(x), torch.empty(4, device="cuda"), torch.empty(4, device="cuda")
    B.rn18op_layernorm_fwd(B.RN18_FP32, x, None, beta, y, mean, rstd, 4, D, D, D)
    assert rstd[1].item() == 0.0 and torch.equal(y[1], beta)
    assert bool(y[2].isnan().all())
    want, _, _ = rows.layernorm_forward(x[0::3].cpu().double().numpy(), None, beta.cpu().double().numpy(), 1e-5)
    assert np.abs(f64(y[0::3]) - want).max() <= TOL * np.abs(want).max()


def test_rows_of_2_30_elements():
    """The widest rows the operators take, one short of whole chunks by
    three, in bf16: positions to the end of the range. A lane adds 2^20
    terms in a chain here: their roundings come to about 1e-5 of the sum."""
    import torch
    D, U, tol = 2 ** 30 - 3, 2.0 ** -8, 1e-4
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((1, D), device="cuda", generator=g, dtype=torch.bfloat16)
    x64 = x.double()
    m = x64.mean()
    x64 -= m
    rs = 1.0 / torch.sqrt((x64 * x64).mean() + 1e-5)
    x64 *= rs
    y, mean, rstd = torch.empty_like(x), torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    B.rn18op_layernorm_fwd(B.RN18_BF16, x, None, None, y, mean, rstd, 1, D, D, D)
    assert abs(mean.item() - m.item()) <= tol and abs(rstd.item() / rs.item() - 1) <= tol
    assert bool(((y.double() - x64).abs() <= U * x64.abs() + tol * 7).all())
    # the gradient of dy = y: xh is y up to a rounding, and so is what remains of dy after its projections
    dgamma, dbeta = torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    dx = torch.empty_like(x)
    B.rn18op_layernorm_bwd(B.RN18_BF16, y, x, None, mean, rstd, dx, dgamma, dbeta, 1, D, D, D, D,
                           ws_of(B.rn18op_layernorm_bwd_workspace(B.RN18_BF16, 1, D)))
    assert torch.equal(dbeta, y[0].float())
    assert bool(((dgamma.double() - y[0].double() * x64[0]).abs() <= tol * 40).all())
    y64 = y.double()
    want = rs * (y64 - y64.mean() - x64 * (y64 * x64).mean())
    assert bool(((dx.double() - want).abs() <= U * want.abs() + tol * 7).all())
    del dgamma, dbeta, dx, y64, want, x64, y
    K = 20
    x[0, D - 1], x[0, 5], x[0, D - 2] = 30.0, 30.0, 20.0
    vals, idx = torch.empty((1, K), device="cuda"), torch.empty((1, K), device="cuda", dtype=torch.int32)
    B.rn18op_topk_logits(B.RN18_BF16, x, vals, idx, 1, D, D, K, ws_of(B.rn18op_topk_logits_workspace(B.RN18_BF16, 1, D, K)))
    assert idx[0, :3].tolist() == [5, D - 1, D - 2]
    v, at = x[0].float().topk(4 * K)
    ties = sorted(zip((-v).tolist(), at.tolist()))
    assert v[-1] < v[K - 1] and [(-a, b) for a, b in ties[:K]] == list(zip(vals[0].tolist(), idx[0].tolist()))
    T = 4.0
    dz, row, loss = torch.empty_like(x), torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    lab = torch.tensor([D - 3], device="cuda", dtype=torch.int32)
    scale = 2.0 ** 20
    B.rn18op_distill_loss(B.RN18_BF16, x, vals, idx, lab, None, dz, row, loss, 1, D, D, D, K, T, 0.5, scale,
                          ws_of(B.rn18op_distill_loss_workspace(B.RN18_BF16, 1, D, K)))
    z = x[0].double()
    q = torch.softmax(vals[0].double() / T, 0)
    i = idx[0].long()
    want = torch.zeros(D, dtype=torch.float64, device="cuda")
    value = 0.0
    for t, w in ((T, 0.5 * T), (1.0, 0.5)):
        lse = torch.logsumexp(z / t, 0)
        want += w * torch.exp(z / t - lse)
        if t == T:
            want.scatter_add_(0, i, -w * q)
            value += 0.5 * T * T * (q * (q.log() - z[i] / T + lse)).sum()
        else:
            want[D - 3] -= w
            value += 0.5 * (lse - z[D - 3])
    want *= scale
    assert abs(row.item() / value.item() - 1) <= tol
    assert bool(((dz[0].double() - want).abs() <= U * want.abs() + tol * want.abs()).all())
