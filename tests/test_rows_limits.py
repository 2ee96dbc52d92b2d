"""More arguments that the row operators refuse on the host, before anything
is launched (fake pointers, no GPU)."""
import os

import numpy as np
import pytest

from paper_2509_26092_amd import binding as B
from test_rows_refusals import P, bwd, distill, topk

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="library not built")


def test_temperatures_whose_exponent_factor_is_infinite_are_refused():
    """Exponentials are powers of 2 with the factor log2(e) / T, which leaves
    fp32's range before 1 / T does: there the row's maximum itself would give
    0 times infinity."""
    log2e, big = 1.44269504088896340736, float(np.finfo(np.float32).max)
    first = np.float32(log2e / big)                  # 4.24e-39, within a step of 1.4e-45
    up, down = first * np.float32(1.001), first * np.float32(0.999)
    for t in (down, np.float32(3e-39), np.float32(2.95e-39)):
        assert distill(temperature=t, R=4) == B.RN18_EINVAL, t
        assert distill(temperature=t, R=0, K=0, z=None, dz=None, row_loss=None) == B.RN18_EINVAL
    # no rows: nothing is launched where the arguments are taken
    for t in (up, np.float32(1e-38), np.float32(1.0), np.float32(3e38)):
        assert distill(temperature=t, R=0, K=0, z=None, dz=None, row_loss=None) == B.RN18_OK, t


def top_case(prec, R, C, K, **kw):
    return topk(prec=prec, R=R, C=C, ldz=C, K=K, **kw)


def norm_case(prec, R, C, K, **kw):
    return bwd(prec=prec, R=R, D=C, lddy=C, ldx=C, lddx=C, **kw)


def loss_case(prec, R, C, K, **kw):
    return distill(prec=prec, R=R, C=C, ldz=C, lddz=C, K=K, **kw)


@pytest.mark.parametrize("prec", [B.RN18_FP32, B.RN18_BF16, B.RN18_FP16])
@pytest.mark.parametrize("f,need", [(top_case, B.rn18op_topk_logits_workspace),
                                    (loss_case, B.rn18op_distill_loss_workspace),
                                    (norm_case, lambda prec, R, C, K: B.rn18op_layernorm_bwd_workspace(prec, R, C))])
@pytest.mark.parametrize("R", [1, 3, 700])
def test_rows_in_parts_refuse_workspaces_too_small_or_missing(prec, f, need, R):
    """Rows of more than 2^14 chunks: every operator needs a workspace."""
    C, K = 131080 // (2 if prec == B.RN18_FP32 else 1), 5
    n = need(prec, R, C, K)
    assert n > 0
    assert f(prec, R, C, K, ws_bytes=n - 1) == B.RN18_ENOMEM
    assert f(prec, R, C, K, ws_bytes=0) == B.RN18_ENOMEM
    assert f(prec, R, C, K, ws=None, ws_bytes=n) == B.RN18_EINVAL
    assert f(prec, R, C, K, ws=P((1 << 20) + 4), ws_bytes=n) == B.RN18_EINVAL
