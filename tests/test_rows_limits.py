"""More arguments that the row operators refuse on the host, before anything
is launched (fake pointers, no GPU)."""
import os

import numpy as np
import pytest

from paper_2509_26092_amd import binding as B
from test_rows_refusals import distill

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
