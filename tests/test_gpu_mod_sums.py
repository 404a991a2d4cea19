"""The gradient of the bias table where its sums are of unusual values or go unusual ways, against 64 bits (mod_oracle.py)."""
import numpy as np
import pytest

from gpu_util import BWD_TOL, to_host
from test_gpu_mod import Case

pytestmark = pytest.mark.gpu


def off_by(c, dtable, ref):
    """|dtable - ref| in units of the bar that test_gpu_mod.py derives."""
    bar = BWD_TOL * (np.abs(ref) + np.sqrt(c.ds_squares()))
    return np.abs(dtable.astype(np.float64) - ref) / np.maximum(bar, 1e-300)


@pytest.mark.parametrize("L", [70, 800])                      # rows of sums taken as they are, and added up by a kernel of their own
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("p", [0.2, 0.8])
def test_a_sequence_that_is_switched_off_adds_zeros(p, d, L):
    # bias -100 and -inf: weights below 2^-125 and dS below 2^-143 |dP|, which rounds to zero in every format of the call.  1 / keep is 5 with p = 0.8.
    c = Case(3, L, L, 2, d, (L, L - 7, L - 33), (L, L - 7, L - 33), "both", 9, 8, None, p=p, seed=23)
    c.bias[1], c.bias[2] = -100.0, -np.inf
    dtable, ref = to_host(c.upload().bwd()[3]), c.reference()[4]
    assert np.all(np.isfinite(dtable)), dtable
    assert np.all(off_by(c, dtable, ref) <= 1)
