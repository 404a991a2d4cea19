"""The gradient of the bias table where its sums are of unusual values or go unusual ways, against 64 bits (mod_oracle.py)."""
import numpy as np
import pytest

from gpu_util import BWD_TOL, to_host
from mod_oracle import mask
from test_gpu_mod import Case, check

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


@pytest.mark.parametrize("op", ["rel", "both"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_what_is_not_finite_stays_in_its_bucket(bad, d, op):
    # every distance a bucket of its own; dS of one of them is not finite: a NaN in the table, or +-Inf in dO and V that meet in one pair alone
    L, R = 90, 40
    c = Case(1, L, L, 1, d, (L,), (L - 3,), op, R, 2 * R + 1, None, p=0.2, seed=24)
    if np.isnan(bad):
        c.table[R + 7] = bad
        hit = [R + 7]
    else:
        # dP = <dO_i, V_j> overflows for query 50 and keys 50 + 7 and 50 + 10 only: both 2^70 in a column that is 0 for all others
        c.g[0, :, 0, 5], c.v[0, :, 0, 5] = 0.0, 0.0
        c.g[0, 50, 0, 5], c.v[0, [57, 60], 0, 5] = 2.0 ** 70, (2.0 ** 70, -2.0 ** 70)
        hit = [R + 7, R + 10]
    with np.errstate(invalid="ignore"):
        ref = c.reference()[4]
        clean = [b for b in range(2 * R + 1) if b not in hit]
        squares = c.ds_squares()[clean]
    dtable = to_host(c.upload().bwd()[3]).astype(np.float64)
    assert np.all(np.isfinite(dtable[clean])), np.argwhere(~np.isfinite(dtable))
    assert np.all(np.abs(dtable[clean] - ref[clean]) <= BWD_TOL * (np.abs(ref[clean]) + np.sqrt(squares)))
    stays = mask(*c.rng, 0, L, L, c.p) if op == "both" else np.ones((L, L), bool)
    for b in hit:                                               # what dropout takes out is not in the sum
        if np.isnan(bad):
            assert np.isnan(dtable[b, 0])
        else:
            assert np.isinf(dtable[b, 0]) == stays[50, 50 + b - R]


WAYS = {
    # sequences with starts of their own and more than 64 rows of sums: near, far out on either side, without queries, without keys
    "starts": dict(B=20, Lq=150, Lk=200, H=2, nq=[150 - 7 * i for i in range(20)], nk=[200, 0, 131, 64] * 5, reach=40, num=16,
                   start=[0, 50, -60, 199, -149, 1000, -1000, 2 ** 31 - 1, -2 ** 31, 31, 32, 33, -31, -32, -33, 63, 64, 65, 1, 7]),
    # more than 1024 entries of a row, with and without starts
    "long rows, starts": dict(B=3, Lq=1000, Lk=700, H=2, nq=(1000, 333, 999), nk=(700, 699, 33), reach=600, num=32, start=(-150, 300, 0)),
    "long rows": dict(B=3, Lq=1000, Lk=700, H=2, nq=(1000, 333, 999), nk=(700, 699, 33), reach=600, num=32, start=None),
    # a bucket for every distance
    "all distances": dict(B=5, Lq=500, Lk=600, H=1, nq=(500, 0, 499, 31, 32), nk=(600, 600, 0, 599, 1), reach=650, num=1301, start=(0, 0, 9, 100, -60)),
    # groups of sequences, each with several
    "groups": dict(B=67, Lq=64, Lk=96, H=1, nq=[64 - i % 65 for i in range(67)], nk=[96 - i for i in range(67)], reach=30, num=12, start=None),
}


@pytest.mark.parametrize("op", ["rel", "both"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("way", WAYS)
def test_every_way_of_adding_up(way, d, op):
    w = WAYS[way]
    assert w["B"] * -(-w["Lq"] // 32) > 64                      # not the kernel of a few rows
    check(Case(w["B"], w["Lq"], w["Lk"], w["H"], d, w["nq"], w["nk"], op, w["reach"], w["num"], w["start"], seed=25))


def test_a_long_row_of_few_queries():
    # more than 1024 entries in the kernel of a few rows
    check(Case(2, 90, 1500, 2, 64, (90, 77), (1500, 1411), "rel", 1400, 32, (700, -20), seed=26))
