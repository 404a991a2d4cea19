"""Pins of the oracle of the calls with a relative position bias and with dropout (mod_oracle.py), and of the bucket map: no GPU."""
import numpy as np
import pytest

import mod_oracle as M
from paper_2604_27124_amd import binding as A


def test_generator_known_answers():
    # the published known answers of the generator for counter and key zero, with ten and with seven rounds
    assert [int(x) for x in M.philox((0, 0, 0, 0), (0, 0), 10)] == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert [int(x) for x in M.philox((0, 0, 0, 0), (0, 0), 7)] == [0x5F6FB709, 0x0D893F64, 0x4F121F81, 0x4F730A48]


@pytest.mark.parametrize("p", [0.003, 0.1, 0.5, 0.9])
def test_mask_share_and_independence(p):
    n = 1024
    m = M.mask(77, 5, 3, n, n, p)
    keep = M.kept(p) / 65536
    assert abs(keep - (1 - p)) <= 0.5 / 65536 + 1e-7                       # p arrives as a float
    sd = np.sqrt(keep * (1 - keep)) / n                                    # of the mean of n^2 decisions
    assert abs(m.mean() - keep) < 5 * sd
    x = m - keep
    for dj, di in ((1, 0), (2, 0), (4, 0), (8, 0), (16, 0), (32, 0), (0, 1), (0, 32), (1, 1)):
        a, b = x[:n - di, :n - dj], x[di:, dj:]
        corr = float((a * b).mean()) / (keep * (1 - keep))
        # keys 2k and 2k + 1 share the low halves of their 16-bit numbers: at most 2/256 of their decisions hang together
        assert abs(corr) < 5 / np.sqrt(a.size) + (2 / 256 if (dj, di) == (1, 0) else 0), (di, dj, corr)
    for other in (M.mask(78, 5, 3, n, n, p), M.mask(77, 6, 3, n, n, p), M.mask(77, 5, 4, n, n, p)):
        assert abs(float((x * (other - keep)).mean())) / (keep * (1 - keep)) < 5 / n


def test_gradients_by_differences():
    r = np.random.default_rng(3)
    n, m, d = 5, 7, 4
    q, k, v, g = r.standard_normal((n, d)), r.standard_normal((m, d)), r.standard_normal((m, d)), r.standard_normal((n, d))
    column, buckets = r.standard_normal(4), np.array([0, 1, 1, 2, 3, 3, 0])
    keep = M.mask(1, 2, 3, n, m, 0.3)
    f = lambda q, k, v, c: float((M.head(q, k, v, None, -0.7, 0.5, c, buckets, 1, keep, 0.7)[0] * g).sum())
    _, dq, dk, dv, dc = M.head(q, k, v, g, -0.7, 0.5, column, buckets, 1, keep, 0.7)
    eps = 1e-6
    args = [q, k, v, column]
    for a, want in zip(args, (dq, dk, dv, dc)):
        for at in np.ndindex(*a.shape):
            was = a[at]
            a[at] = was + eps
            up = f(*args)
            a[at] = was - eps
            low = f(*args)
            a[at] = was
            # a central difference: eps^2 of the third derivative, and rounding of about 1e-16 |f| / eps
            assert abs((up - low) / (2 * eps) - want[at]) < 1e-7 * (1 + abs(want[at]))


@pytest.mark.parametrize("num,reach", [(32, 128), (1, 5), (2, 0), (3, 10), (101, 50), (400, 50), (7, 1000), (64, 3)])
def test_bucket_map(num, reach):
    b = A.sigmoid_attn_rel_buckets(num, reach).numpy()
    assert b.shape == (2 * reach + 1,) and b.min() >= 0 and b.max() < num
    if num >= 2 * reach + 1:
        assert (b == np.arange(2 * reach + 1)).all()
        return
    near, far = b[reach::-1], b[reach + 1:]                                # keys before the query (and itself), keys behind it
    assert (np.diff(near) >= 0).all() and (np.diff(far) >= 0).all()
    if num >= 4 and reach > 1:
        assert set(near) & set(far) == set() and near[0] == 0 and near[1] == 1


def test_mask_by_distance():
    # an entry of -inf takes its pairs out: a window of attention
    r = np.random.default_rng(4)
    q, k, v = (r.standard_normal((9, 4)) for _ in range(3))
    buckets = np.array([0, 1, 1, 1, 0])
    o = M.head(q, k, v, None, 0.0, 0.5, np.array([-np.inf, 0.0]), buckets)[0]
    x = 0.5 * q @ k.T
    near = np.abs(np.arange(9)[None] - np.arange(9)[:, None]) < 2
    assert np.allclose(o, (M.sigma(x) * near) @ v, atol=1e-12)
