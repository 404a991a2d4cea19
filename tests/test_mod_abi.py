"""The calls with a relative position bias and with dropout refuse bad arguments on the host, before any HIP call: no GPU."""
import numpy as np
import pytest
import torch

from paper_2604_27124_amd import binding as A

P = 4096            # a fake, aligned, never dereferenced device address


def rel_fwd(lib, q=P, k=P, v=P, o=P, nq=P, nk=P, b=P, scale=0.125, table=P, buckets=P, num=8, reach=4, start=None, B=2, Lq=300, Lk=200, H=2, d=64,
            ws=None, bytes=0):
    return lib.sigmoid_attn_rel_fwd(q, k, v, o, nq, nk, b, scale, table, buckets, num, reach, start, B, Lq, Lk, H, d, ws, bytes, None)


def both_bwd(lib, g=P, dq=P, dk=P, dv=P, dt=P, scale=0.125, table=P, buckets=P, num=8, reach=4, start=None, p=0.1, rng=P, B=2, Lq=300, Lk=200, H=2, d=64,
             ws=P, bytes=1 << 40):
    return lib.sigmoid_attn_rel_dropout_bwd(P, P, P, g, dq, dk, dv, dt, P, P, P, scale, table, buckets, num, reach, start, p, rng, B, Lq, Lk, H, d,
                                            ws, bytes, None)


@pytest.fixture(scope="module")
def lib():
    return A.load()


@pytest.mark.parametrize("change,code", [
    (dict(q=None), A.SIGATTN_ERR_INVALID_ARG), (dict(o=None), A.SIGATTN_ERR_INVALID_ARG), (dict(nk=None), A.SIGATTN_ERR_INVALID_ARG),
    (dict(table=None), A.SIGATTN_ERR_INVALID_ARG), (dict(buckets=None), A.SIGATTN_ERR_INVALID_ARG), (dict(num=0), A.SIGATTN_ERR_INVALID_ARG),
    (dict(reach=-1), A.SIGATTN_ERR_INVALID_ARG), (dict(scale=float("nan")), A.SIGATTN_ERR_INVALID_ARG), (dict(B=0), A.SIGATTN_ERR_INVALID_ARG),
    (dict(d=96), A.SIGATTN_ERR_UNSUPPORTED_D), (dict(k=P + 8), A.SIGATTN_ERR_MISALIGNED), (dict(o=P + 2), A.SIGATTN_ERR_MISALIGNED),
    (dict(table=P + 1), A.SIGATTN_ERR_MISALIGNED), (dict(buckets=P + 2), A.SIGATTN_ERR_MISALIGNED), (dict(start=P + 2), A.SIGATTN_ERR_MISALIGNED),
    (dict(nq=P + 1), A.SIGATTN_ERR_MISALIGNED), (dict(reach=(1 << 24) + 1), A.SIGATTN_ERR_TOO_LARGE), (dict(num=(1 << 16) + 1), A.SIGATTN_ERR_TOO_LARGE),
    (dict(Lk=(1 << 29) + 1, B=1, H=1), A.SIGATTN_ERR_TOO_LARGE), (dict(B=1 << 20, Lq=1 << 14, H=1), A.SIGATTN_ERR_TOO_LARGE)])
def test_forward_refuses(lib, change, code):
    assert rel_fwd(lib, **change) == code


@pytest.mark.parametrize("change,code", [
    (dict(g=None), A.SIGATTN_ERR_INVALID_ARG), (dict(dt=None), A.SIGATTN_ERR_INVALID_ARG), (dict(dv=None), A.SIGATTN_ERR_INVALID_ARG),
    (dict(rng=None), A.SIGATTN_ERR_INVALID_ARG), (dict(p=1.0), A.SIGATTN_ERR_INVALID_ARG), (dict(p=-0.5), A.SIGATTN_ERR_INVALID_ARG),
    (dict(p=float("nan")), A.SIGATTN_ERR_INVALID_ARG), (dict(rng=P + 4), A.SIGATTN_ERR_MISALIGNED), (dict(dt=P + 1), A.SIGATTN_ERR_MISALIGNED),
    (dict(dk=P + 8), A.SIGATTN_ERR_MISALIGNED), (dict(ws=None), A.SIGATTN_ERR_WORKSPACE), (dict(bytes=1000), A.SIGATTN_ERR_WORKSPACE),
    (dict(ws=P + 8), A.SIGATTN_ERR_MISALIGNED), (dict(d=32), A.SIGATTN_ERR_UNSUPPORTED_D)])
def test_backward_refuses(lib, change, code):
    assert both_bwd(lib, **change) == code


def test_sizes(lib):
    size = A.sigmoid_attn_rel_bwd_workspace_bytes
    assert size(0, 8, 8, 1, 64, 4) == 0 and size(1, 8, 8, 1, 96, 4) == 0 and size(1, 8, 8, 1, 64, -1) == 0 and size(1, 8, 8, 1, 64, (1 << 24) + 1) == 0
    assert size(1, 8, 8, 1, 64, 4) > 0
    # the reach counts only as far as there are distances
    assert size(2, 512, 512, 4, 64, 1 << 20) == size(2, 512, 512, 4, 64, 1 << 24) > size(2, 512, 512, 4, 64, 64)
    few = A.sigmoid_attn_rel_fwd_workspace_bytes
    assert few(1, 1, 1000, 12, 64) == 0 and few(1, 65, 100000, 1, 64) == 0 and few(1, 0, 9, 1, 64) == 0
    assert few(1, 1, 8192, 12, 64) == 8 * 12 * 64 * 4 and few(1, 9, 8192, 1, 128) == 8 * 2 * 8 * 128 * 4
    # five queries and more of many heads, or of few keys, go to the tiled kernels
    assert few(1, 8, 8192, 128, 64) > 0 and few(1, 8, 8192, 129, 64) == 0 and few(1, 9, 8192, 65, 64) == 0 and few(1, 4, 8192, 193, 64) > 0
    assert few(1, 64, 1025, 1, 64) > 0 and few(1, 5, 1024, 1, 64) == 0


def test_bucket_map_refuses(lib):
    buf = np.zeros(3, np.int32)
    assert lib.sigmoid_attn_rel_buckets(None, 4, 1) == A.SIGATTN_ERR_INVALID_ARG
    assert lib.sigmoid_attn_rel_buckets(buf.ctypes.data, 0, 1) == A.SIGATTN_ERR_INVALID_ARG
    assert lib.sigmoid_attn_rel_buckets(buf.ctypes.data, 4, -1) == A.SIGATTN_ERR_INVALID_ARG
    with pytest.raises(ValueError):
        A.sigmoid_attn_rel_buckets(4, -1)
    with pytest.raises(A.SigAttnError):
        A.sigmoid_attn_rel_buckets(0, 1)


def test_tensors_of_the_host_are_refused():
    x, n, b = torch.zeros(1, 8, 1, 64, dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32), torch.zeros(1)
    table, buckets, rng = torch.zeros(4, 1, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int64)
    fast = A._fastcalls()
    assert fast.mod_fwd(1, x, x, x, n, n, b, 0.125, table, buckets, None) is None and fast.mod_bwd(2, x, x, x, x, n, n, b, 0.125, 0.1, rng) is None
    assert fast.mod_fwd(3) is None and fast.mod_fwd("1", x) is None and fast.mod_bwd() is None
    for call in (lambda: A.sigmoid_attn_rel_fwd(x, x, x, n, n, b, 0.125, table, buckets),
                 lambda: A.sigmoid_attn_dropout_fwd(x, x, x, n, n, b, 0.125, 0.1, rng),
                 lambda: A.sigmoid_attn_rel_dropout_bwd(x, x, x, x, n, n, b, 0.125, table, buckets, 0.1, rng)):
        with pytest.raises(ValueError):
            call()
