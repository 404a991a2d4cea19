"""Sequences whose bias is far below zero together with a large scale or few weights that stay: the gradients' factor scale 2^(-bias log2 e) / keep passes fp32,
the gradients do not."""
import numpy as np
import pytest
import torch

from paper_2604_27124_amd import binding as A
from paper_2604_27124_amd import workloads as W
from gpu_util import BWD_TOL, FWD_TOL, Dev, check_against_oracle, check_slices, to_host
from test_gpu_mod import Case

pytestmark = pytest.mark.gpu

ROUTES = [
    # B, N, H, d
    (2, 200, 2, 64),        # small launches
    (40, 150, 12, 64),      # both passes in one launch
    (22, 513, 12, 64),      # one pass
    (2, 200, 2, 128),       # four waves a workgroup
    (40, 200, 16, 128),     # eight
]


@pytest.mark.parametrize("B,N,H,d", ROUTES)
def test_switched_off_sequences_have_zero_gradients(B, N, H, d):
    gen = torch.Generator(device="cuda").manual_seed(N)
    q, k, v, g = (torch.empty(B, N, H, d, dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for _ in range(4))
    q *= 2.0 ** -6                                             # scores of about 1 with a scale of 8
    n = torch.tensor([N - i % 50 for i in range(B)], dtype=torch.int32, device="cuda")
    bias = torch.full((B,), -5.0, device="cuda")
    want = A.sigmoid_attn_bwd(q, k, v, g, n, bias, 8.0)
    bias[1::2] = -100.0
    bias[1::4] = float("-inf")
    got = A.sigmoid_attn_bwd(q, k, v, g, n, bias, 8.0)
    cross = A.sigmoid_attn_cross_bwd(q, k, v, g, n, n, bias, 8.0)
    halves = (A.sigmoid_attn_bwd_dq(q, k, v, g, n, bias, 8.0), *A.sigmoid_attn_bwd_dkdv(q, k, v, g, n, bias, 8.0))
    dbias = A.sigmoid_attn_bwd_dq_dbias(q, k, v, g, n, bias, 8.0)
    for grads in (got, cross, halves, (dbias[0], got[1], got[2])):
        for name, a in zip(("dQ", "dK", "dV"), grads):
            # dS < 2^-143 |dP| is zero; P <= 2^-125, over 513 rows of |dO| < 6
            assert float(a[1::2].float().abs().max()) <= (1e-34 if name == "dV" else 0.0), name
    for a, b in zip(got, want):                                # the others' results are theirs alone
        assert torch.equal(a[::2].view(torch.int16), b[::2].view(torch.int16))
    assert bool((dbias[1][1::2] == 0).all())


@pytest.mark.parametrize("bias", [-42.0, -60.0, -80.0])
def test_weights_near_zero(bias):
    # P keeps its accuracy; dS is held as exp(score + 2 bias) dP, which leaves fp32 between the first two
    w = W.make(1, 256, 1, 64, (256,), seed=14, bias=[bias])
    if bias > -44:
        check_against_oracle(w)
        return
    dev = Dev(w)
    dq, dk, dv = (to_host(a) for a in dev.bwd())
    import oracle
    check_slices("O", to_host(dev.fwd()), oracle.fwd(w.q, w.k, w.v, w.seqlens, w.bias, w.scale), w.seqlens, [(0, 0)], FWD_TOL)
    check_slices("dV", dv, oracle.bwd(w.q, w.k, w.v, w.d_o, w.seqlens, w.bias, w.scale)[2], w.seqlens, [(0, 0)], BWD_TOL)
    # scores below 6 in size: exp(6 - 120) |dP| is below 2^-149
    assert not dq.any() and not dk.any()


def steep(x, bias, scale, spread, seed):
    """x: an object with q and k.  Scores that make up for the bias: q = k = s in the first column, scale s^2 = -bias, and noise in the others."""
    r = np.random.default_rng(seed)
    for name in ("q", "k"):
        a = getattr(x, name)
        s = np.sqrt(spread / scale / np.sqrt(a.shape[3]))     # standard deviation of scale <q, k>: spread
        a[...] = r.standard_normal(a.shape) * s
        a[..., 0] = np.sqrt(-bias / scale)
        setattr(x, name, W.round_to_bf16(a.astype(np.float32)))
    x.bias[:] = -scale * float(x.q[0, 0, 0, 0]) * float(x.k[0, 0, 0, 0])
    x.scale = scale


# scale log2 e is a power of two, so that queries are scaled without rounding; scale 2^(-bias log2 e) is 2^129.5.  dS / 2^(-bias log2 e) is about 2^-103,
# its products with queries and keys 2^-118: far from what fp32 rounds to zero
SCALE, BIAS = float(np.float32(2.0 ** 29 * np.log(2.0))), -70.0


@pytest.mark.parametrize("B,N,H,d", [r for r in ROUTES if r[0] < 22] + [(22, 513, 12, 64)])
def test_gradients_of_steep_scores(B, N, H, d):
    w = W.make(B, N, H, d, [N - 3 * i for i in range(B)], seed=31)
    steep(w, BIAS, SCALE, 2.0, 31)
    slices = [(z, h) for z in range(min(B, 2)) for h in range(2)]
    check_against_oracle(w, slices=slices)


@pytest.mark.parametrize("op", ["rel", "dropout", "both"])
@pytest.mark.parametrize("d", [64, 128])
def test_gradients_of_steep_scores_with_a_table_and_dropout(d, op):
    c = Case(2, 150, 130, 2, d, (150, 77), (130, 99), op, 9, 8, None, seed=33)
    steep(c, BIAS, SCALE, 2.0, 33)
    ref = c.reference()
    c.upload()
    for name, a, r, n, tol in zip(("O", "dQ", "dK", "dV"), (c.fwd(), *c.bwd()[:3]), ref, (c.nq, c.nq, c.nk, c.nk), (FWD_TOL, *[BWD_TOL] * 3)):
        check_slices(name, to_host(a), r, n, [(z, h) for z in range(2) for h in range(2)], tol)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("op", ["dropout", "both"])
def test_switched_off_sequences_with_dropout(op, d):
    # 1 / keep = 33.3, times 0.125 and 2^126: more than fp32 holds
    c = Case(3, 300, 260, 2, d, (300, 131, 77), (260, 200, 77), op, 9, 8, None, p=0.97, seed=34)
    c.bias[1], c.bias[2] = -100.0, -np.inf
    c.scale = max(c.scale, 0.125)
    ref = c.reference()
    c.upload()
    o, (dq, dk, dv) = to_host(c.fwd()), (to_host(a) for a in c.bwd()[:3])
    first = [(0, 0), (0, 1)]
    for name, a, r, n, tol in (("O", o, ref[0], c.nq, FWD_TOL), ("dQ", dq, ref[1], c.nq, BWD_TOL), ("dK", dk, ref[2], c.nk, BWD_TOL), ("dV", dv, ref[3], c.nk, BWD_TOL)):
        check_slices(name, a, r, n, first, tol)
    assert not dq[1:].any() and not dk[1:].any()
    # weights of 2^-126 e^(score + table) each, scores below 6 and the table below 3: 300 x 33.3 x 6 of them
    assert np.abs(o[1:]).max() < 1e-29 and np.abs(dv[1:]).max() < 1e-29
