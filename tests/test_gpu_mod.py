"""GPU parity of the calls with a relative position bias, with dropout and with both, against 64 bits (mod_oracle.py).

Error bars as for the other calls (gpu_util.py): per (z, h) slice max |gpu - ref| / max |ref|, 1e-2 forward, 2e-2 backward.  dtable is
a sum of terms of either sign; its bar is that of dbias, 2e-2 (|ref| + sqrt(sum of dS^2 over the bucket))."""
import numpy as np
import pytest
import torch

import mod_oracle as M
from paper_2604_27124_amd import binding as A
from paper_2604_27124_amd import workloads as W
from gpu_util import BWD_TOL, FWD_TOL, check_slices, to_dev, to_host

pytestmark = pytest.mark.gpu


class Case:
    """Inputs of one call, in numpy and on the device.  Padded rows hold finite values."""

    def __init__(self, B, Lq, Lk, H, d, nq, nk, op="both", reach=9, num=8, start=None, p=0.2, seed=0, table_std=0.5, rng=(0x123456789ABCDEF, 11)):
        r = np.random.default_rng(seed)
        rows = lambda L: W.round_to_bf16(r.standard_normal((B, L, H, d)).astype(np.float32))
        self.q, self.k, self.v, self.g = rows(Lq), rows(Lk), rows(Lk), rows(Lq)
        self.nq, self.nk = np.array(nq, np.int32), np.array(nk, np.int32)
        self.bias = np.array([-np.log(max(1, min(n, Lk))) for n in self.nk], np.float32)
        self.scale = 1.0 / np.sqrt(d)
        self.op, self.p, self.rng = op, p, rng
        self.table = W.round_to_bf16((table_std * r.standard_normal((num, H))).astype(np.float32))
        self.buckets = A.sigmoid_attn_rel_buckets(num, reach).numpy()
        self.start = None if start is None else np.array(start, np.int32)

    def upload(self):
        ints = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
        self.t = dict(q=to_dev(self.q), k=to_dev(self.k), v=to_dev(self.v), g=to_dev(self.g), nq=ints(self.nq), nk=ints(self.nk), bias=ints(self.bias),
                      table=to_dev(self.table), buckets=ints(self.buckets), start=None if self.start is None else ints(self.start),
                      rng=torch.tensor(self.rng, dtype=torch.int64, device="cuda"))
        return self

    def args(self):
        t = self.t
        common = (t["nq"], t["nk"], t["bias"], self.scale)
        rel = (t["table"], t["buckets"]) if self.op != "dropout" else ()
        drop = (self.p, t["rng"]) if self.op != "rel" else ()
        kw = {} if self.op == "dropout" else {"q_start": t["start"]}
        return common + rel + drop, kw

    def name(self):
        return {"rel": "sigmoid_attn_rel", "dropout": "sigmoid_attn_dropout", "both": "sigmoid_attn_rel_dropout"}[self.op]

    def fwd(self, **more):
        a, kw = self.args()
        t = self.t
        return getattr(A, self.name() + "_fwd")(t["q"], t["k"], t["v"], *a, **kw, **more)

    def bwd(self, **more):
        a, kw = self.args()
        t = self.t
        return getattr(A, self.name() + "_bwd")(t["q"], t["k"], t["v"], t["g"], *a, **kw, **more)

    def reference(self, **changed):
        g = lambda n: changed.get(n, getattr(self, n))
        rel = dict(table=g("table"), buckets=self.buckets, start=self.start) if self.op != "dropout" else {}
        drop = dict(p=self.p, rng=self.rng) if self.op != "rel" else {}
        return M.batch(g("q"), g("k"), g("v"), g("g"), self.nq, self.nk, self.bias, self.scale, **rel, **drop)

    def ds_squares(self):
        """sum of dS^2 by bucket and head."""
        out = np.zeros(self.table.shape)
        B, Lq, H, d = self.q.shape
        for z in range(B):
            n, m = (min(max(int(x), 0), L) for x, L in ((self.nq[z], Lq), (self.nk[z], self.k.shape[1])))
            R = (len(self.buckets) - 1) // 2
            away = np.arange(m)[None] - np.arange(n)[:, None] - (0 if self.start is None else int(self.start[z]))
            which = np.clip(self.buckets[np.clip(away, -R, R) + R], 0, len(self.table) - 1)
            for h in range(H):
                x = self.scale * self.q[z, :n, h].astype(np.float64) @ self.k[z, :m, h].T.astype(np.float64) + self.bias[z] + self.table[:, h].astype(np.float64)[which]
                ds = M.sigma(x) * M.sigma(-x) * (self.g[z, :n, h].astype(np.float64) @ self.v[z, :m, h].T.astype(np.float64))
                if self.op == "both" and M.kept(self.p) < 65536:
                    ds = ds * M.mask(*self.rng, z * H + h, n, m, self.p) * 65536 / M.kept(self.p)
                out[:, h] += np.bincount(which.ravel(), weights=(ds * ds).ravel(), minlength=len(out))
        return out


def poisoned(t):
    return torch.full_like(t, float("nan"))


def check(c, ref=None):
    """Forward and backward into poisoned outputs, twice (the same bits), against the oracle."""
    c.upload()
    t = c.t
    o = c.fwd(out=poisoned(t["q"]))
    outs = dict(dq=poisoned(t["q"]), dk=poisoned(t["k"]), dv=poisoned(t["v"]))
    if c.op != "dropout":
        outs["dtable"] = poisoned(t["table"])
    got = c.bwd(**outs)
    torch.cuda.synchronize()
    for a, b in zip((o, *got), (c.fwd(), *c.bwd())):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16)), "another run, other bits"
    torch.cuda.synchronize()
    ref = ref or c.reference()
    B, H = c.q.shape[0], c.q.shape[2]
    slices = [(z, h) for z in range(B) for h in range(H)]
    nq, nk = np.clip(c.nq, 0, c.q.shape[1]), np.clip(c.nk, 0, c.k.shape[1])
    worst = [check_slices("O", to_host(o), ref[0], nq, slices, FWD_TOL)]
    for name, a, r, n in (("dQ", got[0], ref[1], nq), ("dK", got[1], ref[2], nk), ("dV", got[2], ref[3], nk)):
        worst.append(check_slices(name, to_host(a), r, n, slices, BWD_TOL))
    if c.op != "dropout":
        off = np.abs(to_host(got[3]).astype(np.float64) - ref[4])
        bar = BWD_TOL * (np.abs(ref[4]) + np.sqrt(c.ds_squares()))
        worst.append(float(np.max(off / np.maximum(bar, 1e-300) * (off > 0))))
        assert np.all(off <= bar), f"dtable: {off.max()} at {np.argwhere(off > bar)[:5]}"
    print("errors", [f"{x:.1e}" for x in worst], flush=True)


SMALL = [
    # B, Lq, Lk, H, nq, nk, reach, buckets, q_start
    (2, 70, 70, 2, (70, 33), (70, 33), 9, 8, None),
    (3, 33, 200, 2, (33, 1, 0), (200, 77, 50), 40, 16, None),
    (3, 200, 45, 1, (200, 130, 64), (45, 0, 1), 300, 32, (0, 5, -70)),
    (2, 1, 300, 3, (1, 1), (300, 257), 64, 32, (299, 256)),
    (1, 257, 129, 2, (257,), (129,), 0, 1, (1000,)),
    (2, 129, 321, 1, (129, 128), (320, 321), 1, 3, (-1000000, 17)),
    (1, 513, 513, 1, (513,), (513,), 128, 32, None),
    (2, 5, 3000, 1, (5, 3), (2999, 2047), 500, 64, (2994, 0)),
    (3, 8, 131, 3, (8, 7, 0), (131, 128, 5), 30, 12, (123, -4, 0)),
    (2, 2, 64, 2, (2, 1), (0, 64), 3, 5, None),
    (1, 13, 2500, 2, (11,), (2400,), 100, 32, (-3,)),
    (2, 64, 1100, 1, (64, 37), (1100, 1025), 200, 32, (1036, 0)),
    (2, 400, 700, 1, (400, 333), (700, 650), 30, 32, (100, -60)),
    (40, 150, 90, 7, [150 - 3 * i for i in range(40)], [90 - 2 * i for i in range(40)], 30, 32, None),   # two query blocks a wave
    (40, 6, 90, 7, [6 - i % 7 for i in range(40)], [90 - 2 * i for i in range(40)], 30, 32, [84 - 3 * i for i in range(40)]),   # many heads of few queries
    (70, 65, 65, 1, [65 - i % 66 for i in range(70)], [65 - i % 66 for i in range(70)], 20, 41, None),
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("op", ["rel", "dropout", "both"])
@pytest.mark.parametrize("shape", SMALL, ids=lambda s: f"{s[0]}x{s[1]}x{s[2]}r{s[6]}")
def test_parity(shape, op, d):
    B, Lq, Lk, H, nq, nk, reach, num, start = shape
    check(Case(B, Lq, Lk, H, d, nq, nk, op, reach, num, start, seed=d + len(op)))


def same_bits(a, b):
    return torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("Lq", [3, 90])
@pytest.mark.parametrize("low", [float("-inf"), -3.3895313892515355e38])
def test_an_entry_of_minus_infinity_masks_its_pairs(Lq, low):
    # all distances but 0..2 are masked; the queries from 40 on see no key at all
    c = Case(2, Lq, 40, 2, 64, (Lq, Lq - 1), (40, 33), "rel", 5, 11, None, seed=3)
    c.table[:] = low
    c.table[5:8] = 0.25
    ref = c.reference(table=np.where(c.table < -1e30, -np.inf, c.table).astype(np.float64))
    assert Lq < 40 or np.all(ref[0][:, 41:] == 0)
    check(c, ref)
    if Lq > 16:
        dtable = to_host(c.bwd()[3])
        masked = np.ones(len(c.table), bool)
        masked[5:8] = False
        assert np.all(dtable[masked] == 0) and np.all(to_host(c.fwd())[:, 42:] == 0)


@pytest.mark.parametrize("op,d,Lq", [("rel", 64, 70), ("both", 64, 70), ("rel", 128, 70), ("rel", 64, 5)])
def test_what_only_padding_reaches_has_no_influence(op, d, Lq):
    # NaN and Inf in padded rows, NaN in table entries of distances that no valid pair has
    c = Case(2, Lq, 130, 2, d, (min(Lq, 41), 3), (77, 50), op, 129, 259, None, seed=9).upload()
    want = [t.clone() for t in (c.fwd(), *c.bwd())]
    t = c.t
    for n, (lens, names) in enumerate(((c.nq, ("q", "g")), (c.nk, ("k", "v")))):
        for name in names:
            for z in range(2):
                t[name][z, int(lens[z]):] = float("nan") if z else float("inf")
    t["table"][:129 - 40] = float("nan")                                   # distances below -40
    t["table"][129 + 77:] = float("nan")                                   # and above 76
    for a, b in zip((c.fwd(), *c.bwd()), want):
        assert same_bits(a, b)
    # a NaN that valid pairs do reach shows
    t["table"][129] = float("nan")
    assert bool(torch.isnan(c.fwd()).any())


def test_an_infinite_key_leaves_the_table_gradient_finite():
    # P is 0 or 1 against it and dS 0; padded queries of its tile have scores 0 x Inf
    c = Case(1, 50, 64, 1, 64, (37,), (64,), "rel", 7, 15, None, seed=5)
    c.k[0, 20, 0, 3] = np.inf
    with np.errstate(invalid="ignore"):
        ref = c.reference()
        squares = c.ds_squares()
    c.upload()
    dtable = to_host(c.bwd()[3])
    assert np.all(np.isfinite(ref[4])) and np.all(np.abs(dtable - ref[4]) <= BWD_TOL * (np.abs(ref[4]) + np.sqrt(squares)))


def test_buckets_out_of_range_are_clamped():
    c = Case(1, 60, 60, 2, 64, (60,), (60,), "rel", 3, 4, None, seed=6)
    c.buckets[:] = (-7, 0, 1, 99, 2, 3, 2 ** 31 - 1)
    check(c)


@pytest.mark.parametrize("Lq", [4, 300])
@pytest.mark.parametrize("scale", [0.0, -0.2, 1e-30])
def test_other_scales(scale, Lq):
    c = Case(2, Lq, 200, 2, 64, (Lq, Lq // 2), (200, 77), "rel" if Lq < 17 else "both", 40, 8, None, seed=7)
    c.scale = scale
    check(c)


@pytest.mark.parametrize("op", ["dropout", "both"])
def test_no_dropout_and_nearly_all(op):
    c = Case(2, 90, 70, 2, 64, (90, 33), (70, 64), op, 9, 8, None, p=0.0, seed=8).upload()
    t = c.t
    common = (t["nq"], t["nk"], t["bias"], c.scale)
    plain = A.sigmoid_attn_cross_fwd(t["q"], t["k"], t["v"], *common) if op == "dropout" else \
        A.sigmoid_attn_rel_fwd(t["q"], t["k"], t["v"], *common, t["table"], t["buckets"])
    assert same_bits(c.fwd(), plain)
    c.p = 1e-6                                                             # rounds to none
    assert same_bits(c.fwd(), plain)
    check(Case(1, 130, 130, 1, 64, (130,), (130,), op, 9, 8, None, p=0.97, seed=8))
    c.p = 1.0 - 2.0 ** -24                                                 # one weight of 65536 stays at least: finite
    assert bool(torch.isfinite(c.fwd()).all())


def test_seed_and_offset():
    c = Case(1, 64, 96, 2, 64, (64,), (96,), "dropout", seed=10, rng=(-5, 2 ** 40 + 3)).upload()
    check(c)
    base = c.fwd()
    c.t["rng"].copy_(torch.tensor([-5, 3]))                                # the offset counts modulo 2^32
    assert same_bits(c.fwd(), base)
    for other in ((-5, 4), (-6, 3), (-5 + 2 ** 32, 3)):
        c.t["rng"].copy_(torch.tensor(other))
        assert not same_bits(c.fwd(), base)


def test_share_of_weights_that_stay():
    # V of ones and P of one half everywhere: O counts what stays
    B, N, H, d, p = 2, 1024, 3, 64, 0.1
    z = torch.zeros(B, N, H, d, dtype=torch.bfloat16, device="cuda")
    n, b = torch.full((B,), N, dtype=torch.int32, device="cuda"), torch.zeros(B, device="cuda")
    o = A.sigmoid_attn_dropout_fwd(z, z, torch.ones_like(z), n, n, b, 1.0, p, torch.tensor([7, 0], device="cuda"))[..., 0].double()
    keep = M.kept(p) / 65536
    # mean of N^2 H B decisions, and 2^-9 for the rounding of each O, which has no preferred direction (six deviations of either)
    assert abs(float(o.mean()) * keep * 2 / N - keep) < 6 * np.sqrt(keep * (1 - keep) / (B * H * N * N)) + 6 * 2.0 ** -9 / np.sqrt(B * H * N)


@pytest.mark.parametrize("op", ["rel", "dropout", "both"])
@pytest.mark.parametrize("d", [64, 128])
def test_a_sequence_does_not_depend_on_its_batch(op, d):
    # bias, alone in the batch and among others: the same bits (with dropout the mask goes by the place in the batch)
    c = Case(3, 300, 300, 2, d, (300, 200, 131), (300, 200, 131), op, 40, 16, None, seed=12).upload()
    one = Case(1, 300, 300, 2, d, (300,), (300,), op, 40, 16, None, seed=12)
    one.__dict__.update({n: getattr(c, n)[:1] for n in ("q", "k", "v", "g", "nq", "nk", "bias")}, table=c.table, buckets=c.buckets)
    one.upload()
    for a, b in zip((c.fwd(), *c.bwd()[:3]), (one.fwd(), *one.bwd()[:3])):
        assert same_bits(a[:1], b)


@pytest.mark.parametrize("op", ["rel", "dropout", "both"])
@pytest.mark.parametrize("Lq", [2, 100])
def test_other_streams_and_the_python_way(op, Lq):
    c = Case(2, Lq, 3000, 2, 64, (Lq, 1), (3000, 2048), op, 100, 32, (2900, 0), seed=13).upload()
    want = (c.fwd(), *c.bwd())                                             # native calls
    here = torch.cuda.current_stream()
    for a, b in zip((c.fwd(stream=here), *c.bwd(stream=here)), want):      # marshalled in Python
        assert same_bits(a, b)
    side = torch.cuda.Stream()
    side.wait_stream(here)
    outs = [poisoned(x) for x in want]
    names = ("dq", "dk", "dv", "dtable")
    c.fwd(out=outs[0], stream=side)
    c.bwd(**dict(zip(names, outs[1:])), stream=side)
    with torch.cuda.stream(side):
        again = (c.fwd(), *c.bwd())
    torch.cuda.synchronize()
    for got in (outs, again):
        for a, b in zip(got, want):
            assert same_bits(a, b)


def test_few_queries_with_and_without_a_workspace():
    c = Case(1, 7, 5000, 2, 64, (7,), (4900,), "rel", 100, 32, (4893,), seed=14).upload()
    need = A.sigmoid_attn_rel_fwd_workspace_bytes(1, 7, 5000, 2, 64)
    assert need > 0 and A.sigmoid_attn_rel_fwd_workspace_bytes(64, 7, 5000, 12, 64) == 0
    split, whole = c.fwd(workspace=torch.empty(need, dtype=torch.uint8, device="cuda")), c.fwd(workspace=torch.empty(0, device="cuda"))
    assert same_bits(split, c.fwd())
    ref = c.reference()[0]
    for o in (split, whole):
        # fp32 throughout: half a bf16 step of the value, and sums of 4900 fp32 terms
        assert np.all(np.abs(to_host(o) - ref) <= 2.0 ** -8 * np.abs(ref) + 1e-5 * np.abs(ref).max())


@pytest.mark.parametrize("d", [64, 128])
def test_a_step_in_a_hip_graph(d):
    """Bias and dropout captured and replayed, with another offset each time; the workspace and outputs are the program's."""
    c = Case(2, 300, 260, 2, d, (300, 131), (260, 77), "both", 60, 32, None, seed=15).upload()
    t = c.t
    ws = torch.empty(A.sigmoid_attn_rel_bwd_workspace_bytes(2, 300, 260, 2, d, 60), dtype=torch.uint8, device="cuda")
    outs = dict(dq=poisoned(t["q"]), dk=poisoned(t["k"]), dv=poisoned(t["v"]), dtable=poisoned(t["table"]))
    o = poisoned(t["q"])
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.fwd(out=o), c.bwd(**outs, workspace=ws)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            c.fwd(out=o), c.bwd(**outs, workspace=ws)
    torch.cuda.synchronize()
    for replay in range(4):
        t["rng"][1] = 100 + replay
        for x in (o, *outs.values()):
            x.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((o, *outs.values()), (c.fwd(), *c.bwd())):
            assert same_bits(a, b), replay


def test_two_calls_at_once_with_workspaces_of_their_own():
    a, b = (Case(2, 400, 400, 2, 64, (400, 300), (400, 300), "both", 50, 16, None, seed=s).upload() for s in (16, 17))
    want = [(x.fwd(), *x.bwd()) for x in (a, b)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for x, s in zip((a, b), streams):
        with torch.cuda.stream(s):
            got.append((x.fwd(), *x.bwd()))
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        for x, y in zip(g, w):
            assert same_bits(x, y)


@pytest.mark.parametrize("Lq", [1, 20])
def test_offsets_beyond_32_bits(Lq):
    """A context of 4.5 GB a tensor: the last rows lie behind 2^32 bytes."""
    H, d, Lk = 16, 128, 1100000
    gen = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.empty(1, Lk, H, d, dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for _ in range(2))
    q = torch.empty(1, Lq, H, d, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    table = torch.empty(8, H, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    buckets, start = A.sigmoid_attn_rel_buckets(8, 30).cuda(), torch.tensor([Lk - Lq], dtype=torch.int32, device="cuda")
    nq, nk = torch.tensor([Lq], dtype=torch.int32, device="cuda"), torch.tensor([Lk], dtype=torch.int32, device="cuda")
    bias, scale = torch.tensor([-8.0], device="cuda"), d ** -0.5
    o = A.sigmoid_attn_rel_fwd(q, k, v, nq, nk, bias, scale, table, buckets, q_start=start)
    away = torch.arange(Lk, device="cuda")[None] - torch.arange(Lq, device="cuda")[:, None] - (Lk - Lq)
    which = buckets.long()[away.clamp(-30, 30) + 30]
    for h in (0, H - 1):
        x = scale * (q[0, :, h].double() @ k[0, :, h].double().t().contiguous()) - 8.0 + table[:, h].double()[which]
        ref = torch.sigmoid(x) @ v[0, :, h].double()
        assert float((o[0, :, h].double() - ref).abs().max() / ref.abs().max()) < FWD_TOL


def test_refusals():
    c = Case(2, 30, 40, 2, 64, (30, 3), (40, 4), seed=18).upload()
    t, common = c.t, (c.t["nq"], c.t["nk"], c.t["bias"], c.scale)
    q, k, v, g = t["q"], t["k"], t["v"], t["g"]
    fine = dict(table=t["table"], buckets=t["buckets"])
    for bad in (dict(table=t["table"].float()), dict(table=t["table"].t()), dict(table=t["table"][:, :1]), dict(buckets=t["buckets"][:-1]),
                dict(buckets=t["buckets"].long()), dict(buckets=t["buckets"].cpu()), dict(q_start=t["nq"][:1]), dict(out=k), dict(out=q.float())):
        with pytest.raises(ValueError):
            A.sigmoid_attn_rel_fwd(q, k, v, *common, **{**fine, **bad})
    for bad in (dict(dtable=t["table"].float()), dict(dq=k), dict(dk=q)):
        with pytest.raises(ValueError):
            A.sigmoid_attn_rel_bwd(q, k, v, g, *common, **{**fine, **bad})
    with pytest.raises(A.SigAttnError) as e:
        A.sigmoid_attn_rel_bwd(q, k, v, g, *common, **fine, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert e.value.code == A.SIGATTN_ERR_WORKSPACE
    for p, rng in ((1.0, t["rng"]), (-0.1, t["rng"]), (float("nan"), t["rng"])):
        with pytest.raises(A.SigAttnError):
            A.sigmoid_attn_dropout_fwd(q, k, v, *common, p, rng)
    for rng in (t["rng"].int(), t["rng"][:1], t["rng"].cpu()):
        with pytest.raises(ValueError):
            A.sigmoid_attn_dropout_fwd(q, k, v, *common, 0.1, rng)
    with pytest.raises(ValueError):
        A.sigmoid_attn_dropout_fwd(q.transpose(1, 2), k, v, *common, 0.1, t["rng"])


@pytest.mark.parametrize("op", ["rel", "dropout", "both"])
def test_many_runs_of_large_tiles_give_the_same_bits(op):
    # forward with two query blocks a wave: every store's data are those of the store
    c = Case(8, 1000, 1000, 12, 64, [1000 - 37 * i for i in range(8)], [1000 - 37 * i for i in range(8)], op, 60, 32, None, seed=20).upload()
    first = c.fwd()
    assert bool(torch.isfinite(first).all()) and float(first.float().abs().max()) < 10
    for _ in range(40):
        assert same_bits(c.fwd(), first)


@pytest.mark.parametrize("op", ["rel", "dropout", "both"])
def test_many_short_sequences(op):
    # batch order in both directions, more sequences than a wave ranks
    lens = [(13 * i) % 41 for i in range(150)]
    check(Case(150, 40, 40, 2, 64, lens, lens, op, 12, 9, None, seed=21))


def test_what_the_workspace_held_does_not_matter():
    c = Case(3, 300, 400, 2, 64, (300, 0, 131), (400, 77, 33), "rel", 100, 32, (7, 0, -50), seed=22).upload()
    want = c.bwd()
    n = A.sigmoid_attn_rel_bwd_workspace_bytes(3, 300, 400, 2, 64, 100)
    ws = torch.full((n // 4,), float("nan"), device="cuda")
    for a, b in zip(c.bwd(workspace=ws), want):
        assert same_bits(a, b)
    guard = torch.full((n // 4 + 1024,), 3.0, device="cuda")                # nothing behind its end is written
    c.bwd(workspace=guard[:n // 4])
    assert bool((guard[n // 4:] == 3.0).all())
