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
    (2, 400, 700, 1, (400, 333), (700, 650), 30, 32, (100, -60)),
    (70, 65, 65, 1, [65 - i % 66 for i in range(70)], [65 - i % 66 for i in range(70)], 20, 41, None),
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("op", ["rel", "dropout", "both"])
@pytest.mark.parametrize("shape", SMALL, ids=lambda s: f"{s[0]}x{s[1]}x{s[2]}r{s[6]}")
def test_parity(shape, op, d):
    B, Lq, Lk, H, nq, nk, reach, num, start = shape
    check(Case(B, Lq, Lk, H, d, nq, nk, op, reach, num, start, seed=d + len(op)))
