"""Attention with a relative position bias and with dropout, in 64 bits on the CPU, from the definitions: the oracle of these calls' tests.
Single heads as plain numpy; no code of the library."""
import numpy as np

M32 = np.uint64(0xFFFFFFFF)


def philox(counter, key, rounds):
    """Philox4x32 (Salmon, Moraes, Dror, Shaw 2011): four words from a counter of four and a key of two."""
    c = [np.asarray(x, dtype=np.uint64) for x in counter]
    k = [np.uint64(x) for x in key]
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ k[0], b & M32, (a >> np.uint64(32)) ^ c[3] ^ k[1], a & M32]
        k = [(k[0] + np.uint64(0x9E3779B9)) & M32, (k[1] + np.uint64(0xBB67AE85)) & M32]
    return c


def kept(p):
    return max(1, int(np.floor((1.0 - np.float64(np.float32(p))) * 65536 + 0.5)))


def mask(seed, offset, zh, n, m, p):
    """[n, m] truth values of what stays."""
    i, j = np.meshgrid(np.arange(n, dtype=np.uint64), np.arange(m, dtype=np.uint64), indexing="ij")
    two, four, eight, all32 = (np.uint64(x) for x in (2, 4, 8, 32))
    counter = (i, two * (j // all32) + (j // four) % two, np.full_like(i, zh), np.full_like(i, offset & 0xFFFFFFFF))
    r = philox(counter, (seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF), 7)
    t = two * ((j % all32) // eight) + (j // two) % two + np.uint64(16) * (j % two)
    u = np.zeros_like(i)
    for s in range(8):
        shift = np.uint64(8 * (s % 2))
        u += ((r[s // 2] >> (t + shift)) & np.uint64(1)) << np.uint64(8 + s)
        u += ((r[s // 2] >> ((t ^ np.uint64(16)) + shift)) & np.uint64(1)) << np.uint64(7 - s)
    return u + np.uint64(kept(p)) >= np.uint64(65536)


def sigma(x):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-x))


def head(q, k, v, d_o, bias, scale, column=None, buckets=None, start=0, keep=None, share=1.0):
    """One (z, h) slice over its valid rows: O, dQ, dK, dV and the gradient of the table's column (None without a table)."""
    q, k, v = (np.asarray(a, dtype=np.float64) for a in (q, k, v))
    x = scale * (q @ k.T) + float(bias)
    which = None
    if column is not None:
        column = np.asarray(column, dtype=np.float64)
        R = (len(buckets) - 1) // 2
        away = np.arange(len(k))[None, :] - np.arange(len(q))[:, None] - int(start)
        which = np.clip(buckets[np.clip(away, -R, R) + R], 0, len(column) - 1)
        x = x + column[which]
    p = sigma(x)
    w = p if keep is None else p * keep / share
    o = w @ v
    if d_o is None:
        return o, None, None, None, None
    d_o = np.asarray(d_o, dtype=np.float64)
    ds = p * sigma(-x) * (d_o @ v.T)
    if keep is not None:
        ds = ds * keep / share
    dcol = None if column is None else np.bincount(which.ravel(), weights=ds.ravel(), minlength=len(column))
    return o, scale * (ds @ k), scale * (ds.T @ q), w.T @ d_o, dcol


def batch(q, k, v, d_o, nq, nk, bias, scale, table=None, buckets=None, start=None, p=None, rng=None):
    """All slices of [B, L, H, d] arrays: (O, dQ, dK, dV, dtable); padded rows are zeros."""
    B, Lq, H, d = q.shape
    Lk = k.shape[1]
    o, dq, dk, dv = np.zeros(q.shape), np.zeros(q.shape), np.zeros(k.shape), np.zeros(k.shape)
    dtable = None if table is None else np.zeros(table.shape)
    for z in range(B):
        n, m = min(max(int(nq[z]), 0), Lq), min(max(int(nk[z]), 0), Lk)
        for h in range(H):
            keep, share = None, 1.0
            if p is not None and kept(p) < 65536:
                keep, share = mask(rng[0], rng[1], z * H + h, n, m, p), kept(p) / 65536.0
            r = head(q[z, :n, h], k[z, :m, h], v[z, :m, h], None if d_o is None else d_o[z, :n, h], bias[z], scale,
                     None if table is None else table[:, h], buckets, 0 if start is None else start[z], keep, share)
            o[z, :n, h] = r[0]
            if d_o is not None:
                dq[z, :n, h], dk[z, :m, h], dv[z, :m, h] = r[1:4]
                if table is not None:
                    dtable[:, h] += r[4]
    return o, dq, dk, dv, dtable
