"""Attention with heads, a bucket bias and dropout, its gradients, and the same on value arrays, in 64 bits on the CPU, with how far a
result in 16 bits may be off.  Dense and plain: meant for small matrices."""
import math

import numpy as np

HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}      # of a rounding, relative to the value
FLOOR = {"f16": 2.0 ** -25, "bf16": 2.0 ** -134}        # and below the normal numbers
ROTATIONS = (13, 15, 26, 6, 17, 29, 16, 24)


def threefry(key, c0, c1, rounds):
    """Threefry-2x32 (Salmon, Moraes, Dror, Shaw 2011) in Python's and numpy's 64-bit integers."""
    M = 0xFFFFFFFF
    ks = (key[0], key[1], key[0] ^ key[1] ^ 0x1BD11BDA)
    a, b = (c0 + ks[0]) & M, (c1 + ks[1]) & M
    for i in range(rounds):
        a = (a + b) & M
        r = ROTATIONS[i % 8]
        b = ((b << r & M) | (b >> (32 - r))) ^ a
        if i % 4 == 3:
            n = i // 4 + 1
            a, b = (a + ks[n % 3]) & M, (b + ks[(n + 1) % 3] + n) & M
    return a, b


def keep_factors(heads, M, K, p, state):
    """(heads, M, K): 1 / (1 - p) where an entry is kept, else 0."""
    if not p:
        return np.ones((heads, M, K))
    seed, step = (int(v) & 0xFFFFFFFFFFFFFFFF for v in state)
    key = threefry((seed & 0xFFFFFFFF, seed >> 32), step & 0xFFFFFFFF, step >> 32, 20)
    row, col = np.arange(M, dtype=np.int64)[:, None], np.arange(K, dtype=np.int64)[None]
    z = np.zeros((heads, M, K))
    for h in range(heads):
        word = threefry(threefry(key, h, 0, 20), row, col, 13)[0]
        z[h] = np.where(word >= math.floor(p * 2.0 ** 32), 1 / (1 - p), 0.0)
    return z


def bucket_of(M, K, buckets, shift, n_buckets):
    """(M, K): the bucket of every position."""
    reach = len(buckets) // 2
    r = np.arange(K, dtype=np.int64)[None] - np.arange(M, dtype=np.int64)[:, None] - shift
    return np.minimum(np.asarray(buckets, dtype=np.int64)[np.clip(r, -reach, reach) + reach], n_buckets - 1)


class Attention:
    """X (M, heads, d), Y (K, kv, d), H (K, kv, N) and table (heads, buckets) in 64 bits; stored: (M, K) truth values."""

    def __init__(self, stored, X, Y, H, scale, table=None, buckets=None, shift=0, p=0.0, state=(0, 0), dtype="f16"):
        self.stored, self.X, self.Y, self.H, self.scale, self.table, self.dtype = stored, X, Y, H, scale, table, dtype
        self.heads, self.share = X.shape[1], X.shape[1] // Y.shape[1]
        M, K = stored.shape
        self.Z = keep_factors(self.heads, M, K, p, state)
        self.bucket = None if table is None else bucket_of(M, K, buckets, shift, table.shape[1])

    def scores(self, h):
        """(s, size): the scores, minus infinity where nothing is stored, and the sum of the magnitudes that make them."""
        x, y = self.X[:, h], self.Y[:, h // self.share]
        b = 0.0 if self.table is None else self.table[h][self.bucket]
        size = abs(self.scale) * (np.abs(x) @ np.abs(y).T) + np.where(np.isfinite(b), np.abs(b), 0.0)
        return np.where(self.stored, self.scale * (x @ y.T) + b, -np.inf), size

    def forward(self):
        """out, lse, and the bounds of their errors: two half steps (a probability's rounding and the result's) of the magnitudes
        that are added; a probability below fp16's normal numbers, relative to the largest of its row, is off by up to 2^-25; sums of d <= 128
        products in fp32 are off by 2^-17 of their magnitudes, which the exponential passes on."""
        u, f = HALF_STEP[self.dtype], FLOOR[self.dtype]
        out, lse, eo, el = [], [], [], []
        for h in range(self.heads):
            v = self.H[:, h // self.share]
            s, size = self.scores(h)
            top = s.max(1, keepdims=True, initial=-np.inf)
            e = np.where(np.isfinite(s), np.exp(s - np.where(np.isfinite(top), top, 0.0)), 0.0)
            total = e.sum(1, keepdims=True)
            w = np.divide(e, total, out=np.zeros_like(e), where=total > 0)
            with np.errstate(divide="ignore"):
                lse.append((top + np.log(total))[:, 0])
            A = np.where(self.stored, size, 0.0).max(1, keepdims=True, initial=0.0)
            grow = 2.0 ** -16 * (1 + A)
            out.append((w * self.Z[h]) @ v)
            S = (w * self.Z[h]) @ np.abs(v)
            small = np.where((self.Z[h] > 0) & self.stored, self.Z[h], 0.0) @ np.abs(v)
            eo.append((2 * u + u * u + 2 * grow) * S + f * small / np.maximum(total, 1.0) + f)
            el.append((grow + 2.0 ** -22 * np.abs(np.where(np.isfinite(lse[-1]), lse[-1], 0.0))[:, None])[:, 0])
        return np.stack(out, 1), np.stack(lse), np.stack(eo, 1), np.stack(el)

    def backward(self, out, lse, G):
        """Gradients from the out and lse that the call is given, and bounds: the roundings of dS and Z P, of the result, and the
        scores' error as above."""
        u, f = HALF_STEP[self.dtype], FLOOR[self.dtype]
        kv = self.Y.shape[1]
        g = {"dX": np.zeros_like(self.X), "dY": np.zeros_like(self.Y), "dH": np.zeros_like(self.H)}
        e = {k: np.zeros_like(v) for k, v in g.items()}
        if self.table is not None:
            g["dTable"], e["dTable"] = np.zeros_like(self.table), np.zeros_like(self.table)
        for h in range(self.heads):
            k = h // self.share
            x, y, v, go = self.X[:, h], self.Y[:, k], self.H[:, k], G[:, h]
            s, size = self.scores(h)
            l = lse[h][:, None]
            P = np.where(np.isfinite(s), np.exp(s - np.where(np.isfinite(l), l, 0.0)), 0.0) * self.stored
            D = (go * out[:, h]).sum(1, keepdims=True)
            Z = self.Z[h] * self.stored
            dS = P * (Z * (go @ v.T) - D)
            A = np.where(self.stored, size, 0.0).max(1, keepdims=True, initial=0.0)
            grow = 2.0 ** -15 * (1 + A)  # of P, and of the two products of up to 128 terms
            rough = grow * P * (Z * (np.abs(go) @ np.abs(v).T) + (np.abs(go) * np.abs(out[:, h])).sum(1, keepdims=True))
            off = u * np.abs(dS) + rough + f * self.stored  # of an entry of dS as the products take it
            a = abs(self.scale)
            g["dX"][:, h] = self.scale * (dS @ y)
            e["dX"][:, h] = a * (off @ np.abs(y)) + 2.0 ** -14 * a * (np.abs(dS) @ np.abs(y))
            g["dY"][:, k] += self.scale * (dS.T @ x)
            e["dY"][:, k] += a * (off.T @ np.abs(x)) + 2.0 ** -14 * a * (np.abs(dS).T @ np.abs(x))
            W = Z * P
            g["dH"][:, k] += W.T @ go
            e["dH"][:, k] += ((u + grow + 2.0 ** -14) * W + f * Z / 4096).T @ np.abs(go)
            if self.table is not None:
                for b in range(self.table.shape[1]):
                    mine = self.stored & (self.bucket == b)
                    g["dTable"][h, b] = dS[mine].sum()
                    e["dTable"][h, b] = rough[mine].sum() + 2.0 ** -14 * np.abs(dS[mine]).sum()
        assert kv == self.H.shape[1]
        return g, {k: e[k] + u * (np.abs(g[k]) + e[k]) + f for k in g}
