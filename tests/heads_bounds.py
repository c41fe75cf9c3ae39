"""Gradients of attention with heads from the definition alone, with bounds that hold for small gradients, long rows and biases far from zero, and
other operands for a problem of test_gpu_heads."""
import numpy as np

from heads_ref import FLOOR, HALF_STEP
from test_gpu_heads import near


def with_operands(a, X=None, Y=None, H=None, G=None):
    """The problem with other values in its operands (64 bits, rounded once here), and the reference of those."""
    import torch
    for name, v in dict(X=X, Y=Y, H=H, G=G).items():
        if v is not None:
            getattr(a, name).copy_(torch.from_numpy(np.ascontiguousarray(v)))
    a.ref.X, a.ref.Y, a.ref.H = a.f64(a.X), a.f64(a.Y), a.f64(a.H)
    return a


def gradients(a, out, l_off=0.0):
    """dX, dY, dH and dTable from the call's own out, probabilities from the definition; and bounds.  An entry of dS is rounded once (half a step of
    itself; what falls below the normal numbers is off by 2^-25 of a unit that is at most 2^-11 of the largest |dS| of its row of the
    product -- a row of A for dX, a column for dY -- so 2^-36 of that); sums of up to 128 products and the exponential's argument in fp32 as in
    the reference's own bounds (2^-15 of their magnitudes); sums of a row's entries in fp32 (2^-14); the result's rounding.
    l_off: a further relative error of a row's probabilities."""
    r, u, f = a.ref, HALF_STEP[a.dtype], FLOOR[a.dtype]
    G = a.f64(a.G)
    g = {"dX": np.zeros_like(r.X), "dY": np.zeros_like(r.Y), "dH": np.zeros_like(r.H)}
    if r.table is not None:
        g["dTable"] = np.zeros_like(r.table)
    e = {k: np.zeros_like(v) for k, v in g.items()}
    low = 2.0 ** -36 if a.dtype == "f16" else 0.0
    for h in range(r.heads):
        k = h // r.share
        x, y, v, go, o = r.X[:, h], r.Y[:, k], r.H[:, k], G[:, h], out[:, h]
        s, size = r.scores(h)
        top = s.max(1, keepdims=True)
        with np.errstate(invalid="ignore"):
            P = np.where(r.stored & np.isfinite(s), np.exp(s - top), 0.0)
        total = P.sum(1, keepdims=True)
        P = np.divide(P, total, out=np.zeros_like(P), where=total > 0)
        Z = r.Z[h] * r.stored
        D = (go * o).sum(1, keepdims=True)
        dS, W = P * (Z * (go @ v.T) - D), Z * P
        grow = 2.0 ** -15 * (1 + np.where(r.stored & np.isfinite(s), size, 0.0).max(1, keepdims=True)) + l_off
        rough = grow * P * (Z * (np.abs(go) @ np.abs(v).T) + (np.abs(go) * np.abs(o)).sum(1, keepdims=True))
        off, c = u * np.abs(dS) + rough, abs(r.scale)
        rows = off + 2.0 ** -14 * np.abs(dS) + low * (np.abs(dS) + rough).max(1, keepdims=True) * r.stored
        cols = off + 2.0 ** -14 * np.abs(dS) + low * (np.abs(dS) + rough).max(0, keepdims=True) * r.stored
        g["dX"][:, h], e["dX"][:, h] = r.scale * (dS @ y), c * (rows @ np.abs(y))
        g["dY"][:, k] += r.scale * (dS.T @ x)
        e["dY"][:, k] += c * (cols.T @ np.abs(x))
        g["dH"][:, k] += W.T @ go
        e["dH"][:, k] += ((u + grow + 2.0 ** -14) * W + f * Z / 4096).T @ np.abs(go)
        if r.table is not None:
            for b in range(r.table.shape[1]):
                mine = r.stored & (r.bucket == b)
                g["dTable"][h, b], e["dTable"][h, b] = dS[mine].sum(), rough[mine].sum() + 2.0 ** -14 * np.abs(dS[mine]).sum()
    return g, {k: e[k] + u * (np.abs(g[k]) + e[k]) + f for k in g}


def check_gradients(a, **kw):
    out, lse = a.forward()
    got = a.backward(out, lse)
    want, bound = gradients(a, a.f64(out), **kw)
    for k, t in zip(("dX", "dY", "dH", "dTable"), got):
        if t is not None:
            near(t, want[k], bound[k], k)
    return out, lse, got, want
