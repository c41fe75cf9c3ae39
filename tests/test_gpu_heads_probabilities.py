"""Attention with heads: what its probabilities keep on the way to the matrix cores."""
import numpy as np
import pytest

from heads_bounds import gradients, with_operands
from heads_ref import FLOOR, HALF_STEP
from test_gpu_heads import Problem, fs, near  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [4, 8, 16])
@pytest.mark.parametrize("chunk", [0, 64])
def test_probabilities_below_fp16_beside_a_sink(fs, V, chunk):  # noqa: F811
    """A sink takes nearly all of a row and its row of H is zero; what is left are 16384 probabilities of about 1.5e-8, half of fp16's smallest
    number.  A probability is off by half a step of its rest, 2^-22 of itself, or by 2^-37 below the normal numbers (it is held times 2^12);
    a score and the sums as in the reference."""
    M, K = 5, 16385
    a = Problem(fs, 34, M, K, 1, 1, 16, 16, "f16", kind="dense", V=V, V_t=8, chunk=chunk)
    rng = np.random.default_rng(4)
    X, Y = np.zeros((M, 1, 16)), 0.01 * rng.standard_normal((K, 1, 16))
    X[:, :, 0], Y[:, :, 0], Y[7, :, 0] = 4.0, 0.0, 18.0  # scale 1/4: the sink's score is 18
    H = 8 + rng.random((K, 1, 16))
    H[7] = 0.0
    with_operands(a, X=X, Y=Y, H=H)
    out, lse = a.forward()
    want, wl, _, el = a.ref.forward()
    r, u = a.ref, HALF_STEP["f16"]
    s, size = r.scores(0)
    e = np.exp(s - s.max(1, keepdims=True))
    S = (e / e.sum(1, keepdims=True)) @ np.abs(r.H[:, 0])
    few = np.abs(r.H[:, 0]).sum(0) / e.sum(1, keepdims=True)
    grow = 2.0 ** -16 * (1 + size.max(1, keepdims=True))
    near(a.f64(out)[:, 0], want[:, 0], u * np.abs(want[:, 0]) + (u * u + 2 * grow) * S + 2.0 ** -37 * few + FLOOR["f16"], "out")
    near(a.f64(lse), wl, el, "lse")
    assert (want > 1e-3).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("V", [4, 8, 16])
def test_probabilities_meet_values_in_two_numbers(fs, dtype, V):  # noqa: F811
    """Columns of H whose sums under the probabilities cancel: one rounding of a probability would show as half a step of what is added, two as half a
    step of that.  The scores are small, so fp32 gives 2^-15 of it.  The gradient of the bias, whose D = g . out cancels with out, against the
    reference's own out: a row's D is off by the bound of out times |g|, its entries of dS by that times P."""
    import torch
    M, K, N = 64, 5, 64
    a = Problem(fs, 35, M, K, 1, 1, 16, N, dtype, kind="dense", bias=(5, 64), V=V, V_t=V)
    rng = np.random.default_rng(5)
    # every row has the same scores, so the same columns of H cancel in all of them
    with_operands(a, X=np.broadcast_to(0.3 * rng.standard_normal((1, 1, 16)), (M, 1, 16)), Y=0.3 * rng.standard_normal((K, 1, 16)))
    a.bias.table.zero_()
    a.ref.table = a.f64(a.bias.table)
    s, _ = a.ref.scores(0)
    P = np.exp(s - s.max(1, keepdims=True))[0]
    P /= P.sum()
    H = rng.standard_normal((K, N))
    H -= (P @ H) / (P @ P) * P[:, None]
    with_operands(a, H=H[:, None])
    r, u = a.ref, HALF_STEP[dtype]
    s, size = r.scores(0)
    P = np.exp(s - s.max(1, keepdims=True))
    P /= P.sum(1, keepdims=True)
    S = P @ np.abs(r.H[:, 0])
    grow = 2.0 ** -16 * (1 + size.max(1, keepdims=True))
    want, _, _, _ = r.forward()
    eo = u * np.abs(want[:, 0]) + (u * u + 2 * grow) * S + FLOOR[dtype]
    assert (np.abs(want[:, 0]) < 0.05 * S).mean() > 0.9
    # the bound tells one number from two
    once = torch.from_numpy(np.exp(s - s.max(1, keepdims=True))).to(a.dt).double().numpy()
    assert (np.abs(once / np.exp(s - s.max(1, keepdims=True)).sum(1, keepdims=True) @ r.H[:, 0] - want[:, 0]) > 1.5 * eo).any()
    out, lse = a.forward()
    near(a.f64(out)[:, 0], want[:, 0], eo, "out")
    got = a.backward(out, lse)[3]
    w, b = gradients(a, want)
    go = np.abs(a.f64(a.G)[:, 0])
    off = (go * eo).sum(1, keepdims=True) * P
    near(got, w["dTable"], b["dTable"] + np.array([[off[r.bucket == k].sum() for k in range(5)]]) * (1 + u), "dTable")
