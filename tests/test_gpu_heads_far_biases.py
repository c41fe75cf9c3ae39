"""Attention with heads whose biases lie far from zero, the type's lowest and highest value among them: masks that are no infinities."""
import numpy as np
import pytest

from heads_bounds import check_gradients, with_operands
from heads_ref import FLOOR, HALF_STEP
from test_gpu_heads import Problem, fs, near  # noqa: F401

pytestmark = pytest.mark.gpu

MOST = 3.4028234663852886e38 / np.log2(np.e)  # of a bias that counts
SHAPES = [(4, 8, 0, 1), (8, 8, 64, 2), (16, 4, 64, 1)]


def far_problem(fs, dtype, bias, V, V_t, chunk, share):  # noqa: F811
    """Two heads.  The second has the bias everywhere; the first, where it is negative, for the columns three or more behind the row's.  The rows of X that
    have nothing else are zero, so that their scores are the bias exactly and 64 bits say the same of them however little of a score is left
    beside it: probabilities that are all equal.  In the other rows such entries have none."""
    import torch
    M, K = 90, 200
    a = Problem(fs, 36, M, K, 2, 2 // share, 32, 48, dtype, kind="hub", p=0.25, bias=(4, 3), V=V, V_t=V_t, chunk=chunk)
    a.bias.buckets.copy_(torch.tensor([0, 1, 2, 0, 1, 2, 3], dtype=torch.uint8))
    a.bias.table[1] = bias
    if bias < 0:
        a.bias.table[0, 3] = bias
    behind = np.arange(K)[None] - np.arange(M)[:, None] >= 3
    X = a.f64(a.X)
    X[:, 1] = 0.0
    if bias < 0:
        X[~(a.stored & ~behind).any(1), 0] = 0.0
    with_operands(a, X=X)
    a.ref.bucket = np.asarray([0, 1, 2, 0, 1, 2, 3])[np.clip(np.arange(K)[None] - np.arange(M)[:, None], -3, 3) + 3]
    a.ref.table = a.f64(a.bias.table)
    assert (a.stored & behind).any() and ((a.stored & ~behind).any(1) != a.stored.any(1)).any()
    real = a.ref.scores

    def scores(h):  # (a far bias is exact, and no rounding beside it counts)
        s, size = real(h)
        b = a.ref.table[h][a.ref.bucket]
        return s, size - np.where(np.abs(b) > 1000, np.abs(b), 0.0)
    a.ref.scores = scores
    return a


def check_forward(a):
    """out as in the reference; a far row's lse is its bias, of which at most MOST counts, up to a few roundings of it."""
    import torch
    out, lse = a.forward()
    u = HALF_STEP[a.dtype]
    for h in range(2):
        s, size = a.ref.scores(h)
        P = np.where(a.stored, np.exp(s - s.max(1, keepdims=True, initial=-1e300)), 0.0) * a.stored.any(1, keepdims=True)
        total = P.sum(1, keepdims=True)
        P = np.divide(P, total, out=np.zeros_like(P), where=total > 0)
        v = a.ref.H[:, h // a.ref.share]
        want, S = (P * a.ref.Z[h]) @ v, (P * a.ref.Z[h]) @ np.abs(v)
        grow = 2.0 ** -15 * (1 + np.where(a.stored, size, 0.0).max(1, keepdims=True))
        near(a.f64(out)[:, h], want, u * np.abs(want) + (2 * u + u * u + grow) * S + 2.0 ** -25 * np.abs(v).sum(0) + FLOOR[a.dtype], "out of head %d" % h)
    got, n = a.f64(lse)[1], a.stored.sum(1)
    assert torch.isfinite(out).all() and np.isneginf(got[n == 0]).all()
    counts = np.clip(a.ref.table[1, 0], -MOST, MOST)
    assert (np.abs(got[n > 0] - (counts + np.log(n[n > 0]))) <= 2.0 ** -21 * np.abs(counts)).all()


FAR = [("bf16", -1e30), ("bf16", -1e9), ("bf16", 1e9), ("bf16", -1e6), ("bf16", -30000.0), ("f16", -65504.0), ("f16", 65504.0), ("f16", -30000.0), ("f16", -2000.0)]


@pytest.mark.parametrize("dtype,bias", FAR)
@pytest.mark.parametrize("V,V_t,chunk,share", SHAPES)
def test_dropped_and_kept_entries_have_the_same_bias(fs, dtype, bias, V, V_t, chunk, share):  # noqa: F811
    """What dropout leaves of a row is weighted with the probabilities of all of it, also where the last bit of a bias is worth more than the scores."""
    check_forward(far_problem(fs, dtype, bias, V, V_t, chunk, share))


LOWEST = 3.3895313892515355e38


@pytest.mark.parametrize("bias", [-LOWEST, LOWEST, -2.5e38])
@pytest.mark.parametrize("V,V_t,chunk,share", SHAPES)
def test_the_lowest_finite_value_is_no_infinity(fs, bias, V, V_t, chunk, share):  # noqa: F811
    """A row of nothing but the type's lowest value has the mean of its rows of H."""
    check_forward(far_problem(fs, "bf16", bias, V, V_t, chunk, share))


@pytest.mark.parametrize("dtype,bias", FAR + [("bf16", -LOWEST), ("bf16", LOWEST)])
@pytest.mark.parametrize("V,V_t,chunk,share", SHAPES)
def test_gradients_of_rows_whose_biases_are_all_far_from_zero(fs, dtype, bias, V, V_t, chunk, share):  # noqa: F811
    """Such a row's lse holds nothing of what its probabilities add up to."""
    check_gradients(far_problem(fs, dtype, bias, V, V_t, chunk, share))


def test_probabilities_beside_a_far_bias_add_up_to_one(fs):  # noqa: F811
    """A head with a bias of -30000 everywhere: a score keeps eight binary places beside it, a row's probabilities are those of such scores.  With a
    gradient of out that is one in column i of row i alone, column i of dH holds row i's probabilities: each is rounded twice, and what
    they are made of is off by 2^-15 in fp32."""
    import torch
    a = Problem(fs, 37, 32, 120, 2, 2, 32, 32, "f16", kind="dense", bias=(3, 10), chunk=64)
    a.bias.table[1] = -30000.0
    a.G.zero_()
    a.G[torch.arange(32), :, torch.arange(32)] = 1.0
    out, lse = a.forward()
    total = a.f64(a.backward(out, lse)[2]).sum(0)
    assert np.abs(total - 1).max() <= 2 * 2.0 ** -11 + 2.0 ** -15 + 120 * 2.0 ** -25


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("V,V_t,chunk,share", SHAPES)
def test_rows_whose_scores_are_far_from_zero_without_a_bias(fs, dtype, V, V_t, chunk, share):  # noqa: F811
    """Scores of some thousands that differ by a few: whole numbers below 2^24 times a power of two, so that X Y^T is exact and a score, in units of
    log2, is off by 2^-24 of itself; so is a row's largest."""
    rng = np.random.default_rng(6)
    a = Problem(fs, 39, 90, 200, 2, 2 // share, 32, 48, dtype, kind="hub", p=0.25, V=V, V_t=V_t, chunk=chunk)
    a.scale = a.ref.scale = 2.0 ** -4
    X, Y = 32 * np.sign(rng.standard_normal((90, 2, 1))) * np.ones((90, 2, 32)), 64 + np.zeros((200, 2 // share, 32))
    Y[:, :, :2] += rng.integers(-1, 2, (200, 2 // share, 2)) * 0.5
    with_operands(a, X=X, Y=Y)
    s = a.ref.scores(0)[0]
    far = np.abs(s[a.stored])
    assert far.min() > 4000 and far.max() < 4200
    real = a.ref.scores
    a.ref.scores = lambda h: (real(h)[0], np.zeros_like(s))
    check_gradients(a, l_off=2.0 ** -22 * 4200)


@pytest.mark.parametrize("bias", [-LOWEST, LOWEST, -1e30, -1e9, 1e9])
@pytest.mark.parametrize("V,V_t,chunk,share", SHAPES)
def test_gradients_agree_with_an_out_that_has_lost_the_scores(fs, bias, V, V_t, chunk, share):  # noqa: F811
    """fp32 holds nothing of a score of some tens beside such a bias, forward or backward: probabilities that are all equal, in out and in its
    gradients, whose dS adds up to zero in every row as it has to."""
    a = far_problem(fs, "bf16", bias, V, V_t, chunk, share)
    with_operands(a, X=np.random.default_rng(8).standard_normal(a.ref.X.shape))
    real = a.ref.scores

    def scores(h):
        s, size = real(h)
        b = a.ref.table[h][a.ref.bucket]
        return np.where(a.stored & (np.abs(b) > 1000), b, s), size
    a.ref.scores = scores
    check_forward(a)
    check_gradients(a)
