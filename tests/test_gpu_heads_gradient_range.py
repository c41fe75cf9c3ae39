"""Gradients of attention with heads far below, far above and all over the range of fp16's numbers."""
import numpy as np
import pytest

from heads_bounds import check_gradients, gradients, with_operands
from heads_ref import FLOOR
from test_gpu_heads import Problem, fs, near  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("V,V_t", [(4, 16), (8, 8), (16, 4)])
@pytest.mark.parametrize("M,K", [(24, 6000), (6000, 24)])
def test_gradients_far_below_the_normal_numbers_of_an_entry(fs, dtype, V, V_t, M, K):  # noqa: F811
    """Rows of 6000 entries and a gradient of 1e-4: an entry of dS is 1e-8, less than half of fp16's smallest number, and their sums are not."""
    a = Problem(fs, 31, M, K, 2, 1, 16, 16, dtype, kind="dense", bias=(9, 40), V=V, V_t=V_t)
    rng = np.random.default_rng(1)
    Y = np.abs(rng.standard_normal((K, 1, 16)))
    with_operands(a, X=0.1 * rng.standard_normal((M, 2, 16)), Y=Y, H=Y, G=1e-4 * rng.standard_normal((M, 2, 16)))
    _, _, got, want = check_gradients(a)
    assert (np.abs(want["dX"]) > 64 * FLOOR[dtype]).mean() > 0.5 and (got[0] != 0).float().mean() > 0.9


@pytest.mark.parametrize("V", [4, 8, 16])
@pytest.mark.parametrize("share", [1, 2])
def test_gradients_of_an_entry_beyond_fp16(fs, V, share):  # noqa: F811
    """dS of some 1e5, whose products with small rows are numbers of fp16 again."""
    a = Problem(fs, 32, 60, 50, 2, 2 // share, 16, 16, "f16", kind="hub", p=0.2, bias=(5, 6), V=V, V_t=V)
    rng = np.random.default_rng(2)
    with_operands(a, Y=2.0 ** -9 * rng.standard_normal((50, 2 // share, 16)), X=2.0 ** -9 * rng.standard_normal((60, 2, 16)),
                  H=30 * rng.standard_normal((50, 2 // share, 16)), G=2000 * rng.standard_normal((60, 2, 16)))
    a.bias.table.copy_(a.bias.table * 0.1)
    a.ref.table = a.f64(a.bias.table)
    out, lse = a.forward()
    got = a.backward(out, lse)
    want, bound = gradients(a, a.f64(out))
    for k, t in list(zip(("dX", "dY"), got)):
        assert np.abs(want[k]).max() < 60000
        near(t, want[k], bound[k], k)


@pytest.mark.parametrize("V", [4, 8, 16])
def test_gradients_that_grow_along_a_row(fs, V):  # noqa: F811
    """The first entries of a row have gradients of 1e-7, later ones more and more, up to 1e2; some rows have nothing but zeros."""
    M, K = 20, 700
    a = Problem(fs, 33, M, K, 1, 1, 16, 16, "f16", kind="dense", V=V, V_t=V, chunk=64)
    rng = np.random.default_rng(3)
    H = rng.standard_normal((K, 1, 16)) * 10.0 ** np.linspace(-7, 2, K)[:, None, None]
    G = rng.standard_normal((M, 1, 16))
    G[3:6] = 0.0
    with_operands(a, H=H, G=G, X=0.2 * rng.standard_normal((M, 1, 16)))
    check_gradients(a)
