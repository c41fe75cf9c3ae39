"""Attention with heads on operands of one row."""
import pytest

from test_gpu_heads import Problem, fs  # noqa: F401

pytestmark = pytest.mark.gpu


def test_one_row_of_a_matrix_of_any_width(fs):  # noqa: F811
    """A pitch that leads nowhere is not looked at: one token's row of a wider buffer whose rows are no multiple of sixteen bytes."""
    import torch
    a = Problem(fs, 38, 1, 50, 2, 1, 16, 24, "f16", kind="dense", p=0.1, bias=(6, 9))
    out, lse = a.forward()
    grads = a.backward(out, lse)
    wide = torch.zeros((4, 2 * 16 + 5), dtype=torch.float16, device="cuda")
    x = wide.as_strided((1, 2, 16), (37, 16, 1))
    x.copy_(a.X)
    g = torch.zeros((3, 2 * 24 + 3), dtype=torch.float16, device="cuda").as_strided((1, 2, 24), (51, 24, 1))
    g.copy_(a.G)
    assert x.stride(0) % 8 and g.stride(0) % 8
    a.X, a.G = x, g
    o, l = a.forward()
    assert torch.equal(o, out) and torch.equal(l, lse)
    assert all(torch.equal(p, q) for p, q in zip(a.backward(out, lse), grads))
    into = torch.zeros((2, 2 * 24 + 7), dtype=torch.float16, device="cuda").as_strided((1, 2, 24), (55, 24, 1))
    o, l = a.forward(out=into)
    assert torch.equal(o, out)
