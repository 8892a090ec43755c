"""Matrices of one column whose last stride is not 1, as transposing a row gives
them: torch calls them contiguous, and so they are."""
import pytest

import paper_2305_17190_amd as pam
from gpu_util import device, note
from test_gpu_linear import inputs, same

pytestmark = pytest.mark.gpu


def column(t):
    """t (m x 1) with strides (1, m)."""
    c = t.reshape(1, -1).clone().t()
    assert c.shape == t.shape and (c.stride(-1) != 1 or c.shape[0] == 1) and c.is_contiguous()
    return c


@pytest.mark.parametrize("m,k", [(2, 16), (37, 64), (500, 100)])
@pytest.mark.parametrize("activation", [None, "gelu"])
@pytest.mark.parametrize("with_residual", [False, True])
def test_value_head_transposed(m, k, activation, with_residual):
    """A head's values as a row: its gradient comes back as such a column."""
    import torch
    from paper_2305_17190_amd.autograd import pam_linear
    note(f"pam_linear {m}x{k} -> 1, transposed, {activation}, residual {with_residual}")
    x, w, bias, res = inputs(m, k, 1)
    dy = torch.linspace(-1, 1, m, device=device())
    grads = []
    for transposed in (False, True):
        leaves = [t.clone().requires_grad_() for t in (x, w, bias, res)]
        y = pam_linear(*leaves[:3], activation=activation, residual=leaves[3] if with_residual else None)
        if transposed:
            y.t().backward(dy.reshape(1, m))
        else:
            y.backward(dy.reshape(m, 1))
        grads.append([t.grad for t in leaves if t.grad is not None])
    assert len(grads[0]) == 3 + with_residual
    assert all(torch.equal(a, b) for a, b in zip(*grads))


@pytest.mark.parametrize("m,n", [(2, 3), (33, 70), (300, 500)])
def test_calls(m, n):
    """As x and w with k = 1, as residual, as dy and z."""
    note(f"single columns {m}, {n}")
    x, w, bias, res = inputs(m, 1, n)
    assert same(pam.gemm(column(x), column(w), trans_b=True), pam.gemm(x, w, trans_b=True))
    assert same(pam.linear(column(x), column(w), bias, "silu", res), pam.linear(x, w, bias, "silu", res))
    x, w, bias, res = inputs(m, n, 1)
    y, z = pam.linear(x, w, bias, "gelu", res, save_z=True)
    assert same(pam.linear(x, w, bias, "gelu", column(res)), y)
    want = pam.activation_grad(y, z, "gelu")
    assert all(same(a, b) for a, b in zip(pam.activation_grad(column(y), column(z), "gelu"), want))
    a = inputs(m, 1, n)[0].reshape(1, m, 1).expand(2, m, 1).contiguous()
    b = inputs(n, 1, n)[0].reshape(1, 1, n).expand(2, 1, n).contiguous()
    strange = a.transpose(1, 2).contiguous().transpose(1, 2)
    assert same(pam.bmm(strange, b), pam.bmm(a, b))
