"""Linear layers with one output or two: heads that answer with a value.  The few
rows are the weights' there, and the outputs' columns are few enough that rows and
columns can have the same stride."""
import ctypes
import struct

import numpy as np
import pytest

import paper_2305_17190_amd as pam
import training_util as tu
from attention_util import check
from gpu_util import device, note
from oracle import pam_ref
from oracle import training_ref as ref
from test_gpu_linear import expect, inputs, same

pytestmark = pytest.mark.gpu

NAN = float("nan")


def inside(t, before, after):
    """t as columns (or values) of a wider tensor of NaN."""
    import torch
    wide = torch.full((*t.shape[:-1], before + t.shape[-1] + after), NAN, device=t.device, dtype=t.dtype)
    view = wide[..., before:before + t.shape[-1]]
    view.copy_(t)
    return view


@pytest.mark.parametrize("m,k", [(2, 1), (2, 512), (33, 64), (33, 4096), (500, 100), (4096, 512), (4097, 33)])
@pytest.mark.parametrize("n", [1, 2])
@pytest.mark.parametrize("bf16", [False, True])
def test_few_outputs(m, k, n, bf16):
    """The bias within a longer tensor, the residual within a wider matrix: NaN around
    them reaches no output."""
    import torch
    for i, name in enumerate(ref.ACTIVATIONS):
        for out_bf16 in (False, True):
            x, w, bias, res = inputs(m, k, n, bf16, i, out_bf16)
            out = res.dtype
            note(f"linear {m}x{k}x{n} {name} {x.dtype} -> {out}, bias and residual inside others")
            y, z = pam.linear(x, w, inside(bias, 5, 4 * m), name, inside(res, 3, 2), save_z=True, out_dtype=out)
            z32 = pam.gemm(x, w, trans_b=True) + bias
            assert same(z, z32.to(out)) and y.shape == (m, n)
            expect(y, z32, name, res, out_bf16, "y")
            assert same(pam.linear(x, w, bias, name, res, out_dtype=out), y)


@pytest.mark.parametrize("m,k", [(2, 64), (33, 100), (4096, 512)])
def test_one_output_against_the_definition(m, k):
    note(f"linear {m}x{k}x1 against float64")
    x, w, bias, res = inputs(m, k, 1)
    y, z = pam.linear(x, w, bias, "silu", res, save_z=True)
    want, zr, size = ref.linear(*(t.cpu().numpy() for t in (x, w, bias)), "silu", res.cpu().numpy())
    # Every term is exact or rounded once, and k of them are added in some order; the bias rounds once more.
    dz = 2 * k * tu.U * size + k * 2.0 ** -126 + tu.U * np.abs(zr)
    check(z.cpu().numpy(), zr, dz, "z")
    # silu's slope stays below 1.1.
    check(y.cpu().numpy(), want, 1.1 * dz + tu.activation_error(zr, "silu") + tu.U * np.abs(want), "y")


@pytest.mark.parametrize("m,k", [(2, 64), (33, 100), (500, 4096), (4096, 512)])
@pytest.mark.parametrize("n", [1, 2])
@pytest.mark.parametrize("ldy,ldz,ldr", [(0, 0, 4), (0, 6, 0), (5, 0, 3), (4, 2, 0), (5, 3, None)])
def test_c_call_strides(m, k, n, ldy, ldz, ldr):
    """Leading dimensions n + ldy, n + ldz and n + ldr: what lies between the rows
    stays.  None: y on its residual."""
    import torch
    note(f"pam_linear {m}x{k}x{n}, strides {ldy} {ldz} {ldr} past n")
    x, w, bias, res = inputs(m, k, n)
    want, zw = pam.linear(x, w, bias, "gelu_tanh", res, save_z=True)
    y = torch.full((m, n + ldy), 7.0, device=device())
    z = torch.full((m, n + ldz), 9.0, device=device())
    if ldr is None:
        y[:, :n] = res
        r, ldr = y, ldy
    else:
        r = torch.full((m, n + ldr), NAN, device=device())
        r[:, :n] = res
    long_bias = inside(bias, 1, 4 * m)
    lib = pam.training._library()
    need = ctypes.c_size_t()
    assert lib.pam_linear_workspace_size(m, n, k, ctypes.byref(need)) == 0
    ws = torch.empty(max(need.value, 1), dtype=torch.uint8, device=device())
    args = struct.pack("=7q9q4i", x.data_ptr(), w.data_ptr(), long_bias.data_ptr(), r.data_ptr(), y.data_ptr(), z.data_ptr(),
                       ws.data_ptr(), m, n, k, k, k, n + ldr, n + ldy, n + ldz, need.value, 0, 0, 3, 23)
    assert lib.pam_linear(args, torch.cuda.current_stream().cuda_stream) == 0
    assert same(y[:, :n].contiguous(), want) and same(z[:, :n].contiguous(), zw)
    assert bool((y[:, n:] == 7).all()) and bool((z[:, n:] == 9).all())


@pytest.mark.parametrize("m,k", [(2, 64), (33, 100), (500, 96)])
def test_value_head(m, k):
    """PAMLinear with one output, forward and backward, against the definition and,
    for what is ordinary arithmetic, differences."""
    import torch
    from paper_2305_17190_amd.autograd import PAMLinear
    note(f"PAMLinear {m}x{k} -> 1")
    x, w, bias, res = inputs(m, k, 1)
    layer = PAMLinear(k, 1, device=device(), activation="gelu")
    with torch.no_grad():
        layer.weight.copy_(w)
        layer.bias.copy_(bias)
    x.requires_grad_(), res.requires_grad_()
    y = layer(x, residual=res)
    dy = torch.linspace(-1, 1, m, device=device()).reshape(m, 1)
    y.backward(dy)
    d = dy.cpu().numpy()
    z = pam.gemm(x.detach(), w, trans_b=True) + bias
    zn = z.cpu().numpy().astype(np.float64)
    dz, db = ref.activation_grad(d, zn, "gelu")
    ez = np.abs(d) * tu.slope_error(zn, "gelu") + tu.U * np.abs(dz)
    check(layer.bias.grad.cpu().numpy(), db, ez.sum(0) + m * tu.U * np.abs(dz).sum(0), "db")
    # Differences of the definition's sum of d f(z + b) by b, in float64.
    h = 1e-5
    by = [(d * ref.activation(zn + s * h, "gelu")).sum(0) for s in (1, -1)]
    check(db, (by[0] - by[1]) / (2 * h), 1e-8 * (1 + np.abs(d).sum()), "difference")
    assert torch.equal(res.grad, dy)
    # The products' gradients are products with the kernel's own dz.
    got, _ = pam.activation_grad(dy, z, "gelu")
    check(got.cpu().numpy(), dz, ez, "dz")
    assert same(x.grad, pam.gemm(got, w)) and same(layer.weight.grad, pam.gemm(got, x.detach(), trans_a=True))
    want, size = pam_ref.pam_gemm_ref(got.cpu().numpy(), w.cpu().numpy(), False, False)
    check(x.grad.cpu().numpy(), want, 2 * tu.U * size + 2.0 ** -126, "dx")
