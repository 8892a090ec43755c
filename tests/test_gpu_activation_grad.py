"""The gradient of a linear layer's additions against the definition in float64,
and the layer under autograd."""
import numpy as np
import pytest

import paper_2305_17190_amd as pam
import training_util as tu
from attention_util import check
from gpu_util import device, note, to_dev
from oracle import pam_ref
from oracle import training_ref as ref

pytestmark = pytest.mark.gpu

SIZES = [(1, 1), (1, 771), (197, 771), (260, 9), (5, 3), (1000, 1), (4097, 2), (300, 37), (64, 256), (2048, 512), (3000, 770),
         (16384, 5), (7, 9000)]


def problem(m, n, bf16=False, z_bf16=False, seed=0):
    import torch
    rng = np.random.default_rng([m, n, seed])
    dy = to_dev(rng.standard_normal((m, n)).astype(np.float32))
    z = to_dev((2 * rng.standard_normal((m, n))).astype(np.float32))
    return dy.to(torch.bfloat16 if bf16 else torch.float32), z.to(torch.bfloat16 if z_bf16 else torch.float32)


def host(t):
    return t.float().cpu().numpy().astype(np.float64)


def expect(dz, db, dy, z, name, bf16):
    dy, m = host(dy), dy.shape[0]
    want, sums = ref.activation_grad(dy, host(z), name)
    err = np.abs(dy) * tu.slope_error(host(z), name) + tu.U * np.abs(want) + tu.TINY
    if dz is not None:
        check(host(dz), want, err + (2.0 ** -8 * np.abs(want) if bf16 else 0), "dz")
    check(host(db), sums, err.sum(0) + (m + 2) * tu.U * np.abs(want).sum(0), "db")


@pytest.mark.parametrize("m,n", SIZES)
@pytest.mark.parametrize("bf16,z_bf16", [(False, False), (True, True), (True, False), (False, True)])
def test_all_activations(m, n, bf16, z_bf16):
    note(f"activation_grad {m}x{n} dy bf16 {bf16} z bf16 {z_bf16}")
    for i, name in enumerate(ref.ACTIVATIONS[1:]):
        dy, z = problem(m, n, bf16, z_bf16, i)
        dz, db = pam.activation_grad(dy, z, name)
        assert dz.dtype == dy.dtype and dz.shape == dy.shape and db.shape == (n,)
        expect(dz, db, dy, z, name, bf16)
        again, sums = pam.activation_grad(dy, z, name)
        assert bool((again == dz).all()) and bool((sums == db).all())
        alone, none = pam.activation_grad(dy, z, name, bias=False)
        assert none is None and bool((alone == dz).all())
        none, alone = pam.activation_grad(dy, z, name, input_grad=False)
        assert none is None and bool((alone == db).all())


@pytest.mark.parametrize("m,n", SIZES)
def test_without_an_activation(m, n):
    note(f"column sums {m}x{n}")
    for bf16 in (False, True):
        dy, _ = problem(m, n, bf16)
        dz, db = pam.activation_grad(dy, None, None)
        assert dz is dy
        expect(None, db, dy, dy, None, bf16)


@pytest.mark.parametrize("m,n", [(300, 771), (40, 13), (9, 3), (2000, 130)])
@pytest.mark.parametrize("bf16", [False, True])
def test_c_call_in_place(m, n, bf16):
    """dz on dy, and on z, rows longer than n: the columns between stay."""
    import ctypes
    import struct
    import torch
    note(f"pam_activation_grad {m}x{n} in place, bf16 {bf16}")
    dy, z = problem(m, n, bf16, bf16)
    want, sums = pam.activation_grad(dy, z, "gelu")
    lib, need = pam.training._library(), ctypes.c_size_t()
    assert lib.pam_activation_grad_workspace_size(m, n, ctypes.byref(need)) == 0
    for onto in (0, 1):
        wide = torch.full((2, m, n + 5), 7.0, device=device(), dtype=dy.dtype)
        wide[0, :, :n], wide[1, :, :n] = dy, z
        db = torch.empty(n, device=device())
        ws = torch.empty(max(need.value, 1), dtype=torch.uint8, device=device())
        args = struct.pack("=5q6q4i", wide[0].data_ptr(), wide[1].data_ptr(), wide[onto].data_ptr(), db.data_ptr(),
                           ws.data_ptr(), m, n, n + 5, n + 5, n + 5, need.value, int(bf16), int(bf16), 2, 0)
        assert lib.pam_activation_grad(args, torch.cuda.current_stream().cuda_stream) == 0
        assert torch.equal(wide[onto, :, :n], want) and torch.equal(db, sums)
        assert torch.equal(wide[1 - onto, :, :n], (z, dy)[onto]) and bool((wide[:, :, n:] == 7).all())


@pytest.mark.parametrize("seed", range(24))
def test_random_sizes(seed):
    import random
    rng = random.Random(700 + seed)
    m, n = (int(round(20000 ** rng.random())) for _ in "mn")
    m = min(m, 4000000 // n)
    bf16, z_bf16, name = rng.random() < 0.5, rng.random() < 0.5, rng.choice(ref.ACTIVATIONS[1:])
    note(f"random activation_grad {seed}: {m}x{n} {name} bf16 {bf16} {z_bf16}")
    dy, z = problem(m, n, bf16, z_bf16, seed)
    dz, db = pam.activation_grad(dy, z, name)
    expect(dz, db, dy, z, name, bf16)


def test_views_and_no_rows():
    import torch
    note("activation_grad of views")
    dy, z = problem(300, 130)
    wide = torch.full((2, 300, 141), float("nan"), device=device())
    wide[0, :, 5:135], wide[1, :, 3:133] = dy, z
    got = pam.activation_grad(wide[0, :, 5:135], wide[1, :, 3:133], "silu")
    for a, b in zip(got, pam.activation_grad(dy, z, "silu")):
        assert bool((a == b).all())
    dz, db = pam.activation_grad(dy[:0], z[:0], "silu")
    assert dz.shape == (0, 130) and bool((db == 0).all())
    assert pam.activation_grad(dy[:, :0], z[:, :0], "silu")[1].shape == (0,)


@pytest.mark.parametrize("name", ref.ACTIVATIONS[1:])
def test_special_values(name):
    note(f"slopes at special values {name}")
    z = np.array([0.0, -0.0, np.inf, -np.inf, np.nan, 3e38, -3e38, 1e20, -1e20, 200, -200, 119, -119, 88.5, -88.5, 16.5,
                  -16.5, 15.5, -15.5, 5, -5, 1e-30, -1e-30], np.float32)[None]
    dy = np.full_like(z, 2)
    dz, _ = pam.activation_grad(to_dev(dy), to_dev(z), name)
    check(host(dz), ref.activation_grad(dy, z, name)[0],
          np.nan_to_num(2 * tu.slope_error(z, name) + tu.U * 4 + tu.TINY), "dz")
    if name == "relu":     # what reaches a closed unit counts for nothing
        dy = np.array([[np.inf, np.nan, np.inf]], np.float32)
        dz, _ = pam.activation_grad(to_dev(dy), to_dev(np.array([[-1.0, -1.0, 1.0]], np.float32)), name)
        assert host(dz).tolist() == [[0.0, 0.0, np.inf]]


# Under autograd ------------------------------------------------------------

def layer_inputs(seed=0, m=37, k=50, n=29):
    rng = np.random.default_rng(seed)
    x, w, b, r, dy = (rng.standard_normal(s).astype(np.float32) for s in ((m, k), (n, k), (n,), (m, n), (m, n)))
    return x, (w / 7).astype(np.float32), b, r, dy


@pytest.mark.parametrize("name", ref.ACTIVATIONS)
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("derivative", ["approximate", "exact"])
def test_pam_linear_gradients(name, residual, derivative):
    """dX and dW are products with dz, db its sums, the residual's gradient dy."""
    import torch
    from paper_2305_17190_amd.autograd import pam_linear
    note(f"pam_linear {name} residual {residual} {derivative}")
    x, w, b, r, dy = layer_inputs()
    leaves = [to_dev(t).requires_grad_() for t in (x, w, b, r)]
    y = pam_linear(leaves[0].view(1, 37, 50), leaves[1], leaves[2], derivative=derivative, activation=name,
                   residual=leaves[3].view(1, 37, 29) if residual else None)
    z = pam.gemm(leaves[0].detach(), leaves[1].detach(), trans_b=True) + leaves[2].detach()
    assert torch.equal(y[0], pam.linear(*(t.detach() for t in leaves[:3]), name, leaves[3].detach() if residual else None))
    y.backward(to_dev(dy)[None])
    dz, db = (to_dev(dy), None) if name is None else pam.activation_grad(to_dev(dy), z, name)
    if derivative == "exact":
        dx, dw = pam.exact_grad(dz, leaves[1].detach(), leaves[0].detach()), pam.exact_grad(
            dz, leaves[0].detach(), leaves[1].detach(), trans_a=True)
    else:
        dx, dw = pam.gemm(dz, leaves[1].detach()), pam.gemm(dz, leaves[0].detach(), trans_a=True)
    assert torch.equal(leaves[0].grad, dx) and torch.equal(leaves[1].grad, dw)
    want, sums = ref.activation_grad(dy, host(z), name)
    check(host(leaves[2].grad), sums, (np.abs(dy) * tu.slope_error(host(z), name)).sum(0) +
          40 * tu.U * np.abs(want).sum(0) + tu.TINY, "db")
    if residual:
        assert torch.equal(leaves[3].grad, to_dev(dy))


def test_gradient_against_differences():
    """Operands that are powers of two, whose PAM products are true ones: the loss's
    differences along the bias and the residual."""
    import torch
    from paper_2305_17190_amd.autograd import pam_linear
    note("pam_linear against differences")
    rng = np.random.default_rng(4)
    x, w = ((2.0 ** rng.integers(-2, 1, s) * rng.choice([-1, 1], s)).astype(np.float32) for s in ((20, 16), (12, 16)))
    b, dy = (rng.standard_normal(s).astype(np.float32) for s in ((12,), (20, 12)))
    z = pam_ref.pam_gemm_ref(x, w, False, True)[0]
    for name in ref.ACTIVATIONS[1:]:
        leaf = to_dev(b).requires_grad_()
        pam_linear(to_dev(x), to_dev(w), leaf, activation=name).backward(to_dev(dy))
        h = 1e-5
        for j in range(12):
            up, down = (ref.activation(z[:, j] + b[j].astype(np.float64) + e, name) for e in (h, -h))
            assert abs(float(leaf.grad[j]) - (dy[:, j] * (up - down)).sum() / (2 * h)) < 2e-4


def test_what_needs_no_gradient_keeps_nothing():
    import torch
    from paper_2305_17190_amd.autograd import PAMLinear, pam_linear
    note("pam_linear without gradients")
    x, w, b, r, dy = (to_dev(t) for t in layer_inputs())
    with torch.no_grad():
        plain = pam_linear(x, w, b, activation="gelu", residual=r)
    assert not plain.requires_grad and torch.equal(plain, pam.linear(x, w, b, "gelu", r))
    only = r.clone().requires_grad_()
    pam_linear(x, w, b, activation="gelu", residual=only).backward(dy)
    assert torch.equal(only.grad, dy)
    layer = PAMLinear(50, 29, device=device(), activation="silu")
    y = layer(x, residual=r)
    assert torch.equal(y, pam.linear(x, layer.weight.detach(), layer.bias.detach(), "silu", r))
    y.backward(dy.t().contiguous().t())              # a gradient whose rows are not dense
    z = pam.gemm(x, layer.weight.detach(), trans_b=True) + layer.bias.detach()
    dz, db = pam.activation_grad(dy, z, "silu")
    assert torch.equal(layer.bias.grad, db) and torch.equal(layer.weight.grad, pam.gemm(dz, x, trans_a=True))


def test_broadcast_gradients():
    """The gradient of a sum reaches the layer with strides of zero."""
    import torch
    from paper_2305_17190_amd.autograd import pam_linear
    note("pam_linear, expanded gradient")
    x, w, b, r, _ = (to_dev(t) for t in layer_inputs())
    leaf = b.clone().requires_grad_()
    pam_linear(x, w, leaf, activation="relu", residual=r).sum().backward()
    z = pam.gemm(x, w, trans_b=True) + b
    assert torch.equal(leaf.grad, (z > 0).float().sum(0))


def test_second_derivatives_raise():
    import torch
    from paper_2305_17190_amd.autograd import pam_linear
    note("pam_linear, second derivatives")
    x, w, b, r, _ = (to_dev(t) for t in layer_inputs())
    x.requires_grad_()
    dx, = torch.autograd.grad(pam_linear(x, w, b, activation="gelu").pow(2).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="first derivatives"):
        dx.sum().backward()
