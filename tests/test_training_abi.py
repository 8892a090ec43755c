"""The layer-and-step entry points on the host: every declared symbol is exported,
bad arguments are refused before anything is launched, and good ones are not."""
import ctypes
import os
import re
import struct
import subprocess

import pytest

import paper_2305_17190_amd as pam
from paper_2305_17190_amd import training

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "pam_training.h")
INVALID, LAUNCH = 1, 2
MB = 1 << 20


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pam.library_path()):
        pytest.skip("libpam.so not built (run __graft_entry__.build())")
    import torch
    if torch.cuda.is_available():
        pytest.skip("stand-in addresses: only where nothing can be launched")
    return training._library()


def test_header_is_c():
    """Without C++."""
    import shutil
    rocm = os.path.join(os.path.dirname(os.path.dirname(shutil.which("hipcc") or "/opt/rocm/bin/hipcc")), "include")
    subprocess.run(["gcc", "-std=c99", "-fsyntax-only", "-Wall", "-Werror", "-D__HIP_PLATFORM_AMD__", "-isystem", rocm,
                    "-I", os.path.dirname(HEADER), "-x", "c", HEADER], check=True)


def test_every_declared_symbol_is_exported():
    with open(HEADER) as f:
        declared = set(re.findall(r"^pam_status_t (pam_\w+)\(", f.read(), re.M))
    assert declared == set(training.EXPORTS)
    if os.path.exists(pam.library_path()):
        symbols = subprocess.run(["nm", "-D", "--defined-only", pam.library_path()], capture_output=True, text=True).stdout
        assert declared <= set(symbols.split())


# Addresses 256 MB apart; the host reads none of them.
def at(i):
    return (i + 1) * 256 * MB


def linear(lib, **change):
    f = dict(x=at(0), w=at(1), bias=at(2), residual=at(3), y=at(4), z=at(5), workspace=at(6), m=300, n=200, k=100, ldx=100,
             ldw=100, ldr=200, ldy=200, ldz=200, workspace_bytes=64 * MB, type=0, out_type=0, activation=2, mantissa_bits=23)
    assert set(change) <= set(f)
    f.update(change)
    return lib.pam_linear(struct.pack("=7q9q4i", *f.values()), None)


@pytest.mark.parametrize("change", [
    dict(x=0), dict(w=0), dict(y=0), dict(m=-1), dict(n=-1), dict(k=-1), dict(m=1 << 31), dict(n=1 << 31), dict(k=1 << 31),
    dict(ldx=99), dict(ldw=99), dict(ldr=199), dict(ldy=199), dict(ldz=199), dict(ldy=(1 << 31) + 1), dict(type=2),
    dict(type=-1), dict(out_type=2), dict(activation=5), dict(activation=-1), dict(mantissa_bits=24),
    dict(mantissa_bits=-1), dict(type=1, mantissa_bits=7), dict(y=at(0)), dict(y=at(1) + 4), dict(z=at(4)), dict(z=at(3)),
    dict(z=at(4) + 4 * 300 * 200 - 4), dict(y=at(2)), dict(residual=at(4), ldr=201), dict(residual=at(4) + 4),
    dict(k=8192, ldx=8192, ldw=8192, workspace=at(4)), dict(k=8192, ldx=8192, ldw=8192, workspace=at(0)),
    dict(m=(1 << 31) - 1024, ldr=1 << 31, ldy=1 << 31, ldz=1 << 31), dict(m=(1 << 31) - 1023), dict(n=(1 << 31) - 1023), dict(k=8192, ldx=8192, ldw=8192, workspace=0),
    dict(k=8192, ldx=8192, ldw=8192, workspace_bytes=4), dict(k=8192, ldx=8192, ldw=8192, workspace=at(6) + 4)])
def test_linear_refuses(lib, change):
    assert linear(lib, **change) == INVALID, lib.pam_last_error()


@pytest.mark.parametrize("change", [
    {}, dict(bias=0), dict(residual=0, ldr=0), dict(z=0, ldz=0), dict(residual=at(4)), dict(workspace=0, workspace_bytes=0),
    dict(type=1, out_type=1), dict(mantissa_bits=0), dict(k=0, x=0, w=0, ldx=1, ldw=1), dict(ldy=1000, ldx=1 << 17),
    dict(z=at(4) + 4 * 300 * 200), dict(workspace=at(6), workspace_bytes=1 << 40)])
def test_linear_accepts(lib, change):
    """As far as the device, which is missing here."""
    assert linear(lib, **change) == LAUNCH
    assert linear(lib, **{**change, "m": 0}) == 0 and linear(lib, **{**change, "n": 0}) == 0


def test_linear_workspace(lib):
    """The plan's partial sums, and the tiles' running sums where K is taken in parts."""
    need, plan = ctypes.c_size_t(), ctypes.c_size_t()
    for m, k, n in ((1, 512, 2048), (8, 8192, 4096), (197, 64, 197), (2048, 512, 2048), (0, 4096, 4096), (4096, 0, 4096)):
        assert lib.pam_linear_workspace_size(m, n, k, ctypes.byref(need)) == 0
        assert lib.pam_gemm_workspace_size(m, n, k, 1, ctypes.byref(plan)) == 0
        assert plan.value <= need.value <= plan.value + 255
    assert lib.pam_linear_workspace_size(16384, 4096, 4096, ctypes.byref(need)) == 0
    assert need.value >= 16384 * 4096 * 4
    args = dict(m=16384, k=4096, n=4096, x=at(0), w=at(8), bias=0, residual=0, y=at(16), z=0, workspace=at(32), ldx=4096,
                ldw=4096, ldy=4096)
    assert linear(lib, workspace_bytes=need.value - 1, **args) == INVALID
    assert linear(lib, workspace_bytes=need.value, **args) == LAUNCH
    for bad in ((-1, 1, 1), (1, -1, 1), (1, 1, -1), (1 << 31, 1, 1), (1 << 30, 1 << 30, 1)):
        assert lib.pam_linear_workspace_size(*bad, ctypes.byref(need)) == INVALID
    assert lib.pam_linear_workspace_size(1, 1, 1, None) == INVALID


def grad(lib, **change):
    f = dict(dy=at(0), z=at(1), dz=at(2), db=at(3), workspace=at(4), m=3000, n=200, lddy=200, ldz=200, lddz=200,
             workspace_bytes=64 * MB, type=0, z_type=0, activation=4, reserved=0)
    assert set(change) <= set(f)
    f.update(change)
    return lib.pam_activation_grad(struct.pack("=5q6q4i", *f.values()), None)


@pytest.mark.parametrize("change", [
    dict(dy=0), dict(z=0), dict(m=-1), dict(n=-1), dict(m=1 << 31), dict(n=(1 << 31) - 1023), dict(lddy=199), dict(ldz=199),
    dict(lddz=199), dict(type=2), dict(z_type=-1), dict(activation=5), dict(activation=0),
    dict(activation=0, z=0), dict(workspace=0), dict(workspace_bytes=4), dict(workspace=at(4) + 8), dict(dz=at(0) + 4),
    dict(dz=at(0), lddz=300), dict(dz=at(1), z_type=1), dict(db=at(0)), dict(db=at(2)), dict(db=at(4)),
    dict(workspace=at(1)), dict(workspace=at(2))])
def test_activation_grad_refuses(lib, change):
    assert grad(lib, **change) == INVALID


@pytest.mark.parametrize("change", [
    {}, dict(dz=at(0)), dict(dz=at(1)), dict(dz=0), dict(db=0, workspace=0, workspace_bytes=0), dict(type=1, z_type=0),
    dict(activation=0, z=0, dz=0), dict(m=0)])
def test_activation_grad_accepts(lib, change):
    assert grad(lib, **change) == LAUNCH
    assert grad(lib, **{**change, "n": 0, "db": 0}) == 0


def test_activation_grad_workspace(lib):
    need = ctypes.c_size_t()
    for m, n in ((1, 1), (5, 10000), (0, 7), (7, 0)):
        assert lib.pam_activation_grad_workspace_size(m, n, ctypes.byref(need)) == 0 and need.value == 0
    for m, n in ((16384, 4096), (1 << 30, 1), (1 << 30, 3), (100000, 771)):
        assert lib.pam_activation_grad_workspace_size(m, n, ctypes.byref(need)) == 0
        assert 0 < need.value <= 16 * MB and need.value % (4 * n) == 0
    assert lib.pam_activation_grad_workspace_size(-1, 1, ctypes.byref(need)) == INVALID
    assert lib.pam_activation_grad_workspace_size(1, 1, None) == INVALID


def tensor(base=0, n=1000, eight=False, copies=True, **change):
    f = dict(p=at(base), g=at(base + 1), avg=at(base + 2), sq=at(base + 3), avg_scale=at(base + 4) if eight else 0,
             sq_scale=at(base + 5) if eight else 0, copy=at(base + 6) if copies else 0, n=n)
    f.update(change)
    return f


def step(lib, tensors, **change):
    f = dict(norm=at(200), step_device=0, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, max_norm=1.0, step=1,
             seed=0, state_bits=32, grad_type=0, reserved=0)
    assert set(change) <= set(f)
    f.update(change)
    array = b"".join(struct.pack("=8q", *t.values()) for t in tensors)
    return lib.pam_adamw_step(array, len(tensors), struct.pack("=qqddddddqIiii", *f.values()), None)


def test_step_refuses(lib):
    good = [tensor(0), tensor(10)]
    for change in (dict(step=0), dict(step=-1), dict(lr=-1.0), dict(lr=float("nan")), dict(beta1=1.0), dict(beta1=-0.1),
                   dict(beta2=1.0), dict(beta2=float("nan")), dict(eps=-1.0), dict(weight_decay=-1.0), dict(max_norm=0.0),
                   dict(max_norm=float("nan")), dict(state_bits=16), dict(state_bits=8), dict(grad_type=2),
                   dict(norm=at(0)), dict(norm=at(10) + 3996), dict(step_device=at(2))):
        assert step(lib, good, **change) == INVALID, change
    for bad in (tensor(n=-1), tensor(p=0), tensor(g=0), tensor(avg=0), tensor(sq=0), tensor(avg_scale=at(4)),
                tensor(g=at(0)), tensor(sq=at(2)), tensor(copy=at(0)), tensor(copy=at(1) + 3998), tensor(n=1 << 39)):
        assert step(lib, [tensor(10), bad]) == INVALID, bad
    # The same tensor twice, in any list; one that reaches into the next.
    assert step(lib, [tensor(0), tensor(0)]) == INVALID
    for name, other in (("p", 0), ("avg", 2), ("sq", 3), ("copy", 6), ("p", 12), ("g", 0), ("g", 10)):
        assert step(lib, [tensor(0), tensor(10, **{name: at(other)})]) == INVALID, name
    assert step(lib, [tensor(0), tensor(10, p=at(0) + 3996)]) == INVALID
    assert step(lib, [tensor(0, eight=True), tensor(10, eight=True, sq_scale=at(4) + 12)], state_bits=8) == INVALID
    assert lib.pam_adamw_step(None, 1, struct.pack("=qqddddddqIiii", 0, 0, *([0.5] * 6), 1, 0, 32, 0, 0), None) == INVALID
    assert lib.pam_adamw_step(b"", 0, None, None) == INVALID
    assert lib.pam_adamw_step(b"", -1, struct.pack("=qqddddddqIiii", 0, 0, *([0.5] * 6), 1, 0, 32, 0, 0), None) == INVALID


def test_step_accepts(lib):
    for tensors, change in (([tensor(0)], {}), ([tensor(0), tensor(10)], {}), ([tensor(0, eight=True)], dict(state_bits=8)),
                            ([tensor(0, copies=False)], dict(norm=0, max_norm=0.0)), ([tensor(0)], dict(step=0, step_device=at(300))),
                            ([tensor(0), tensor(10, p=at(0) + 4000)], {}), ([tensor(0), tensor(10, g=at(1))], {}),
                            ([tensor(0, n=0, p=0, g=0), tensor(10)], {}), ([tensor(10 * i) for i in range(10)], {}),
                            ([tensor(0)], dict(beta1=0.0, beta2=0.0, eps=0.0, lr=0.0, weight_decay=0.0))):
        assert step(lib, tensors, **change) == LAUNCH, (tensors, change, lib.pam_last_error())
    assert step(lib, []) == 0 and step(lib, [tensor(0, n=0)]) == 0


def norm(lib, tensors, workspace=at(100), nbytes=MB, out=at(101), kind=0):
    return lib.pam_grad_norm(b"".join(struct.pack("=8q", *t.values()) for t in tensors), len(tensors), kind, out, workspace,
                             nbytes, None)


def test_grad_norm(lib):
    some = [tensor(0, n=100000), tensor(10, n=0, g=0), tensor(20, n=5, p=0)]
    assert norm(lib, some) == LAUNCH and norm(lib, []) == LAUNCH
    for change in (dict(workspace=0), dict(nbytes=8), dict(workspace=at(100) + 4), dict(out=0), dict(out=at(100)),
                   dict(out=at(1)), dict(workspace=at(21)), dict(kind=2)):
        assert norm(lib, some, **change) == INVALID, change
    assert norm(lib, [tensor(0, g=0)]) == INVALID and norm(lib, [tensor(0, n=-1)]) == INVALID
    need = ctypes.c_size_t()
    for n in (1, 4096, 1 << 20, 1 << 36):
        array = struct.pack("=8q", *tensor(0, n=n).values())
        assert lib.pam_grad_norm_workspace_size(array, 1, ctypes.byref(need)) == 0
        assert 8 <= need.value <= 8 * 2048


# The binding ---------------------------------------------------------------

def test_binding_refuses_what_is_not_on_the_gpu(lib):
    import torch
    x, w = torch.zeros(3, 4), torch.zeros(5, 4)
    with pytest.raises(pam.PamError, match="no CPU path"):
        pam.linear(x, w)
    with pytest.raises(pam.PamError, match="no CPU path"):
        pam.activation_grad(x, x, "relu")
    with pytest.raises(pam.PamError, match="no CPU path"):
        pam.grad_norm([x])
    with pytest.raises(pam.PamError, match="no CPU path"):
        pam.adamw_step([x], [x], [x], [x], 1)
    with pytest.raises(TypeError):
        pam.linear(None, w)
    with pytest.raises(TypeError):
        pam.grad_norm(x)
    with pytest.raises(TypeError):
        pam.grad_norm([None])
    with pytest.raises(ValueError, match="at least one"):
        pam.grad_norm([])
    with pytest.raises(TypeError, match="grads"):
        pam.grad_norm(None)
    for missing in range(4):
        lists = [[x]] * 4
        lists[missing] = None
        with pytest.raises(TypeError, match="list or tuple"):
            pam.adamw_step(*lists, 1)


def test_checks_of_the_binding(monkeypatch):
    """What the checks say of tensors that would otherwise do (on the meta device,
    taken for the GPU)."""
    import torch
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True))

    def new(*shape, dtype=torch.float32):
        return torch.empty(shape, device="meta", dtype=dtype)

    x, w = new(3, 4), new(5, 4)
    plan = training._linear_plan
    for args, error, match in (
            ((x, new(5, 4, dtype=torch.bfloat16), None, None, None, None, 23), TypeError, "both be float32"),
            ((x, new(5, 6), None, None, None, None, 23), ValueError, "inner dimensions"),
            ((x, w, new(4), None, None, None, 23), ValueError, "5 values"),
            ((x, w, new(5, dtype=torch.bfloat16), None, None, None, 23), TypeError, "bias must be float32"),
            ((x, w, None, new(3, 4), None, None, 23), ValueError, "3x5"),
            ((x, w, None, new(3, 5), None, torch.bfloat16, 23), TypeError, "output's type"),
            ((x, w, None, None, "tanh", None, 23), ValueError, "activation"),
            ((x, w, None, None, None, torch.float16, 23), TypeError, "out_dtype"),
            ((x.bfloat16(), w.bfloat16(), None, None, None, None, 5), ValueError, "7 mantissa bits"),
            ((new(4, 3).t(), w, None, None, None, None, 23), ValueError, "contiguous last dimension"),
            ((new(1, 4).expand(3, 4), w, None, None, None, None, 23), ValueError, "overlapping rows")):
        with pytest.raises(error, match=match):
            plan(*args)
    check = training._activation_grad_plan
    for args, error, match in (((x, None, "relu", True, True), ValueError, "with an activation"),
                               ((x, x, None, True, True), ValueError, "with an activation"),
                               ((x, new(3, 5), "relu", True, True), ValueError, "differ in shape"),
                               ((new(3, 4, dtype=torch.float16), x, "relu", True, True), TypeError, "float32 or bfloat16")):
        with pytest.raises(error, match=match):
            check(*args)
    lists = training._check_lists
    one, u8, scale = [new(300)], [new(300, dtype=torch.uint8)], [new(2)]
    lists(one, one, one, one, None, None, None)
    lists(one, one, u8, u8, scale, scale, [new(300, dtype=torch.bfloat16)])
    for args, error, match in (((one, one, u8, u8, None, None, None), ValueError, "uint8 states"),
                               ((one, one, one, one, scale, scale, None), ValueError, "uint8 states"),
                               ((one, one, u8, u8, [new(1)], scale, None), ValueError, "2 values"),
                               ((one, [new(299)], one, one, None, None, None), ValueError, "299 values"),
                               ((one, one * 2, one, one, None, None, None), ValueError, "1 tensors, grads 2"),
                               (([new(300).bfloat16()], one, one, one, None, None, None), TypeError, "params"),
                               ((one, [new(20, 15).t()], one, one, None, None, None), ValueError, "contiguous"),
                               ((one * 2, [new(300), new(300).bfloat16()], one * 2, one * 2, None, None, None), TypeError,
                                "grads")):
        with pytest.raises(error, match=match):
            lists(*args)


def test_optimizer_refusals():
    import torch
    from paper_2305_17190_amd.optim import AdamW
    p = [torch.nn.Parameter(torch.zeros(3))]
    with pytest.raises(ValueError, match="state_bits"):
        AdamW(p, state_bits=16)
    with pytest.raises(ValueError, match="max_norm"):
        AdamW(p, max_norm=0.0)
    for bad in (dict(lr=-1.0), dict(eps=-1.0), dict(weight_decay=-0.1), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1))):
        with pytest.raises(ValueError, match=next(iter(bad))):
            AdamW(p, **bad)
    import copy
    import pickle
    made = AdamW(p, lr=0.5, max_norm=2.0, state_bits=8, seed=3)
    for other in (copy.deepcopy(made), pickle.loads(pickle.dumps(made))):
        assert (other.max_norm, other.state_bits, other.seed) == (2.0, 8, 3) and other.param_groups[0]["lr"] == 0.5
    state = torch.optim.AdamW(p).state_dict()
    made.load_state_dict(state)
    state["state"] = {0: dict(step=1, exp_avg=torch.zeros(3))}
    for bits in (8, 32):
        with pytest.raises(ValueError, match="8 bits" if bits == 8 else "32 bits"):
            AdamW(p, state_bits=bits).load_state_dict(state)
