"""The layer-and-step side of a PAM transformer: linear layers with bias,
activation and residual around their PAM product, the gradient of what they add
to it, and the optimizer's step over all parameters at once.

Thin binding over ``include/pam_training.h`` in the manner of the package's
other calls: every step runs in the library's HIP kernels on the current
stream, nothing waits for the GPU, and there is no CPU path.

    linear(x, w, bias, activation, residual, ...)    act(x .^ w^T + bias) + residual
    activation_grad(dy, z, activation, ...)          the gradient up to the product, and the bias's
    grad_norm(grads)                                 the norm of all gradients
    adamw_step(params, grads, avgs, sqs, step, ...)  one AdamW step, states in 32 or 8 bits

The products are PAM products (Sec. 3.2 replaces those of the linear layers);
bias, activation, residual and the optimizer are ordinary float32 arithmetic.
``autograd.pam_linear`` and ``optim.AdamW`` are what a model is trained with.
"""
from __future__ import annotations

import ctypes
import functools
import struct

from . import PamError, _check, _launch, _require, _same_device, _torch, load

__all__ = ["linear", "activation_grad", "grad_norm", "adamw_step", "STATE_BLOCK"]

# Every symbol include/pam_training.h declares.
EXPORTS = ("pam_linear_workspace_size", "pam_linear", "pam_activation_grad_workspace_size", "pam_activation_grad",
           "pam_grad_norm_workspace_size", "pam_grad_norm", "pam_adamw_step")

# pam_activation_t.
ACTIVATIONS = {None: 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}

# Values of a tensor that share a scale in 8-bit states.
STATE_BLOCK = 256
# Partial sums of a norm, beside one a tensor.
NORM_PARTIALS = 2048

_bound = None


def _library() -> ctypes.CDLL:
    global _bound
    if _bound is None:
        lib = load()
        i32, i64, vp, psz = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.POINTER(ctypes.c_size_t)
        lib.pam_linear_workspace_size.argtypes = [i64, i64, i64, psz]
        lib.pam_linear.argtypes = [ctypes.c_char_p, vp]
        lib.pam_activation_grad.argtypes = [ctypes.c_char_p, vp]
        lib.pam_activation_grad_workspace_size.argtypes = [i64, i64, psz]
        lib.pam_grad_norm_workspace_size.argtypes = [ctypes.c_char_p, i64, psz]
        lib.pam_grad_norm.argtypes = [ctypes.c_char_p, i64, i32, vp, vp, i64, vp]
        lib.pam_adamw_step.argtypes = [ctypes.c_char_p, i64, ctypes.c_char_p, vp]
        for name in EXPORTS:
            getattr(lib, name).restype = i32
        _bound = lib
    return _bound


_pack_module = None


def _packer():
    """csrc/python/pack.cpp's functions."""
    global _pack_module
    if _pack_module is None:
        _torch()                                     # whose libraries _pack.so links
        try:
            from . import _pack as module
        except ImportError as e:
            raise PamError(f"_pack.so is missing: build it with `python -m paper_2305_17190_amd.build` ({e})") from e
        _pack_module = module
    return _pack_module


@functools.lru_cache(maxsize=None)
def _entry(name: str):
    """The entry point `name`, for ``_launch``: takes integers and bytes."""
    return functools.partial(_packer().call, ctypes.cast(getattr(_library(), name), ctypes.c_void_p).value)


# Calls whose arguments' types, shapes, strides and devices have been checked
# before, as in attention.py.
_calls = {}


def _known(key, plan, *args):
    """The call's plan: plan(*args) checks the arguments and makes it."""
    made = _calls.get(key)
    if made is None:
        made = plan(*args)
        if len(_calls) >= 4096:
            _calls.clear()
        _calls[key] = made
    return made


def _activation(name) -> int:
    if name not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {', '.join(map(repr, ACTIVATIONS))}, got {name!r}")
    return ACTIVATIONS[name]


def _type(dtype, name: str) -> int:
    torch = _torch()
    if dtype not in (torch.float32, torch.bfloat16):
        raise TypeError(f"{name} must be float32 or bfloat16, got {dtype}")
    return int(dtype == torch.bfloat16)


def _ld(t) -> int:
    return 0 if t is None else max(t.stride(0) if t.shape[0] > 1 and t.numel() > 0 else t.shape[1], 1)


def _rows(t, name: str, bf16_ok: bool = True):
    """A matrix whose rows are dense and, where they may be written, apart."""
    _require(t, name, 2, bf16_ok=bf16_ok)
    if t.shape[0] > 1 and t.numel() > 0 and t.stride(0) < t.shape[1]:
        raise ValueError(f"{name} has overlapping rows")


def _linear_plan(x, w, bias, residual, activation, out_dtype, mantissa_bits):
    torch = _torch()
    _rows(x, "x")
    _rows(w, "w")
    if x.dtype != w.dtype:
        raise TypeError("x and w must both be float32 or both bfloat16")
    if x.shape[1] != w.shape[1]:
        raise ValueError(f"inner dimensions differ: x is {tuple(x.shape)}, w {tuple(w.shape)}")
    m, k, n = x.shape[0], x.shape[1], w.shape[0]
    act = _activation(activation)
    if x.dtype == torch.bfloat16 and mantissa_bits < 7:
        raise ValueError("bfloat16 operands have 7 mantissa bits; round float32 operands for fewer")
    bits = 23 if x.dtype == torch.bfloat16 else mantissa_bits
    if bias is not None:
        _require(bias, "bias", 1)
        if bias.shape[0] != n:
            raise ValueError(f"bias must have {n} values, got {bias.shape[0]}")
    if out_dtype is None:
        out_dtype = torch.float32 if residual is None else residual.dtype
    out = _type(out_dtype, "out_dtype")
    if residual is not None:
        _rows(residual, "residual")
        if tuple(residual.shape) != (m, n):
            raise ValueError(f"residual must be {m}x{n}, got {tuple(residual.shape)}")
        if residual.dtype != out_dtype:
            raise TypeError(f"residual must have the output's type {out_dtype}, got {residual.dtype}")
    _same_device(x, ("w", w), ("bias", bias), ("residual", residual))
    need = ctypes.c_size_t()
    _check(_library().pam_linear_workspace_size(m, n, k, ctypes.byref(need)))
    nbytes = int(need.value)
    tail = struct.pack("=qqqqqqqqqiiii", m, n, k, _ld(x), _ld(w), _ld(residual), max(n, 1), max(n, 1), nbytes,
                       int(x.dtype == torch.bfloat16), out, act, bits)
    return tail, nbytes, out, m, n


def linear(x, w, bias=None, activation=None, residual=None, save_z: bool = False, out_dtype=None,
           mantissa_bits: int = 23):
    """A linear layer, act(x .^ w^T + bias) + residual, in the product's own
    launches; x (m x k) and w (n x k) as for ``gemm``, bias float32 (n).

    ``activation``: None, "relu", "gelu", "gelu_tanh" (the tanh approximation)
    or "silu".  Returns y, or (y, z) with ``save_z``: what the activation took,
    for ``activation_grad``.  Both, and ``residual`` (m x n), are of
    ``out_dtype``: float32 or bfloat16, the residual's type or float32 if not
    given.  float32 arithmetic, rounded once.  ``mantissa_bits`` as in
    ``gemm``."""
    mantissa_bits, save_z = int(mantissa_bits), bool(save_z)
    module = _pack_module or _packer()
    packed = module.pack(x, w, bias, residual)
    args = (x, w, bias, residual, activation, out_dtype, mantissa_bits)
    if packed is None:
        _linear_plan(*args)                          # says which argument is none
        raise TypeError("linear takes dense tensors")
    tail, nbytes, out, m, n = _known((0, packed[0], activation, out_dtype, mantissa_bits), _linear_plan, *args)
    y, z, keep, outs = module.matrices(x, nbytes, out, m, n, out if save_z else -1, m, n)
    _launch(x, _entry("pam_linear"), packed[1] + outs + tail)
    del keep
    return (y, z) if save_z else y


def _activation_grad_plan(dy, z, activation, bias, input_grad):
    torch = _torch()
    _rows(dy, "dy")
    m, n = dy.shape
    act = _activation(activation)
    if (act == 0) != (z is None):
        raise ValueError("z is given with an activation, and only then")
    if z is not None:
        _rows(z, "z")
        if z.shape != dy.shape:
            raise ValueError(f"dy {tuple(dy.shape)} and z {tuple(z.shape)} differ in shape")
        _same_device(dy, ("z", z))
    nbytes = 0
    if bias:
        need = ctypes.c_size_t()
        _check(_library().pam_activation_grad_workspace_size(m, n, ctypes.byref(need)))
        nbytes = int(need.value)
    kind = int(dy.dtype == torch.bfloat16)
    tail = struct.pack("=qqqqqqiiii", m, n, _ld(dy), _ld(z), max(n, 1), nbytes, kind,
                       int(z is not None and z.dtype == torch.bfloat16), act, 0)
    return tail, nbytes, kind if act and input_grad else -1, 0 if bias else -1, m, n


def activation_grad(dy, z, activation, bias: bool = True, input_grad: bool = True):
    """The gradient of what a linear layer adds to its product: from the
    gradient dy (m x n, float32 or bfloat16) of the layer's output and its z
    (``linear`` with ``save_z``), (dz, db): dz = dy act'(z), of dy's type, and the
    bias's gradient db, the sum of dz's rows before their rounding, in float32
    and an order fixed by the sizes.  relu's slope at 0 is 0.

    Without an activation (``activation`` and ``z`` None) dz is dy itself.
    ``bias=False`` leaves db out (None), ``input_grad=False`` dz."""
    bias, input_grad = bool(bias), bool(input_grad)
    module = _pack_module or _packer()
    packed = module.pack(dy, z)
    args = (dy, z, activation, bias, input_grad)
    if packed is None:
        _activation_grad_plan(*args)
        raise TypeError("activation_grad takes dense tensors")
    tail, nbytes, dz_type, db_type, m, n = _known((1, packed[0], activation, bias, input_grad), _activation_grad_plan,
                                                  *args)
    dz, db, keep, outs = module.matrices(dy, nbytes, dz_type, m, n, db_type, -1, n)
    if bias or dz is not None:
        _launch(dy, _entry("pam_activation_grad"), packed[1] + outs + tail)
    del keep
    return dy if activation is None and input_grad else dz, db


# The lists of a step, in the order of pam_step_tensor_t.
_LISTS = ("params", "grads", "avgs", "sqs", "avg_scales", "sq_scales", "copies")


def _check_lists(*lists) -> None:
    """What is wrong with the lists of a step."""
    torch = _torch()
    named = {}
    for name, tensors in zip(_LISTS, lists):
        if tensors is None:
            continue
        if not isinstance(tensors, (list, tuple)):
            raise TypeError(f"{name} must be a list or tuple of tensors")
        for j, t in enumerate(tensors):
            if not isinstance(t, torch.Tensor):
                raise TypeError(f"{name}[{j}] must be a torch.Tensor")
            if not t.is_cuda:
                raise PamError(f"{name}[{j}] must be a HIP (cuda) tensor; the PAM library has no CPU path")
            if t.layout != torch.strided or not t.is_contiguous():
                raise ValueError(f"{name}[{j}] must be contiguous")
        named[name] = tensors
    if "grads" not in named:
        raise TypeError("grads must be a list or tuple of tensors")
    grads = named["grads"]
    for name, tensors in named.items():
        if len(tensors) != len(grads):
            raise ValueError(f"{name} has {len(tensors)} tensors, grads {len(grads)}")
    states = [t.dtype for name in ("avgs", "sqs") for t in named.get(name, ())]
    held = states[0] if states else torch.float32
    if held not in (torch.float32, torch.uint8):
        raise TypeError(f"avgs and sqs must be float32 or uint8, got {held}")
    if states and (held == torch.uint8) != ("avg_scales" in named) or ("avg_scales" in named) != ("sq_scales" in named):
        raise ValueError("avg_scales and sq_scales are given with uint8 states, and only then")
    want = dict(params=torch.float32, avgs=held, sqs=held, avg_scales=torch.float32, sq_scales=torch.float32,
                copies=torch.bfloat16)
    for name, tensors in named.items():
        for j, t in enumerate(tensors):
            if name == "grads":
                _type(t.dtype, f"grads[{j}]")
                if t.dtype != grads[0].dtype:
                    raise TypeError(f"grads[{j}] is {t.dtype}, grads[0] {grads[0].dtype}")
            elif t.dtype != want[name]:
                raise TypeError(f"{name}[{j}] must be {want[name]}, got {t.dtype}")
            n = grads[j].numel()
            n = -(-n // STATE_BLOCK) if name.endswith("_scales") else n
            if t.numel() != n:
                raise ValueError(f"{name}[{j}] must have {n} values, got {t.numel()}")
            _same_device(grads[0], (f"{name}[{j}]", t))


def _step_tensors(*lists):
    """(count, pam_step_tensor_t array, bfloat16 gradients, 8-bit states, the first
    gradient)."""
    packed = (_pack_module or _packer()).step(*lists)
    if packed is None:
        _check_lists(*lists)
        raise TypeError("the lists hold dense tensors")
    return packed


def grad_norm(grads):
    """The square root of the sum of the squares of all gradients (a list of
    contiguous float32 or bfloat16 tensors), as a float32 tensor of no
    dimensions: ``adamw_step``'s ``norm``.  Summed in float64, in an order fixed
    by the sizes."""
    count, tensors, bf16, _, first = _step_tensors(None, grads, None, None, None, None, None)
    if count == 0:
        raise ValueError("grad_norm takes at least one gradient")
    nbytes = 8 * (NORM_PARTIALS + count)             # at least what pam_grad_norm_workspace_size says
    norm, _, keep, outs = _packer().matrices(first, nbytes, 0, -2, 1, -1, 0, 0)
    _launch(first, _entry("pam_grad_norm"), tensors, count, bf16, *_norm_outs(outs), nbytes)
    del keep
    return norm


_norm_outs = struct.Struct("=q8xq").unpack
_step_args = struct.Struct("=qqddddddqIiii").pack


def adamw_step(params, grads, avgs, sqs, step, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8,
               weight_decay: float = 0.01, avg_scales=None, sq_scales=None, copies=None, norm=None, max_norm=None,
               seed: int = 0) -> None:
    """One AdamW step over lists of contiguous tensors, in place: with g the
    gradient, limited by ``max_norm / (norm + 1e-6)`` where that is below 1,

        avg = beta1 avg + (1 - beta1) g          sq = beta2 sq + (1 - beta2) g^2
        p = p (1 - lr weight_decay) - lr / (1 - beta1^t) avg / (sqrt(sq) / sqrt(1 - beta2^t) + eps)

    ``params`` are float32, ``grads`` float32 or bfloat16 (all of one type),
    ``avgs`` and ``sqs`` float32, or uint8 with ``avg_scales`` and ``sq_scales``:
    8-bit floating point codes in blocks of ``STATE_BLOCK`` values of a tensor, a
    float32 scale each (one for the last, shorter block too), rounded
    stochastically by a hash of ``seed``, t, tensor and element (the codes:
    include/pam_training.h).  States start as zeros.  ``copies`` take the new
    parameters in bfloat16.

    ``step`` is t: an integer from 1 on, or a one-element int64 HIP tensor, read
    when the kernels run (a captured step counts on when the graph also adds 1
    to it; its parameters may differ from the integer's in their last bits).
    ``norm`` is ``grad_norm``'s result (or any float32 tensor of one element)."""
    for name, tensors in (("params", params), ("grads", grads), ("avgs", avgs), ("sqs", sqs)):
        if tensors is None:
            raise TypeError(f"{name} must be a list or tuple of tensors")
    packed = _step_tensors(params, grads, avgs, sqs, avg_scales, sq_scales, copies)
    _adamw(packed, step, lr, betas, eps, weight_decay, norm, max_norm, seed)


def _adamw(packed, step, lr, betas, eps, weight_decay, norm, max_norm, seed) -> None:
    """adamw_step over _step_tensors' lists."""
    torch = _torch()
    count, tensors, bf16, eight, first = packed
    for name, t in (("norm", norm), ("step", step if isinstance(step, torch.Tensor) else None)):
        if t is None:
            continue
        dtype = torch.float32 if name == "norm" else torch.int64
        if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.numel() != 1:
            raise TypeError(f"{name} must be a {dtype} tensor of one element")
        if not t.is_cuda:
            raise PamError(f"{name} must be a HIP (cuda) tensor; the PAM library has no CPU path")
        if first is not None:
            _same_device(first, (name, t))
    if (norm is None) != (max_norm is None):
        raise ValueError("norm and max_norm are given together")
    on_device = isinstance(step, torch.Tensor)
    args = _step_args(0 if norm is None else norm.data_ptr(), step.data_ptr() if on_device else 0, lr, betas[0], betas[1],
                      eps, weight_decay, 0.0 if max_norm is None else max_norm, 0 if on_device else int(step),
                      int(seed) & 0xFFFFFFFF, 8 if eight else 32, bf16, 0)
    if first is None:
        _check((_bound or _library()).pam_adamw_step(tensors, count, args, None))   # its refusals; launches nothing
        return
    _launch(first, _entry("pam_adamw_step"), tensors, count, args)
