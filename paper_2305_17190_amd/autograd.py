"""PyTorch autograd wrappers over the PAM matrix products.

Sec. 3.2 of the paper replaces every multiplication of a linear layer and of
the attention's batched products by PAM, and Table 1 gives the backward pass
used in training, the approximate derivative: the gradients are PAM products
of the incoming gradient with the other operand, exactly as a standard
matrix multiply's gradients are ordinary products.

    Y = X .^ W^T (+ b)     dX = dY .^ W       dW = dY^T .^ X     db = sum dY
    C = A .^ B (batched)   dA = dC .^ B^T     dB = A^T .^ dC

Every product runs in the library's HIP kernels (``pam.gemm`` / ``pam.bmm``);
the bias gradient is an ordinary sum (no multiplication).  ``pam_linear``
and ``PAMLinear`` also offer Table 1's exact derivative
(``derivative="exact"``): dX[i,k] = sum_j dY[i,j] d(X[i,k] .^ W[j,k])/dX[i,k]
and dW likewise, through ``pam.exact_grad``.  With
``mantissa_bits`` < 23 every product, forward and backward, first rounds its
two operands to that many mantissa bits (App. "PAM with Narrower
Mantissas"); the tensors themselves are not modified.  Inputs must be float32
HIP tensors; there is no CPU path.  First derivatives only: what a second one
would need of a backward pass's products raises.

``pam_norm_rope`` is the attention's norm of queries and keys with the position
rotation (``pam.norm_rope``), ordinary arithmetic, float32 or bfloat16.
"""
from __future__ import annotations

import math

import torch

from . import bmm as _bmm
from . import exact_grad as _exact_grad
from . import gemm as _gemm
from . import norm_rope as _norm_rope
from . import norm_rope_grad as _norm_rope_grad

__all__ = ["pam_linear", "pam_matmul", "pam_norm_rope", "PAMLinear"]


class _FirstOrder(torch.autograd.Function):
    """A backward pass's own kernels under ``create_graph``: they record nothing,
    so that a second derivative would count their results as constants."""

    @staticmethod
    def forward(ctx, gradients, *tensors):
        return gradients(*tensors)

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("the PAM wrappers have first derivatives only")


def _first_order(gradients, *tensors):
    """gradients(*tensors); differentiating the results raises."""
    if torch.is_grad_enabled():
        return _FirstOrder.apply(gradients, *tensors)
    return gradients(*tensors)


def _float32(**named) -> None:
    """The wrappers' gradients are float32 products: refuse other dtypes up
    front rather than in the backward pass."""
    for name, t in named.items():
        if t is not None and t.dtype != torch.float32:
            raise TypeError(f"{name} must be float32, got {t.dtype}")


def _last_contiguous(t: torch.Tensor) -> torch.Tensor:
    """t itself when its rows are dense and non-overlapping (a valid leading
    dimension for the C ABI), else a contiguous copy."""
    ok = t.stride(-1) == 1 and (t.dim() < 2 or t.shape[-2] <= 1 or t.stride(-2) >= t.shape[-1])
    return t if ok else t.contiguous()


class _PAMLinearFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x2d, weight, bias, bits, exact):
        x2d = _last_contiguous(x2d)
        weight = _last_contiguous(weight)
        ctx.save_for_backward(x2d, weight)
        ctx.has_bias = bias is not None
        ctx.bits = bits
        ctx.exact = exact
        y = _gemm(x2d, weight, trans_b=True, mantissa_bits=bits)   # Y = X .^ W^T
        if bias is not None:
            y += bias
        return y

    @staticmethod
    def backward(ctx, dy):
        x2d, weight = ctx.saved_tensors
        dy = _last_contiguous(dy)
        dx = dw = db = None
        # Under create_graph each result's first two operands count as what it depends
        # on: the exact derivative is constant in the operand it is taken by.
        if ctx.exact:
            if ctx.needs_input_grad[0]:                                     # sum_j dY d(X .^ W)/dX
                dx = _first_order(lambda d, w: _exact_grad(d, w, x2d), dy, weight)
            if ctx.needs_input_grad[1]:                                     # sum_i dY d(W .^ X)/dW
                dw = _first_order(lambda d, x: _exact_grad(d, x, weight, trans_a=True), dy, x2d)
        else:
            if ctx.needs_input_grad[0]:                                     # dX = dY .^ W
                dx = _first_order(lambda d, w: _gemm(d, w, mantissa_bits=ctx.bits), dy, weight)
            if ctx.needs_input_grad[1]:                                     # dW = dY^T .^ X
                dw = _first_order(lambda d, x: _gemm(d, x, trans_a=True, mantissa_bits=ctx.bits), dy, x2d)
        if ctx.has_bias and ctx.needs_input_grad[2]:
            db = dy.sum(dim=0)
        return dx, dw, db, None, None


def pam_linear(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor = None,
               mantissa_bits: int = 23, derivative: str = "approximate") -> torch.Tensor:
    """``x .^ weight^T + bias`` over the last dimension of x (any leading dims).

    ``derivative``: "approximate" (Table 1's approximate derivative, PAM
    products) or "exact" (Table 1's exact derivative)."""
    if x.dim() < 1:
        raise ValueError("x must have at least one dimension")
    if derivative not in ("approximate", "exact"):
        raise ValueError('derivative must be "approximate" or "exact"')
    if derivative == "exact" and mantissa_bits != 23:
        raise ValueError("the exact derivative takes full float32 mantissas")
    _float32(x=x, weight=weight, bias=bias)
    lead = x.shape[:-1]
    y = _PAMLinearFn.apply(x.reshape(-1, x.shape[-1]), weight, bias, int(mantissa_bits), derivative == "exact")
    return y.reshape(*lead, weight.shape[0])


class _PAMBmmFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, a, b, bits):
        a = _last_contiguous(a)
        b = _last_contiguous(b)
        ctx.save_for_backward(a, b)
        ctx.bits = bits
        return _bmm(a, b, mantissa_bits=bits)                 # C = A .^ B

    @staticmethod
    def backward(ctx, dc):
        a, b = ctx.saved_tensors
        dc = _last_contiguous(dc)
        da = db = None
        if ctx.needs_input_grad[0]:
            da = _first_order(lambda d, b: _bmm(d, b, trans_b=True, mantissa_bits=ctx.bits), dc, b)     # dA = dC .^ B^T
        if ctx.needs_input_grad[1]:
            db = _first_order(lambda a, d: _bmm(a, d, trans_a=True, mantissa_bits=ctx.bits), a, dc)     # dB = A^T .^ dC
        return da, db, None


def pam_matmul(a: torch.Tensor, b: torch.Tensor, mantissa_bits: int = 23) -> torch.Tensor:
    """``a .^ b`` for 2-D or batched 3-D operands (leading batch dimension)."""
    _float32(a=a, b=b)
    if a.dim() == 2 and b.dim() == 2:
        return _PAMBmmFn.apply(a.unsqueeze(0), b.unsqueeze(0), int(mantissa_bits)).squeeze(0)
    if a.dim() == 3 and b.dim() == 3:
        return _PAMBmmFn.apply(a, b, int(mantissa_bits))
    raise ValueError("pam_matmul takes two 2-D or two 3-D tensors")


def _dense_heads(t: torch.Tensor) -> torch.Tensor:
    return t if t is None or t.stride(-1) == 1 or t.numel() == 0 else t.contiguous()


class _NormRopeFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, positions, cos, sin, q_weight, k_weight, eps, interleaved):
        q, k = _dense_heads(q), _dense_heads(k)
        ctx.save_for_backward(q, k, positions, cos, sin, q_weight, k_weight)
        ctx.rest = eps, interleaved
        return _norm_rope(q, k, positions, cos, sin, q_weight, k_weight, eps, interleaved)

    @staticmethod
    def backward(ctx, dq, dk):
        q, k, positions, cos, sin, qw, kw = ctx.saved_tensors
        needs = ctx.needs_input_grad
        if not (needs[0] or needs[5]):
            dq = q = qw = None
        if not (needs[1] or needs[6]):
            dk = k = kw = None
        gq, gk, gqw, gkw = _first_order(lambda *tensors: _norm_rope_grad(*tensors, *ctx.rest), _dense_heads(dq),
                                        _dense_heads(dk), q, k, positions, cos, sin, qw, kw)
        return gq, gk, None, None, None, gqw, gkw, None, None


def pam_norm_rope(q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor = None, cos: torch.Tensor = None,
                  sin: torch.Tensor = None, q_weight: torch.Tensor = None, k_weight: torch.Tensor = None,
                  eps: float = 1e-6, interleaved: bool = False):
    """``pam.norm_rope`` of queries and keys (tokens, heads, d) with gradients for
    q, k and the weights; the tables of angles are constants."""
    if q is None or k is None:
        raise ValueError("pam_norm_rope takes queries and keys; norm_rope takes one of them")
    return _NormRopeFn.apply(q, k, positions, cos, sin, q_weight, k_weight, eps, interleaved)


class PAMLinear(torch.nn.Module):
    """A linear layer whose products are PAM (forward and approximate-derivative backward)."""

    def __init__(self, in_features: int, out_features: int, bias: bool = True, device=None,
                 mantissa_bits: int = 23, derivative: str = "approximate"):
        super().__init__()
        self.in_features = in_features
        self.out_features = out_features
        self.mantissa_bits = mantissa_bits
        self.derivative = derivative
        self.weight = torch.nn.Parameter(torch.empty(out_features, in_features, device=device))
        self.bias = torch.nn.Parameter(torch.empty(out_features, device=device)) if bias else None
        self.reset_parameters()

    def reset_parameters(self) -> None:
        bound = 1.0 / math.sqrt(self.in_features) if self.in_features > 0 else 0.0
        with torch.no_grad():
            self.weight.uniform_(-bound, bound)
            if self.bias is not None:
                self.bias.uniform_(-bound, bound)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        return pam_linear(x, self.weight, self.bias, self.mantissa_bits, self.derivative)

    def extra_repr(self) -> str:
        return (f"in_features={self.in_features}, out_features={self.out_features}, bias={self.bias is not None}, "
                f"mantissa_bits={self.mantissa_bits}, derivative={self.derivative}")
