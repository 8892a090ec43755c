"""The attention-side operators of a PAM transformer: norms of queries and keys
with the position rotation, a paged key/value cache, and PAM attention over it.

Thin binding over ``include/pam_attention.h`` in the manner of the package's
other calls: every step runs in the library's HIP kernels on the current
stream, nothing waits for the GPU, and there is no CPU path.

    norm_rope(q, k, positions, cos, sin, ...)        norm and rotation of queries and keys
    norm_rope_grad(dq, dk, q, k, ...)                its gradient
    append_kv(k, v, k_cache, v_cache, slots, ...)    keys and values into a paged cache
    paged_attention(q, k_cache, v_cache, ...)        softmax(scale Q .^ K^T) .^ V over the cache

Heads are (tokens, heads, d) tensors, float32 or bfloat16, with a contiguous
last dimension and any strides (views of a projection's output); caches are
(pages, page_size, heads, d) tensors, likewise.  Norm, rotation and softmax
are ordinary float32 arithmetic (Sec. 3.2 replaces the products of the linear
layers and of the attention), the attention's two products are PAM products.
"""
from __future__ import annotations

import ctypes
import math
import struct

from . import PamError, _check, _launch, _require, _same_device, _torch, load

__all__ = ["norm_rope", "norm_rope_grad", "append_kv", "paged_attention"]

# Every symbol include/pam_attention.h declares.
EXPORTS = ("pam_norm_rope", "pam_norm_rope_grad_workspace_size", "pam_norm_rope_grad", "pam_append_kv",
           "pam_paged_attention_workspace_size", "pam_paged_attention")

# The argument structures of include/pam_attention.h: the pointers, then the
# layouts and sizes (``_HEADS``, ``_ROTATION``, ``_CACHE``).
_HEADS, _ROTATION, _CACHE = "qqii", "qii", "qqqqiiii"
_NONE = (0, 0, 0, 0)

_bound = None


def _library() -> ctypes.CDLL:
    global _bound
    if _bound is None:
        lib = load()
        i32, i64, vp, psz = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.POINTER(ctypes.c_size_t)
        for name in ("pam_norm_rope", "pam_norm_rope_grad", "pam_append_kv", "pam_paged_attention"):
            getattr(lib, name).argtypes = [ctypes.c_char_p, vp]
        lib.pam_norm_rope_grad_workspace_size.argtypes = [i64, i32, i32, i32, psz]
        lib.pam_paged_attention_workspace_size.argtypes = [i32, i32, i32, i32, i32, i32, i32, psz]
        for name in EXPORTS:
            getattr(lib, name).restype = i32
        _bound = lib
    return _bound


def _is_bf16(t) -> int:
    return int(t.dtype == _torch().bfloat16)


def _heads(t):
    return _NONE if t is None else (t.stride(0), t.stride(1), t.shape[1], _is_bf16(t))


def _cache(t):
    return (t.stride(0), t.stride(1), t.stride(2), t.shape[0], t.shape[1], t.shape[2], _is_bf16(t), 0)


def _ints(t, name: str, dtype, *shape):
    """An index tensor of the given type and shape (None: any), contiguous, on the GPU."""
    torch = _torch()
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != len(shape) or any(want is not None and have != want for have, want in zip(t.shape, shape)):
        raise ValueError(f"{name} must have shape {shape}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _weight(w, name: str, d: int):
    if w is not None:
        _require(w, name, 1)
        if w.shape[0] != d:
            raise ValueError(f"{name} must have {d} values, got {w.shape[0]}")


def _rotation(positions, cos, sin, interleaved: bool, tokens: int, d: int):
    """The rotation's layout; rot = 0 where there is none."""
    torch = _torch()
    given = [x is not None for x in (positions, cos, sin)]
    if not any(given):
        return (0, 0, 0)
    if not all(given):
        raise ValueError("positions, cos and sin must be given together")
    _ints(positions, "positions", torch.int32, tokens)
    for name, t in (("cos", cos), ("sin", sin)):
        _require(t, name, 2)
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    if cos.shape != sin.shape:
        raise ValueError(f"cos and sin differ in shape: {tuple(cos.shape)} and {tuple(sin.shape)}")
    if 2 * cos.shape[1] > d:
        raise ValueError(f"the tables turn {2 * cos.shape[1]} values, the heads have {d}")
    return (cos.shape[0], 2 * cos.shape[1], int(interleaved))


def _head_tensors(*named):
    """Checks the (tokens, heads, d) tensors that are given; they agree in
    tokens, d, type and device with the first."""
    first = None
    for name, t in named:
        if t is None:
            continue
        _require(t, name, 3, bf16_ok=True)
        if first is None:
            first = (name, t)
            continue
        ref = first[1]
        if t.shape[0] != ref.shape[0] or t.shape[2] != ref.shape[2]:
            raise ValueError(f"{name} {tuple(t.shape)} and {first[0]} {tuple(ref.shape)} differ in tokens or head size")
        if t.dtype != ref.dtype:
            raise TypeError(f"{name} is {t.dtype}, {first[0]} {ref.dtype}")
        _same_device(ref, (name, t))
    if first is None:
        raise ValueError("neither queries nor keys given")
    return first[1]


# Calls whose arguments' types, shapes, strides and devices have been checked
# before: by all of these, the part of the argument structure that follows the
# pointers, and what else the call needs.  (Checked anew, each call of
# append_kv took 21 us of host time, of paged_attention 15.)
_calls = {}
_pack_tensors = _make = None                         # of csrc/python/pack.cpp


def _pack(*tensors):
    """(key, addresses) of the tensors; None where one is none."""
    global _pack_tensors, _make
    if _pack_tensors is None:
        _torch()                                     # whose libraries _pack.so links
        try:
            from . import _pack as module
        except ImportError as e:
            raise PamError(f"_pack.so is missing: build it with `python -m paper_2305_17190_amd.build` ({e})") from e
        _make = module.make                          # first: the calls look at _pack_tensors alone
        _pack_tensors = module.pack
    return _pack_tensors(*tensors)


def _known(key, plan, *args):
    """The call's plan: plan(*args) checks the arguments and makes it."""
    made = _calls.get(key)
    if made is None:
        made = plan(*args)
        if len(_calls) >= 4096:
            _calls.clear()
        _calls[key] = made
    return made


def _norm_rope_plan(q, k, positions, cos, sin, q_weight, k_weight, eps, interleaved, out_dtype):
    torch = _torch()
    ref = _head_tensors(("q", q), ("k", k))
    tokens, _, d = ref.shape
    _weight(q_weight, "q_weight", d)
    _weight(k_weight, "k_weight", d)
    rot = _rotation(positions, cos, sin, interleaved, tokens, d)
    _same_device(ref, ("q_weight", q_weight), ("k_weight", k_weight), ("positions", positions), ("cos", cos),
                 ("sin", sin))
    dtype = ref.dtype if out_dtype is None else out_dtype
    if dtype not in (torch.float32, torch.bfloat16):
        raise TypeError(f"out_dtype must be float32 or bfloat16, got {dtype}")
    outs = [_NONE if t is None else (t.shape[1] * d, d, t.shape[1], int(dtype == torch.bfloat16)) for t in (q, k)]
    tail = struct.pack("=" + _HEADS * 4 + _ROTATION + "qif", *_heads(q), *outs[0], *_heads(k), *outs[1], *rot, tokens, d,
                       eps)
    return tail, int(dtype == torch.bfloat16)


def norm_rope(q, k, positions=None, cos=None, sin=None, q_weight=None, k_weight=None, eps: float = 1e-6,
              interleaved: bool = False, out_dtype=None):
    """Norm and position rotation of queries (tokens, heads, d) and keys (tokens,
    key heads, d) in one pass; returns (q', k'), either input may be None.

    With a weight (d float32 values) a head's values x become x * weight /
    sqrt(mean(x^2) + eps).  ``cos`` and ``sin`` are float32 (rows, rot / 2)
    tables, ``positions`` int32 (tokens): the first ``rot`` values of each head
    are turned in pairs (p, p + rot / 2), or (2p, 2p + 1) if ``interleaved``,
    by the angles of the token's position.  float32 arithmetic, rounded once to
    ``out_dtype`` (the inputs' type)."""
    eps, interleaved = float(eps), bool(interleaved)
    if q is None:
        q_weight = None
    if k is None:
        k_weight = None
    packed = (_pack_tensors or _pack)(q, q_weight, k, k_weight, positions, cos, sin)
    args = (q, k, positions, cos, sin, q_weight, k_weight, eps, interleaved, out_dtype)
    if packed is None:
        _norm_rope_plan(*args)                       # says which argument is none
        raise TypeError("norm_rope takes dense tensors")
    tail, bf16 = _known((0, packed[0], eps, interleaved, out_dtype), _norm_rope_plan, *args)
    qo, ko, _, outs = _make(bf16, 0, q, k)
    _launch(q if q is not None else k, (_bound or _library()).pam_norm_rope, packed[1] + outs[:-8] + tail)
    return qo, ko


def _norm_rope_grad_plan(dq, dk, q, k, positions, cos, sin, q_weight, k_weight, eps, interleaved):
    if (dq is None) != (q is None) or (dk is None) != (k is None):
        raise ValueError("q and dq, k and dk must be given together")
    ref = _head_tensors(("q", q), ("dq", dq), ("k", k), ("dk", dk))
    for x, dx, name in ((q, dq, "dq"), (k, dk, "dk")):
        if x is not None and x.shape != dx.shape:
            raise ValueError(f"{name} must have shape {tuple(x.shape)}, got {tuple(dx.shape)}")
    tokens, _, d = ref.shape
    _weight(q_weight, "q_weight", d)
    _weight(k_weight, "k_weight", d)
    rot = _rotation(positions, cos, sin, interleaved, tokens, d)
    _same_device(ref, ("q_weight", q_weight), ("k_weight", k_weight), ("positions", positions), ("cos", cos),
                 ("sin", sin))
    nbytes = 0
    if q_weight is not None or k_weight is not None:
        need = ctypes.c_size_t()
        _check(_library().pam_norm_rope_grad_workspace_size(tokens, d, 0 if q is None else q.shape[1],
                                                            0 if k is None else k.shape[1], ctypes.byref(need)))
        nbytes = int(need.value)
    outs = [_NONE if t is None else (t.shape[1] * d, d, t.shape[1], _is_bf16(t)) for t in (q, k)]
    tail = struct.pack("=" + _HEADS * 6 + _ROTATION + "qqif", *_heads(q), *_heads(dq), *outs[0], *_heads(k), *_heads(dk),
                       *outs[1], *rot, tokens, nbytes, d, eps)
    return tail, nbytes


def norm_rope_grad(dq, dk, q, k, positions=None, cos=None, sin=None, q_weight=None, k_weight=None,
                   eps: float = 1e-6, interleaved: bool = False):
    """Gradient of ``norm_rope``: from the gradients (dq, dk) of its outputs and
    its inputs, (gradient of q, of k, of q_weight, of k_weight); None for what
    was not given.  Gradients have their input's type, the weights' float32."""
    eps, interleaved = float(eps), bool(interleaved)
    if q is None:
        q_weight = None
    if k is None:
        k_weight = None
    packed = (_pack_tensors or _pack)(q, q_weight, dq, k, k_weight, dk, positions, cos, sin)
    args = (dq, dk, q, k, positions, cos, sin, q_weight, k_weight, eps, interleaved)
    if packed is None:
        _norm_rope_grad_plan(*args)
        raise TypeError("norm_rope_grad takes dense tensors")
    tail, nbytes = _known((1, packed[0], eps, interleaved), _norm_rope_grad_plan, *args)
    gq, gqw, gk, gkw, keep, outs = _make(-1, nbytes, q, q_weight, k, k_weight)
    _launch(q if q is not None else k, (_bound or _library()).pam_norm_rope_grad, packed[1] + outs + tail)
    del keep
    return gq, gk, gqw, gkw


def _caches(k_cache, v_cache):
    for name, t in (("k_cache", k_cache), ("v_cache", v_cache)):
        _require(t, name, 4, bf16_ok=True)
    if k_cache.shape != v_cache.shape:
        raise ValueError(f"the caches differ in shape: {tuple(k_cache.shape)} and {tuple(v_cache.shape)}")
    _same_device(k_cache, ("v_cache", v_cache))


def _append_plan(k, v, k_cache, v_cache, slots, positions, cos, sin, k_weight, q, q_weight, eps, interleaved):
    torch = _torch()
    ref = _head_tensors(("k", k), ("v", v), ("q", q))
    _caches(k_cache, v_cache)
    tokens, heads, d = k.shape
    if v.shape != k.shape or tuple(k_cache.shape[2:]) != (heads, d):
        raise ValueError(f"k {tuple(k.shape)}, v {tuple(v.shape)} and caches {tuple(k_cache.shape)} do not agree")
    _weight(q_weight, "q_weight", d)
    _weight(k_weight, "k_weight", d)
    _ints(slots, "slots", torch.int64, tokens)
    rot = _rotation(positions, cos, sin, interleaved, tokens, d)
    _same_device(ref, ("k_cache", k_cache), ("slots", slots), ("q_weight", q_weight), ("k_weight", k_weight),
                 ("positions", positions), ("cos", cos), ("sin", sin))
    out = _NONE if q is None else (q.shape[1] * d, d, q.shape[1], _is_bf16(q))
    return struct.pack("=" + _HEADS * 4 + _CACHE * 2 + _ROTATION + "qif", *_heads(k), *_heads(v), *_heads(q), *out,
                       *_cache(k_cache), *_cache(v_cache), *rot, tokens, d, eps)


def append_kv(k, v, k_cache, v_cache, slots, positions=None, cos=None, sin=None, k_weight=None, q=None, q_weight=None,
              eps: float = 1e-6, interleaved: bool = False):
    """Writes the keys and values (tokens, key heads, d) of new tokens into the
    paged caches (pages, page_size, key heads, d): token t to slot ``slots[t]``
    (int64, page * page_size + place; outside the cache, as -1: not stored).
    Keys are normed (``k_weight``) and rotated as by ``norm_rope`` on the way;
    both are rounded to the cache's type.  With ``q``, the same tokens' queries
    are normed (``q_weight``) and rotated in the same launch and returned in
    q's type, else None."""
    eps, interleaved = float(eps), bool(interleaved)
    if q is None:
        q_weight = None
    packed = (_pack_tensors or _pack)(k, k_weight, v, q, q_weight, slots, positions, cos, sin, k_cache, v_cache)
    args = (k, v, k_cache, v_cache, slots, positions, cos, sin, k_weight, q, q_weight, eps, interleaved)
    if packed is None:
        _append_plan(*args)
        raise TypeError("append_kv takes dense tensors")
    tail = _known((2, packed[0], eps, interleaved), _append_plan, *args)
    qo, _, outs = _make(-1, 0, q)
    _launch(k, (_bound or _library()).pam_append_kv, packed[1] + outs[:-8] + tail)
    return qo


# Workspace bytes of an attention call by its sizes, as the library reports them.
_attention_bytes = {}


def _attention_workspace(sizes: tuple) -> int:
    nbytes = _attention_bytes.get(sizes)
    if nbytes is None:
        need = ctypes.c_size_t()
        _check(_library().pam_paged_attention_workspace_size(*sizes, ctypes.byref(need)))
        nbytes = int(need.value)
        if len(_attention_bytes) >= 4096:
            _attention_bytes.clear()
        _attention_bytes[sizes] = nbytes
    return nbytes


_attention_end = struct.Struct("=iiq").pack
_MOST_INT = 2 ** 31 - 1


def _count(value, name: str) -> int:
    value = int(value)
    if not 0 <= value <= _MOST_INT:
        raise ValueError(f"{name} must be in [0, 2^31), got {value}")
    return value


def _attention_plan(q, k_cache, v_cache, table, kv_lens, q_starts, scale, causal, window, out):
    torch = _torch()
    _require(q, "q", 3, bf16_ok=True)
    _caches(k_cache, v_cache)
    tokens, heads, d = q.shape
    page_size, kv_heads, cache_d = k_cache.shape[1:]
    if k_cache.dtype != v_cache.dtype:
        raise TypeError(f"the caches differ in type: {k_cache.dtype} and {v_cache.dtype}")
    if cache_d != d:
        raise ValueError(f"q has heads of {d} values, the caches of {cache_d}")
    if not isinstance(kv_lens, torch.Tensor) or kv_lens.dim() != 1:
        raise ValueError("kv_lens must be a one-dimensional tensor")
    batch = kv_lens.shape[0]
    _ints(kv_lens, "kv_lens", torch.int32, batch)
    _ints(table, "table", torch.int32, batch, None)
    if q_starts is not None:
        _ints(q_starts, "q_starts", torch.int32, batch + 1)
    elif tokens != batch:
        raise ValueError(f"without q_starts q must have one token a sequence: {tokens} tokens, {batch} sequences")
    if window < 0:
        raise ValueError("window must be >= 0")
    outs = (heads * d, d, heads, 0)
    if out is not None:
        _require(out, "out", 3)
        if out.shape != q.shape:
            raise ValueError(f"out must have shape {tuple(q.shape)}, got {tuple(out.shape)}")
        outs = _heads(out)
    _same_device(q, ("k_cache", k_cache), ("table", table), ("kv_lens", kv_lens), ("q_starts", q_starts), ("out", out))
    width = table.shape[1]
    tail = struct.pack("=" + _HEADS * 2 + _CACHE * 2 + "qqiiiiif", *_heads(q), *outs, *_cache(k_cache), *_cache(v_cache),
                       width, tokens, d, batch, width, int(causal), window, 1.0 / math.sqrt(d) if scale is None else scale)
    return tail, (d, heads, kv_heads, _is_bf16(k_cache), batch), width * page_size


def paged_attention(q, k_cache, v_cache, table, kv_lens, q_starts=None, max_q: int | None = None,
                    max_kv: int | None = None, scale: float | None = None, causal: bool = True, window: int = 0, out=None):
    """softmax(scale Q .^ K^T) .^ V of new tokens over a paged cache, as float32
    (tokens, heads, d).

    ``q`` (tokens, heads, d) holds the new tokens of all sequences in order;
    sequence b's are ``q_starts[b] : q_starts[b + 1]`` (int32, batch + 1
    entries), at most ``max_q`` (all of q) of them; without ``q_starts`` every
    sequence has one.  ``kv_lens`` (int32) counts each sequence's cached keys, its
    new ones among them as the last; ``table`` (int32, batch x pages a row) names
    their pages.  ``max_kv`` (the table's whole reach) bounds ``kv_lens``: the
    nearer the two bounds are, the better the work is cut.  A token sees its
    sequence's keys up to its own position (all, without ``causal``), the last
    ``window`` of them where that is positive; a token without keys gets zeros.
    ``scale`` is 1 / sqrt(d) if not given.  Tokens of no sequence are left
    unwritten."""
    # Keys count to below 2^31: a window of as many is as good as a wider one.
    causal, window, scale = bool(causal), min(int(window), _MOST_INT), None if scale is None else float(scale)
    packed = (_pack_tensors or _pack)(q, k_cache, v_cache, q_starts, kv_lens, table, out)
    args = (q, k_cache, v_cache, table, kv_lens, q_starts, scale, causal, window, out)
    if packed is None:
        _attention_plan(*args)
        raise TypeError("paged_attention takes dense tensors")
    tail, sizes, reach = _known((3, packed[0], scale, causal, window), _attention_plan, *args)
    max_q = 1 if q_starts is None else q.shape[0] if max_q is None else _count(max_q, "max_q")
    max_kv = min(reach, _MOST_INT) if max_kv is None else _count(max_kv, "max_kv")
    nbytes = _attention_workspace((*sizes, max_q, max_kv))
    if out is None:
        out, keep, outs = _make(0, nbytes, q)
        pointers = packed[1][:-8] + outs
    else:
        _, keep, outs = _make(0, nbytes, q[:0])
        pointers = packed[1] + outs[8:]
    _launch(q, (_bound or _library()).pam_paged_attention, pointers + tail + _attention_end(max_q, max_kv, nbytes))
    del keep
    return out
