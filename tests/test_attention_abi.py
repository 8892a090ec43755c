"""The attention-side entry points on the host: every declared symbol is
exported, and bad arguments are refused before anything is launched."""
import ctypes
import os
import re

import pytest

import paper_2305_17190_amd as pam
from paper_2305_17190_amd import attention as att

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "pam_attention.h")
P = 4096          # stands for every device address
INVALID = 1


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pam.library_path()):
        pytest.skip("libpam.so not built (run __graft_entry__.build())")
    return att._library()


class Heads(ctypes.Structure):
    _fields_ = [("stride_token", ctypes.c_int64), ("stride_head", ctypes.c_int64), ("heads", ctypes.c_int32),
                ("type", ctypes.c_int32)]


class Rotation(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("rot", ctypes.c_int32), ("interleaved", ctypes.c_int32)]


class Cache(ctypes.Structure):
    _fields_ = [("stride_page", ctypes.c_int64), ("stride_slot", ctypes.c_int64), ("stride_head", ctypes.c_int64),
                ("pages", ctypes.c_int64), ("page_size", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("type", ctypes.c_int32), ("reserved", ctypes.c_int32)]


def heads(token=512, head=64, count=8, kind=0):
    return Heads(token, head, count, kind)


def cache(page=8192, slot=512, head=64, pages=10, size=16, count=8, kind=0):
    return Cache(page, slot, head, pages, size, count, kind, 0)


def rotation(rows=100, rot=64, interleaved=0):
    return Rotation(rows, rot, interleaved)


NONE = heads(0, 0, 0, 0)


def call(lib, name, pointers, layouts, **changes):
    """The entry point `name` on a structure of `pointers` (names, all valid)
    and then `layouts` (name, C type, value), with some of them changed."""
    fields = [(n, ctypes.c_void_p) for n in pointers] + [(n, t) for n, t, _ in layouts]
    values = dict({n: P for n in pointers}, **{n: v for n, _, v in layouts})
    assert set(changes) <= set(values), set(changes) - set(values)
    values.update(changes)
    args = type(name, (ctypes.Structure,), {"_fields_": fields})(*(values[n] for n, _ in fields))
    return getattr(lib, name)(bytes(args), None)


def test_every_declared_symbol_is_exported(lib):
    with open(HEADER) as f:
        text = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    names = set(re.findall(r"\b(pam_[a-z_0-9]+)\s*\(", text))
    assert names == set(att.EXPORTS)
    for name in names:
        assert hasattr(lib, name)


I32, I64, F32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_float


def norm_rope(lib, **kw):
    return call(lib, "pam_norm_rope", ["q_in", "q_weight", "k_in", "k_weight", "positions", "cos", "sin", "q_out", "k_out"],
                [(n, Heads, heads()) for n in ("q_in_heads", "q_out_heads", "k_in_heads", "k_out_heads")]
                + [("rotation", Rotation, rotation()), ("tokens", I64, 4), ("d", I32, 64), ("eps", F32, 1e-6)], **kw)


BAD_HEADS = [heads(count=-1), heads(token=-1), heads(head=-5), heads(kind=2), heads(token=1 << 60)]
BAD_ROTATIONS = [dict(positions=None), dict(cos=None), dict(sin=None)] + [
    dict(rotation=r) for r in (rotation(rot=63), rotation(rot=66), rotation(rot=-2), rotation(rows=-1),
                               rotation(rows=1 << 31))]


@pytest.mark.parametrize("kw", [
    dict(tokens=-1), dict(d=63), dict(d=0), dict(d=258), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
    dict(q_out_heads=NONE), dict(k_in_heads=NONE), dict(q_in=None), dict(k_out=None),
    dict(q_in_heads=NONE, q_out_heads=NONE, k_in_heads=NONE, k_out_heads=NONE), dict(k_in_heads=heads(kind=1)),
    dict(q_out_heads=heads(count=4)), dict(q_out_heads=heads(token=32)), dict(k_out_heads=heads(head=63)),
    dict(tokens=1 << 30)] + [dict(q_in_heads=h) for h in BAD_HEADS] + [dict(k_out_heads=h) for h in BAD_HEADS]
    + BAD_ROTATIONS)
def test_norm_rope_refuses(lib, kw):
    assert norm_rope(lib, **kw) == INVALID and lib.pam_last_error() != b""


def test_no_arguments_are_refused(lib):
    for name in ("pam_norm_rope", "pam_norm_rope_grad", "pam_append_kv", "pam_paged_attention"):
        assert getattr(lib, name)(None, None) == INVALID


def test_nothing_to_do_launches_nothing(lib):
    assert norm_rope(lib, tokens=0, q_in=None, q_out=None, k_in=None, k_out=None, positions=None, cos=None, sin=None) == 0
    assert append(lib, tokens=0, k=None, v=None, k_cache=None, v_cache=None, slots=None, q_in_heads=NONE,
                  q_out_heads=NONE, rotation=rotation(rot=0)) == 0
    assert attention(lib, batch=0) == 0
    assert attention(lib, tokens=0, q=None, out=None) == 0
    assert grad(lib, tokens=0, q_weight=None, dq_weight=None, k_weight=None, dk_weight=None, workspace=None) == 0


def grad(lib, **kw):
    return call(lib, "pam_norm_rope_grad",
                ["q_in", "q_weight", "dq_out", "k_in", "k_weight", "dk_out", "positions", "cos", "sin", "dq_in", "dq_weight",
                 "dk_in", "dk_weight", "workspace"],
                [(n + "_heads", Heads, heads()) for n in ("q_in", "dq_out", "dq_in", "k_in", "dk_out", "dk_in")]
                + [("rotation", Rotation, rotation()), ("tokens", I64, 4), ("workspace_bytes", I64, 1 << 30),
                   ("d", I32, 64), ("eps", F32, 1e-6)], **kw)


@pytest.mark.parametrize("kw", [
    dict(tokens=-1), dict(d=65), dict(eps=-1.0), dict(dq_out_heads=NONE), dict(dk_in_heads=NONE), dict(q_in_heads=NONE),
    dict(dq_out=None), dict(dk_in=None), dict(q_weight=None), dict(dk_weight=None),
    dict(q_in_heads=NONE, dq_out_heads=NONE, dq_in_heads=NONE), dict(dq_out_heads=heads(count=3)),
    dict(dq_in_heads=heads(kind=1)), dict(dk_out_heads=heads(kind=1)), dict(dq_in_heads=heads(token=8)),
    dict(workspace=None), dict(workspace_bytes=8), dict(workspace_bytes=-1), dict(workspace=P + 4)]
    + [dict(dq_out_heads=h) for h in BAD_HEADS] + BAD_ROTATIONS)
def test_grad_refuses(lib, kw):
    assert grad(lib, **kw) == INVALID and lib.pam_last_error() != b""


def test_grad_workspace_sizes(lib):
    need = ctypes.c_size_t()
    size = lib.pam_norm_rope_grad_workspace_size
    assert size(4, 64, 8, 8, None) == INVALID
    for bad in ((-1, 64, 8, 8), (4, 63, 8, 8), (4, 64, -1, 8), (4, 64, 0, 0), (1 << 30, 64, 8, 8)):
        assert size(*bad, ctypes.byref(need)) == INVALID
    assert size(0, 64, 8, 8, ctypes.byref(need)) == 0 and need.value == 0
    last = 0
    for tokens in (1, 10, 1000, 100000):
        assert size(tokens, 64, 8, 2, ctypes.byref(need)) == 0
        assert need.value >= last and need.value <= 16 << 20
        last = need.value


def append(lib, **kw):
    return call(lib, "pam_append_kv",
                ["k", "k_weight", "v", "q_in", "q_weight", "slots", "positions", "cos", "sin", "k_cache", "v_cache", "q_out"],
                [(n, Heads, heads()) for n in ("k_heads", "v_heads", "q_in_heads", "q_out_heads")]
                + [("k_cache_layout", Cache, cache()), ("v_cache_layout", Cache, cache()),
                   ("rotation", Rotation, rotation()), ("tokens", I64, 4), ("d", I32, 64), ("eps", F32, 1e-6)], **kw)


BAD_CACHES = [cache(page=-1), cache(slot=-1), cache(head=-1), cache(pages=-1), cache(size=0), cache(count=0),
              cache(kind=7), cache(pages=1 << 27), cache(page=1 << 60)]


@pytest.mark.parametrize("kw", [
    dict(tokens=-1), dict(d=7), dict(k=None), dict(v=None), dict(k_cache=None), dict(v_cache=None), dict(slots=None),
    dict(q_out_heads=NONE), dict(q_out=None), dict(v_heads=heads(kind=1)), dict(q_in_heads=heads(kind=1)),
    dict(k_heads=heads(count=4)), dict(v_heads=heads(count=4)), dict(k_heads=NONE), dict(v_cache_layout=cache(pages=9)),
    dict(v_cache_layout=cache(size=8)), dict(q_out_heads=heads(count=2)), dict(q_out_heads=heads(head=8))]
    + [dict(k_heads=h) for h in BAD_HEADS] + [dict(v_cache_layout=c) for c in BAD_CACHES] + BAD_ROTATIONS)
def test_append_refuses(lib, kw):
    assert append(lib, **kw) == INVALID and lib.pam_last_error() != b""


def attention(lib, **kw):
    return call(lib, "pam_paged_attention",
                ["q", "k_cache", "v_cache", "q_starts", "kv_lens", "table", "out", "workspace"],
                [("q_heads", Heads, heads()), ("out_heads", Heads, heads()), ("k_cache_layout", Cache, cache()),
                 ("v_cache_layout", Cache, cache()), ("table_stride", I64, 1250), ("tokens", I64, 40), ("d", I32, 64),
                 ("batch", I32, 4), ("table_width", I32, 1250), ("causal", I32, 1), ("window", I32, 0),
                 ("scale", F32, 0.125), ("max_q", I32, 10), ("max_kv", I32, 20000), ("workspace_bytes", I64, 1 << 40)],
                **kw)


@pytest.mark.parametrize("kw", [
    dict(d=12), dict(d=0), dict(d=264), dict(tokens=-1), dict(batch=-1), dict(max_q=-1), dict(max_kv=-1),
    dict(max_kv=20001), dict(table_width=-1), dict(table_stride=1249), dict(kv_lens=None), dict(table=None),
    dict(q_starts=None, tokens=3), dict(scale=float("inf")), dict(scale=float("nan")), dict(window=-1), dict(q=None),
    dict(out=None), dict(k_cache=None), dict(v_cache=None), dict(q_heads=heads(count=12)), dict(q_heads=NONE),
    dict(out_heads=heads(kind=1)), dict(out_heads=heads(count=4)), dict(out_heads=heads(head=32)),
    dict(v_cache_layout=cache(kind=1)), dict(v_cache_layout=cache(pages=4)), dict(v_cache_layout=cache(size=8)),
    dict(v_cache_layout=cache(count=4)), dict(workspace=None), dict(workspace_bytes=0), dict(workspace_bytes=-1),
    dict(workspace=P + 8), dict(batch=1 << 30, max_q=1 << 20)]
    + [dict(q_heads=h) for h in BAD_HEADS] + [dict(k_cache_layout=c) for c in BAD_CACHES])
def test_attention_refuses(lib, kw):
    assert attention(lib, **kw) == INVALID and lib.pam_last_error() != b""


def test_attention_workspace_sizes(lib):
    need = ctypes.c_size_t()
    size = lib.pam_paged_attention_workspace_size
    assert size(64, 8, 8, 0, 1, 1, 10, None) == INVALID
    for bad in ((60, 8, 8, 0, 1, 1, 10), (64, 8, 3, 0, 1, 1, 10), (64, 8, 8, 2, 1, 1, 10), (64, 8, 0, 0, 1, 1, 10),
                (64, 8, 8, 0, -1, 1, 10), (64, 8, 8, 0, 1, -1, 10), (64, 8, 8, 0, 1, 1, -1)):
        assert size(*bad, ctypes.byref(need)) == INVALID
    for sizes in ((64, 8, 8, 0, 0, 1, 10), (64, 8, 8, 0, 1, 0, 10), (64, 8, 8, 1, 1, 1, 0), (64, 8, 8, 1, 1, 1, 10)):
        assert size(*sizes, ctypes.byref(need)) == 0 and need.value == 0
    assert size(128, 32, 8, 1, 1, 1, 1 << 20, ctypes.byref(need)) == 0 and need.value > 0


def test_python_refuses():
    torch = pytest.importorskip("torch")
    q = torch.zeros(2, 4, 64)
    with pytest.raises(pam.PamError):
        pam.norm_rope(q, None)                                   # no CPU path
    with pytest.raises(TypeError):
        pam.norm_rope(q.half(), None)
    with pytest.raises(TypeError):
        pam.norm_rope(q.numpy(), None)
    with pytest.raises(ValueError):
        pam.norm_rope(None, None)
    with pytest.raises(ValueError):
        pam.norm_rope_grad(None, None, q, None)
    with pytest.raises(pam.PamError):
        pam.paged_attention(q, q[None], q[None], None, None)
    with pytest.raises(pam.PamError):
        pam.append_kv(q, q, q[None], q[None], None)
