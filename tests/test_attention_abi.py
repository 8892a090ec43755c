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


def heads(data=P, token=512, head=64, count=8, kind=0):
    return att._Heads(data, token, head, count, kind)


def cache(data=P, page=8192, slot=512, head=64, pages=10, size=16, count=8, kind=0):
    return att._Cache(data, page, slot, head, pages, size, count, kind)


def rotation(positions=P, cos=P, sin=P, rows=100, rot=64, interleaved=0):
    return att._Rotation(positions, cos, sin, rows, rot, interleaved)


def ref(x):
    return None if x is None else ctypes.byref(x)


def test_every_declared_symbol_is_exported(lib):
    with open(HEADER) as f:
        text = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    names = set(re.findall(r"\b(pam_[a-z_0-9]+)\s*\(", text))
    assert names == set(att.EXPORTS)
    for name in names:
        assert hasattr(lib, name)


def norm_rope(lib, **kw):
    a = dict(tokens=4, d=64, q_in=heads(), qw=P, q_out=heads(), k_in=heads(), kw=P, k_out=heads(), eps=1e-6,
             rot=rotation())
    a.update(kw)
    return lib.pam_norm_rope(a["tokens"], a["d"], ref(a["q_in"]), a["qw"], ref(a["q_out"]), ref(a["k_in"]), a["kw"],
                             ref(a["k_out"]), a["eps"], ref(a["rot"]), None)


BAD_HEADS = [heads(data=None), heads(count=0), heads(token=-1), heads(head=-5), heads(kind=2), heads(token=1 << 60)]
BAD_ROTATIONS = [rotation(positions=None), rotation(cos=None), rotation(sin=None), rotation(rot=63), rotation(rot=66),
                 rotation(rot=-2), rotation(rows=-1), rotation(rows=1 << 31)]


@pytest.mark.parametrize("kw", [
    dict(tokens=-1), dict(d=63), dict(d=0), dict(d=258), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
    dict(q_out=None), dict(k_in=None), dict(q_in=None, q_out=None, k_in=None, k_out=None),
    dict(k_in=heads(kind=1)), dict(q_out=heads(count=4)), dict(q_out=heads(token=32)), dict(k_out=heads(head=63)),
    dict(tokens=1 << 30)] + [dict(q_in=h) for h in BAD_HEADS] + [dict(k_out=h) for h in BAD_HEADS]
    + [dict(rot=r) for r in BAD_ROTATIONS])
def test_norm_rope_refuses(lib, kw):
    assert norm_rope(lib, **kw) == INVALID and lib.pam_last_error() != b""


def test_nothing_to_do_launches_nothing(lib):
    none = heads(data=None)
    assert norm_rope(lib, tokens=0, q_in=none, q_out=none, k_in=none, k_out=none, rot=rotation(None, None, None)) == 0
    assert append(lib, tokens=0, k=none, v=none, k_cache=cache(data=None), v_cache=cache(data=None), slots=None,
                  q_in=None, q_out=None, rot=None) == 0
    assert attention(lib, batch=0) == 0
    assert attention(lib, tokens=0, q=none, out=none) == 0
    assert grad(lib, tokens=0, qw=None, dqw=None, kw=None, dkw=None, workspace=None) == 0


def grad(lib, **kw):
    a = dict(tokens=4, d=64, q=heads(), qw=P, dq=heads(), gq=heads(), dqw=P, k=heads(), kw=P, dk=heads(), gk=heads(),
             dkw=P, eps=1e-6, rot=rotation(), workspace=P, bytes=1 << 30)
    a.update(kw)
    return lib.pam_norm_rope_grad(a["tokens"], a["d"], ref(a["q"]), a["qw"], ref(a["dq"]), ref(a["gq"]), a["dqw"],
                                  ref(a["k"]), a["kw"], ref(a["dk"]), ref(a["gk"]), a["dkw"], a["eps"], ref(a["rot"]),
                                  a["workspace"], a["bytes"], None)


@pytest.mark.parametrize("kw", [
    dict(tokens=-1), dict(d=65), dict(eps=-1.0), dict(dq=None), dict(gk=None), dict(q=None), dict(qw=None), dict(dkw=None),
    dict(q=None, dq=None, gq=None), dict(dq=heads(count=3)), dict(gq=heads(kind=1)), dict(dk=heads(kind=1)),
    dict(gq=heads(token=8)), dict(workspace=None), dict(bytes=8), dict(workspace=P + 4)]
    + [dict(dq=h) for h in BAD_HEADS] + [dict(rot=r) for r in BAD_ROTATIONS])
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
    a = dict(tokens=4, d=64, k=heads(), kw=P, v=heads(), q_in=heads(), qw=P, q_out=heads(), eps=1e-6, rot=rotation(),
             k_cache=cache(), v_cache=cache(), slots=P)
    a.update(kw)
    return lib.pam_append_kv(a["tokens"], a["d"], ref(a["k"]), a["kw"], ref(a["v"]), ref(a["q_in"]), a["qw"],
                             ref(a["q_out"]), a["eps"], ref(a["rot"]), ref(a["k_cache"]), ref(a["v_cache"]), a["slots"],
                             None)


BAD_CACHES = [cache(data=None), cache(page=-1), cache(slot=-1), cache(head=-1), cache(pages=-1), cache(size=0),
              cache(count=0), cache(kind=7), cache(pages=1 << 27), cache(page=1 << 60)]


@pytest.mark.parametrize("kw", [
    dict(tokens=-1), dict(d=7), dict(k=None), dict(v=None), dict(k_cache=None), dict(slots=None), dict(q_out=None),
    dict(v=heads(kind=1)), dict(q_in=heads(kind=1)), dict(k=heads(count=4)), dict(v=heads(count=4)),
    dict(v_cache=cache(pages=9)), dict(v_cache=cache(size=8)), dict(q_out=heads(count=2)), dict(q_out=heads(head=8))]
    + [dict(k=h) for h in BAD_HEADS] + [dict(v_cache=c) for c in BAD_CACHES] + [dict(rot=r) for r in BAD_ROTATIONS])
def test_append_refuses(lib, kw):
    assert append(lib, **kw) == INVALID and lib.pam_last_error() != b""


def attention(lib, q=None, k_cache=None, v_cache=None, out=None, d=64, workspace=P, bytes=1 << 40, **kw):
    s = dict(q_starts=P, kv_lens=P, table=P, table_stride=20, tokens=40, batch=4, table_width=20, max_q=10, max_kv=300,
             causal=1, window=0, scale=0.125)
    s.update(kw)
    seq = att._Sequences(*(s[name] for name, _ in att._Sequences._fields_))
    return lib.pam_paged_attention(d, ref(q or heads()), ref(k_cache or cache()), ref(v_cache or cache()), ref(seq),
                                   ref(out or heads()), workspace, bytes, None)


@pytest.mark.parametrize("kw", [
    dict(d=12), dict(d=0), dict(d=264), dict(tokens=-1), dict(batch=-1), dict(max_q=-1), dict(max_kv=-1),
    dict(max_kv=321), dict(table_width=-1), dict(table_stride=19), dict(kv_lens=None), dict(table=None),
    dict(q_starts=None, tokens=3), dict(scale=float("inf")), dict(scale=float("nan")), dict(q=heads(count=12)),
    dict(out=heads(kind=1)), dict(out=heads(count=4)), dict(out=heads(head=32)), dict(v_cache=cache(kind=1)),
    dict(v_cache=cache(pages=4)), dict(v_cache=cache(size=8)), dict(v_cache=cache(count=4)), dict(workspace=None),
    dict(bytes=0), dict(workspace=P + 8), dict(batch=1 << 30, max_q=1 << 20)]
    + [dict(q=h) for h in BAD_HEADS] + [dict(k_cache=c) for c in BAD_CACHES])
def test_attention_refuses(lib, kw):
    # Long enough that the call has a workspace.
    if "max_kv" not in kw and "table_width" not in kw and "table_stride" not in kw:
        kw = dict(max_kv=20000, table_width=1250, table_stride=1250, **kw)
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
