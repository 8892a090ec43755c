"""Norm and rotation of heads, their gradient and the append to a paged cache
on the GPU against the float64 definitions."""
import numpy as np
import pytest

import attention_util as au
from gpu_util import device, note, to_dev
from oracle import attention_ref as ref

pytestmark = pytest.mark.gpu
EPS = 1e-5


def tensor(x, bf16, padded=False):
    """x (tokens, heads, d) on the device, as a view of a wider tensor at an odd offset if padded."""
    import torch
    t = to_dev(x)
    t = t.bfloat16() if bf16 else t
    if padded:
        wide = torch.full((t.shape[0], t.shape[1] + 2, t.shape[2] + 3), float("nan"), dtype=t.dtype, device=t.device)
        wide[:, 1:-1, 1:-2] = t
        t = wide[:, 1:-1, 1:-2]
    return t


def values(rng, tokens, heads, d, bf16):
    x = (rng.standard_normal((tokens, heads, d)) * 3).astype(np.float32)
    if tokens > 2:
        x[1] = 0                                   # a row of zeros
        x[2] *= 1e-12                              # one far below eps
    return au.bf16(x) if bf16 else x


class Inputs:
    def __init__(self, tokens, hq, hk, d, rot, bf16, seed=0, rows=50):
        rng = np.random.default_rng(seed + tokens + d)
        self.rng = rng
        self.q, self.k, self.v, self.dq, self.dk = (values(rng, tokens, h, d, bf16) for h in (hq, hk, hk, hq, hk))
        self.wq, self.wk = ((1 + 0.3 * rng.standard_normal(d)).astype(np.float32) for _ in range(2))
        self.pos = rng.integers(0, rows, tokens).astype(np.int32)
        self.cos, self.sin = au.tables(rows, rot) if rot else (None, None)

    def kw(self, interleaved, weights=True):
        kw = dict(eps=EPS, interleaved=interleaved)
        if self.cos is not None:
            kw.update(positions=to_dev(self.pos), cos=to_dev(self.cos), sin=to_dev(self.sin))
        if weights:
            kw.update(q_weight=to_dev(self.wq), k_weight=to_dev(self.wk))
        return kw


SIZES = [
    # tokens, query heads, key heads, d, rot
    (1, 1, 1, 2, 2), (3, 2, 1, 64, 64), (5, 8, 8, 64, 32), (33, 4, 2, 128, 128), (7, 3, 3, 80, 80), (9, 5, 1, 96, 24),
    (4, 2, 2, 256, 256), (6, 1, 3, 250, 6), (6, 2, 1, 130, 128), (257, 3, 2, 72, 36), (10, 2, 2, 32, 0), (2, 32, 8, 192, 64),
    (5, 1, 2, 10, 4), (1031, 2, 1, 16, 16),
]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("tokens,hq,hk,d,rot", SIZES)
def test_norm_rope(tokens, hq, hk, d, rot, bf16, interleaved):
    import torch
    import paper_2305_17190_amd as pam
    note(f"norm_rope {tokens} {hq} {hk} {d} {rot} {bf16} {interleaved}")
    s = Inputs(tokens, hq, hk, d, rot, bf16)
    for weights in (True, False):
        for out_dtype in (None, torch.float32, torch.bfloat16):
            got = pam.norm_rope(tensor(s.q, bf16, True), tensor(s.k, bf16), out_dtype=out_dtype,
                                **s.kw(interleaved, weights))
            for name, g, x, w in (("q", got[0], s.q, s.wq), ("k", got[1], s.k, s.wk)):
                want, size = ref.norm_rope(x, w if weights else None, s.pos, s.cos, s.sin, EPS, interleaved)
                to_bf16 = g.dtype == torch.bfloat16
                assert to_bf16 == (bf16 if out_dtype is None else out_dtype == torch.bfloat16)
                au.check(g.float().cpu().numpy(), want, au.norm_rope_tolerance(size, d, to_bf16), name)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("tokens,hq,hk,d,rot", SIZES)
def test_norm_rope_grad(tokens, hq, hk, d, rot, bf16, interleaved):
    import paper_2305_17190_amd as pam
    note(f"norm_rope_grad {tokens} {hq} {hk} {d} {rot} {bf16} {interleaved}")
    s = Inputs(tokens, hq, hk, d, rot, bf16, seed=1)
    for weights in (True, False):
        got = pam.norm_rope_grad(tensor(s.dq, bf16), tensor(s.dk, bf16, True), tensor(s.q, bf16, True), tensor(s.k, bf16),
                                 **s.kw(interleaved, weights))
        for i, (dz, x, w) in enumerate(((s.dq, s.q, s.wq), (s.dk, s.k, s.wk))):
            dx, dx_size, dw, dw_size = ref.norm_rope_grad(dz, x, w if weights else None, s.pos, s.cos, s.sin, EPS,
                                                          interleaved)
            tol = 2 * (d + 12) * au.U * dx_size + (2.0 ** -8 * np.abs(dx) if bf16 else 0) + 2.0 ** -126
            au.check(got[i].float().cpu().numpy(), dx, tol, "dx")
            if weights:
                n = tokens * x.shape[1]
                au.check(got[2 + i].cpu().numpy(), dw, (n + d / 2 + 12) * au.U * dw_size + 2.0 ** -126 * n, "dweight")
            else:
                assert got[2 + i] is None


def test_gradient_against_differences():
    """The GPU's gradient against central differences of the GPU's forward in
    float32: h = 1/16 on values of order 1 leaves h^2/6 of a third derivative of
    order 10 (0.007) and 2^-24 * 30 / h."""
    import torch
    import paper_2305_17190_amd as pam
    note("differences")
    s = Inputs(2, 1, 1, 8, 8, False, seed=2)
    s.q = (s.q / 3 + 1).astype(np.float32)
    s.q[1] = np.linspace(0.5, 2, 8)
    dz = s.rng.standard_normal(s.q.shape).astype(np.float32)
    kw = s.kw(False)
    gq, _, gw, _ = pam.norm_rope_grad(to_dev(dz), None, to_dev(s.q), None, **kw)
    h = 1 / 16

    def loss(q, w):
        out, _ = pam.norm_rope(to_dev(q), None, **dict(kw, q_weight=to_dev(w)))
        return float((out.cpu().double() * torch.from_numpy(dz).double()).sum())

    for value, grad in ((s.q, gq), (s.wq, gw)):
        for i in np.ndindex(value.shape):
            up, down = value.copy(), value.copy()
            up[i] += h
            down[i] -= h
            args = [(up, s.wq), (down, s.wq)] if value is s.q else [(s.q, up), (s.q, down)]
            diff = (loss(*args[0]) - loss(*args[1])) / (2 * h)
            assert abs(diff - float(grad.cpu().numpy()[i])) < 0.02, (i, diff, float(grad.cpu().numpy()[i]))


@pytest.mark.parametrize("bf16_cache", [False, True])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("tokens,hq,hk,d,rot", SIZES)
def test_append(tokens, hq, hk, d, rot, bf16, bf16_cache):
    import torch
    import paper_2305_17190_amd as pam
    page = [1, 7, 16][tokens % 3]
    note(f"append {tokens} {hq} {hk} {d} {rot} {bf16} {bf16_cache} page {page}")
    s = Inputs(tokens, hq, hk, d, rot, bf16, seed=3)
    pages = -(-tokens // page) + 2
    slots = s.rng.permutation(pages * page)[:tokens].astype(np.int64)
    drop = s.rng.random(tokens) < 0.2
    slots[drop] = s.rng.choice([-1, pages * page, -2 ** 40, 2 ** 40, 2 ** 32], drop.sum())
    dtype = torch.bfloat16 if bf16_cache else torch.float32
    for layout in ("page", "head"):
        caches = [torch.full((pages, page, hk, d), 7.0, dtype=dtype, device=device()) for _ in "kv"]
        if layout == "head":
            caches = [c.transpose(1, 2).contiguous().transpose(1, 2) for c in caches]
        q = pam.append_kv(tensor(s.k, bf16), tensor(s.v, bf16, True), *caches, to_dev(slots), q=tensor(s.q, bf16),
                          **s.kw(layout == "head"))
        want, size = ref.norm_rope(s.q, s.wq, s.pos, s.cos, s.sin, EPS, layout == "head")
        au.check(q.float().cpu().numpy(), want, au.norm_rope_tolerance(size, d, bf16), "q")
        want, size = ref.norm_rope(s.k, s.wk, s.pos, s.cos, s.sin, EPS, layout == "head")
        tol = au.norm_rope_tolerance(size, d, bf16_cache)
        k, v = (c.float().cpu().numpy().reshape(pages * page, hk, d) for c in caches)
        stored = au.bf16(s.v) if bf16_cache else s.v
        untouched = np.ones(pages * page, bool)
        for t in np.flatnonzero(~drop):
            au.check(k[slots[t]], want[t], tol[t], f"key {t}")
            assert np.array_equal(v[slots[t]], stored[t])
            untouched[slots[t]] = False
        assert np.all(k[untouched] == 7.0) and np.all(v[untouched] == 7.0)


def test_append_as_it_is():
    """Without weight, rotation or queries: a copy, rounded to the cache's type."""
    import torch
    import paper_2305_17190_amd as pam
    note("plain append")
    rng = np.random.default_rng(4)
    k, v = (rng.standard_normal((5, 2, 64)).astype(np.float32) for _ in range(2))
    k[0, 0, :4] = [np.nan, np.inf, -np.inf, 3.4e38]
    caches = [torch.zeros(2, 16, 2, 64, dtype=torch.bfloat16, device=device()) for _ in "kv"]
    slots = np.array([3, 17, 31, 0, 16], np.int64)
    assert pam.append_kv(to_dev(k), to_dev(v), *caches, to_dev(slots)) is None
    for c, x in zip(caches, (k, v)):
        got = c.view(32, 2, 64)[to_dev(slots)]
        want = to_dev(x).bfloat16()
        assert torch.equal(torch.nan_to_num(got.float(), 5.0), torch.nan_to_num(want.float(), 5.0))


def test_positions_without_a_table_row_give_nan():
    import paper_2305_17190_amd as pam
    note("positions")
    s = Inputs(5, 2, 1, 64, 32, False)
    s.pos[:] = [0, -1, 50, 49, 2 ** 31 - 1]
    q, k = pam.norm_rope(to_dev(s.q), to_dev(s.k), **s.kw(False))
    for got in (q.cpu().numpy(), k.cpu().numpy()):
        assert np.isnan(got[[1, 2, 4], :, :32]).all() and np.isfinite(got[[0, 3]]).all()
        assert np.isfinite(got[..., 32:]).all()


def test_special_values():
    """inf, NaN and squares past the range spread over their own head alone."""
    import paper_2305_17190_amd as pam
    note("special values")
    s = Inputs(6, 2, 2, 64, 64, False)
    s.q[0, 0, 5], s.q[1, 1, 0], s.q[3, 0, 9] = np.nan, np.inf, 3e38
    q, k = (t.cpu().numpy() for t in pam.norm_rope(to_dev(s.q), to_dev(s.k), **s.kw(False)))
    bad = np.zeros((6, 2), bool)
    bad[0, 0] = bad[1, 1] = True
    assert np.array_equal(np.isnan(q).any(-1), bad)
    assert np.all(np.isnan(q[0, 0])) and np.isfinite(k).all()
    want, size = ref.norm_rope(s.q, s.wq, s.pos, s.cos, s.sin, EPS, False)
    fine = ~bad
    fine[3, 0] = False                              # its mean square is inf in float32: zeros
    au.check(q[fine], want[fine], au.norm_rope_tolerance(size, 64, False)[fine], "q")
    assert np.all(q[3, 0] == 0)


def test_one_side_only_and_no_tokens():
    import torch
    import paper_2305_17190_amd as pam
    note("one side")
    s = Inputs(4, 2, 1, 64, 64, False)
    kw = s.kw(False)
    both = pam.norm_rope(to_dev(s.q), to_dev(s.k), **kw)
    q, none = pam.norm_rope(to_dev(s.q), None, **kw)
    assert none is None and torch.equal(q, both[0])
    none, k = pam.norm_rope(None, to_dev(s.k), **kw)
    assert none is None and torch.equal(k, both[1])
    g = pam.norm_rope_grad(None, to_dev(s.dk), None, to_dev(s.k), **kw)
    assert g[0] is None and g[2] is None and g[1].shape == s.k.shape and g[3].shape == (64,)
    e = Inputs(0, 2, 1, 64, 64, False)
    q, k = pam.norm_rope(to_dev(e.q), to_dev(e.k), **e.kw(False))
    assert q.shape == (0, 2, 64) and k.shape == (0, 1, 64)
    g = pam.norm_rope_grad(to_dev(e.dq), to_dev(e.dk), to_dev(e.q), to_dev(e.k), **e.kw(False))
    assert bool((g[2] == 0).all()) and bool((g[3] == 0).all())
    caches = [torch.zeros(2, 4, 1, 64, device=device()) for _ in "kv"]
    assert pam.append_kv(to_dev(e.k), to_dev(e.v), *caches, to_dev(np.zeros(0, np.int64))) is None


def test_strides_of_a_projection_and_broadcast_gradients():
    """Views of one fused projection, heads outermost, and gradients that are
    an expanded tensor (stride 0)."""
    import torch
    import paper_2305_17190_amd as pam
    note("strides")
    s = Inputs(9, 4, 2, 64, 64, False, seed=5)
    kw = s.kw(False)
    fused = torch.cat((to_dev(s.q), to_dev(s.k), to_dev(s.v)), 1).reshape(9, -1)
    views = [t.view(9, -1, 64) for t in fused.split([256, 128, 128], 1)]
    want = pam.norm_rope(to_dev(s.q), to_dev(s.k), **kw)
    for a, b in zip(pam.norm_rope(views[0], views[1], **kw), want):
        assert torch.equal(a, b)
    outer = [to_dev(x).transpose(0, 1).contiguous().transpose(0, 1) for x in (s.q, s.k)]
    for a, b in zip(pam.norm_rope(*outer, **kw), want):
        assert torch.equal(a, b)
    one = to_dev(s.dq[:1, :1])
    wide = one.expand(9, 4, 64)
    a = pam.norm_rope_grad(wide, None, to_dev(s.q), None, **kw)
    b = pam.norm_rope_grad(wide.contiguous(), None, to_dev(s.q), None, **kw)
    assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2])


def test_same_bits_on_another_stream_and_in_a_graph():
    import torch
    import paper_2305_17190_amd as pam
    note("streams and graphs")
    s = Inputs(3000, 4, 2, 64, 64, True, seed=6)
    kw = s.kw(False)
    args = [tensor(x, True) for x in (s.dq, s.dk, s.q, s.k)]
    first = pam.norm_rope_grad(*args, **kw)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        other = pam.norm_rope_grad(*args, **kw)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, other))
    graph = torch.cuda.CUDAGraph()
    caches = [torch.zeros(200, 16, 2, 64, dtype=torch.bfloat16, device=device()) for _ in "kv"]
    slots = to_dev(s.rng.permutation(3200)[:3000].astype(np.int64))
    with torch.cuda.graph(graph):
        grads = pam.norm_rope_grad(*args, **kw)
        q = pam.append_kv(args[3], args[1], *caches, slots, q=args[2], **kw)
    for i in range(3):
        args[2].copy_(args[2].flip(0))
        args[0].mul_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(grads, pam.norm_rope_grad(*args, **kw))), i
        keep = [c.clone() for c in caches]
        assert torch.equal(q, pam.append_kv(args[3], args[1], *caches, slots, q=args[2], **kw)), i
        assert all(torch.equal(a, b) for a, b in zip(keep, caches)), i
