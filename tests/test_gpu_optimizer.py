"""The norm of all gradients and the AdamW step over many tensors against the
definitions, 8-bit states code for code."""
import numpy as np
import pytest

import paper_2305_17190_amd as pam
import training_util as tu
from attention_util import bf16, check
from gpu_util import device, note, to_dev
from oracle import training_ref as ref

pytestmark = pytest.mark.gpu

KW = dict(lr=3e-3, betas=(0.9, 0.99), eps=1e-7, weight_decay=0.05)
SIZES = [[1], [3, 257, 1], [256, 255, 4096, 4097, 5], [0, 70, 0, 1000, 0], [100003], [2 * 1024 * 1024 + 7, 513, 300000],
         list(range(1, 130))]


def blocks(n):
    return -(-n // ref.BLOCK)


def make(sizes, seed=0, grad_bf16=False, eight=False):
    """Numpy tensors of a step: lists of p, g, avg, sq (and scales)."""
    rng = np.random.default_rng([seed, len(sizes), sum(sizes)])
    out = dict(p=[], g=[], avg=[], sq=[], avg_scale=[], sq_scale=[])
    for n in sizes:
        out["p"].append(rng.standard_normal(n).astype(np.float32))
        g = (rng.standard_normal(n) * np.exp(rng.standard_normal(n))).astype(np.float32)
        out["g"].append(bf16(g) if grad_bf16 else g)
        if eight:
            out["avg"].append(rng.integers(0, 256, n).astype(np.uint8))
            out["sq"].append(rng.integers(100, 256, n).astype(np.uint8))
            out["avg_scale"].append((0.1 + rng.random(blocks(n))).astype(np.float32))
            out["sq_scale"].append((0.1 + rng.random(blocks(n))).astype(np.float32))
        else:
            out["avg"].append(rng.standard_normal(n).astype(np.float32))
            out["sq"].append((rng.standard_normal(n) ** 2).astype(np.float32))
    return out


def on_device(arrays, dtype=None, offset=0, fill=0):
    """Views of one allocation, `offset` elements between them."""
    import torch
    flat = [torch.from_numpy(a) if dtype is None else torch.from_numpy(a).to(dtype) for a in arrays]
    total = sum(t.numel() + offset for t in flat) + offset
    whole = torch.full((total,), fill, dtype=flat[0].dtype).to(device())
    at, views = offset, []
    for t in flat:
        views.append(whole[at:at + t.numel()])
        views[-1].copy_(t)
        at += t.numel() + offset
    return views, whole


def fresh(n, eight):
    return [np.zeros(n, np.uint8 if eight else np.float32) for _ in range(2)]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("grad_bf16", [False, True])
def test_grad_norm(sizes, grad_bf16):
    import torch
    note(f"grad_norm {len(sizes)} tensors, {sum(sizes)} values, bf16 {grad_bf16}")
    g = make(sizes, grad_bf16=grad_bf16)["g"]
    views, _ = on_device(g, torch.bfloat16 if grad_bf16 else None, offset=3)
    got = pam.grad_norm(views)
    assert got.dtype == torch.float32 and got.dim() == 0
    want = ref.grad_norm(g)
    assert abs(float(got) - want) <= tu.U * want * 1.01
    assert float(pam.grad_norm(views)) == float(got)


def test_grad_norm_of_special_values():
    import torch
    note("grad_norm specials")
    for values, want in (([3e30, 4e30], 5e30), ([3e-30, 4e-30], 5e-30), ([0.0], 0.0), ([np.inf, 1], np.inf)):
        got = float(pam.grad_norm([torch.tensor(values, dtype=torch.float32, device=device())]))
        assert got == want or abs(got - want) <= 2 * tu.U * want
    assert np.isnan(float(pam.grad_norm([torch.tensor([1.0, np.nan], device=device())])))
    assert float(pam.grad_norm([torch.empty(0, device=device())])) == 0.0


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("grad_bf16", [False, True])
def test_32_bit_states(sizes, grad_bf16):
    """Three steps, with and without a limit, copies among them; what lies between
    the tensors stays."""
    import torch
    note(f"adamw 32 bits, {len(sizes)} tensors, {sum(sizes)} values, bf16 {grad_bf16}")
    host = make(sizes, grad_bf16=grad_bf16)
    p, pw = on_device(host["p"], offset=1, fill=5)
    m, mw = on_device(host["avg"], offset=3, fill=5)
    v, vw = on_device(host["sq"], offset=2, fill=5)
    c, cw = on_device(host["p"], torch.bfloat16, offset=1, fill=5)
    for step, limited in ((1, False), (2, True), (100, True)):
        old = [[t.cpu().numpy().copy() for t in x] for x in (p, m, v)]
        gn = make(sizes, step, grad_bf16)["g"]
        g, _ = on_device(gn, torch.bfloat16 if grad_bf16 else None, offset=1)
        norm = pam.grad_norm(g) if limited else None
        most = 0.5 * float(norm) if limited else None
        pam.adamw_step(p, g, m, v, step, **KW, norm=norm, max_norm=most, copies=c if step > 1 else None)
        limit, err = tu.norm_limit(float(norm), most) if limited else (1.0, 0.0)
        for j in range(len(sizes)):
            args = old[0][j], gn[j], old[1][j], old[2][j]
            want = ref.adamw(*args, step, limit=float(limit), **KW)
            tol = tu.step_errors(*args, err, step, limit=float(limit), **KW)
            for t, w_, e, what in zip((p[j], m[j], v[j]), want, tol, ("p", "avg", "sq")):
                check(t.cpu().numpy(), w_, e, f"{what} of tensor {j}, step {step}")
        if step > 1:
            assert all(torch.equal(a.bfloat16(), b) for a, b in zip(p, c))
    for whole, gap in ((pw, 1), (mw, 3), (vw, 2), (cw, 1)):
        at = 0
        for n in sizes + [0]:
            assert bool((whole[at:at + gap] == 5).all())
            at += gap + n


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("grad_bf16", [False, True])
def test_8_bit_states(sizes, grad_bf16):
    """Codes and scales are the definition's, bit for bit."""
    import torch
    note(f"adamw 8 bits, {len(sizes)} tensors, {sum(sizes)} values, bf16 {grad_bf16}")
    host = make(sizes, grad_bf16=grad_bf16, eight=True)
    p, pw = on_device(host["p"], offset=1, fill=5)
    states = [on_device(host[k], offset=o, fill=5) for k, o in (("avg", 1), ("sq", 3), ("avg_scale", 1), ("sq_scale", 2))]
    m, v, ms, vs = (s[0] for s in states)
    c, cw = on_device(host["p"], torch.bfloat16, offset=1, fill=5)
    for step, limited, seed in ((1, False, 0), (2, True, 7), (1000, False, 2 ** 32 - 5)):
        old = [[t.cpu().numpy().copy() for t in x] for x in (p, m, v, ms, vs)]
        gn = make(sizes, step, grad_bf16)["g"]
        g, _ = on_device(gn, torch.bfloat16 if grad_bf16 else None, offset=1)
        norm = pam.grad_norm(g) if limited else None
        most = 0.5 * float(norm) if limited else None
        pam.adamw_step(p, g, m, v, step, **KW, avg_scales=ms, sq_scales=vs, norm=norm, max_norm=most, seed=seed,
                       copies=c if step > 1 else None)
        limit = tu.norm_limit(float(norm), most)[0] if limited else None
        for j in range(len(sizes)):
            want = ref.adamw8(old[0][j], gn[j], *(x[j] for x in old[1:]), step=step, seed=seed, tensor=j, limit=limit, **KW)
            for t, w_, what in zip((m[j], v[j], ms[j], vs[j]), want[1:5], ("avg", "sq", "avg_scale", "sq_scale")):
                got = t.cpu().numpy()
                assert np.array_equal(got, w_), (f"{what} of tensor {j}, step {step}: {int((got != w_).sum())} of "
                                                 f"{got.size} differ")
            tol = np.abs(want[5]) * 12 * tu.U + 3 * tu.U * np.maximum(np.abs(old[0][j]), np.abs(want[0])) + tu.TINY
            check(p[j].cpu().numpy(), want[0], tol, f"p of tensor {j}, step {step}")
        if step > 1:
            assert all(torch.equal(a.bfloat16(), b) for a, b in zip(p, c))
    for whole, gap, length in ((pw, 1, int), (states[0][1], 1, int), (states[1][1], 3, int), (states[2][1], 1, blocks),
                               (states[3][1], 2, blocks), (cw, 1, int)):
        at = 0
        for n in sizes + [0]:
            assert bool((whole[at:at + gap] == 5).all())
            at += gap + length(n)


@pytest.mark.parametrize("seed", range(12))
def test_random_lists(seed):
    """Lists of random lengths and sizes, four steps from fresh states: 8-bit codes bit for
    bit, 32-bit states within their tolerance of the definition carried along."""
    import random
    import torch
    rng = random.Random(500 + seed)
    eight, grad_bf16 = seed % 2 == 0, rng.random() < 0.5
    sizes = [int(round(30000 ** rng.random())) - (rng.random() < 0.1) for _ in range(rng.choice((1, 5, 60, 140)))]
    note(f"random adamw {seed}: {len(sizes)} tensors, {sum(sizes)} values, 8 bits {eight}, bf16 {grad_bf16}")
    p0 = [np.ascontiguousarray(t) for t in make(sizes, seed)["p"]]
    state = [[np.zeros(n, np.uint8 if eight else np.float32) for n in sizes] for _ in "mv"]
    scales = [[np.zeros(blocks(n), np.float32) for n in sizes] for _ in "mv"] if eight else [None, None]
    p = [to_dev(t) for t in p0]
    d = [None if x is None else [to_dev(t) for t in x] for x in (*state, *scales)]
    for step in range(1, 5):
        gn = make(sizes, 10 * seed + step, grad_bf16)["g"]
        g = [to_dev(t) for t in gn]
        g = [t.bfloat16() for t in g] if grad_bf16 else g
        old = [[t.cpu().numpy().copy() for t in x] for x in (p, d[0], d[1])]
        pam.adamw_step(p, g, d[0], d[1], step, **KW, avg_scales=d[2], sq_scales=d[3], seed=seed)
        for j in range(len(sizes)):
            if eight:
                want = ref.adamw8(old[0][j], gn[j], state[0][j], state[1][j], scales[0][j], scales[1][j], step=step, seed=seed,
                                  tensor=j, **KW)
                state[0][j], state[1][j], scales[0][j], scales[1][j] = want[1:5]
                for t, w_ in zip((d[0][j], d[1][j], d[2][j], d[3][j]), want[1:5]):
                    assert np.array_equal(t.cpu().numpy(), w_), (step, j)
            else:
                args = old[0][j], gn[j], old[1][j], old[2][j]
                for t, w_, e in zip((p[j], d[0][j], d[1][j]), ref.adamw(*args, step, **KW),
                                    tu.step_errors(*args, 0.0, step, **KW)):
                    check(t.cpu().numpy(), w_, e, f"tensor {j}, step {step}")


def test_special_gradients():
    """Zero gradients, whole blocks of them, infinities and NaN stay in their block."""
    import torch
    note("adamw 8 bits, special gradients")
    n = 5 * 256 + 100
    g = make([n])["g"][0]
    g[256:512] = 0
    g[600], g[800], g[1100] = np.inf, np.nan, 1e10
    g[1024:1030] = 0
    state = [*fresh(n, True), np.zeros(6, np.float32), np.zeros(6, np.float32)]
    p0 = np.ones(n, np.float32)
    p = to_dev(p0)
    d = [to_dev(x) for x in state]
    for step in (1, 2):
        pam.adamw_step([p], [to_dev(g)], [d[0]], [d[1]], step, **KW, avg_scales=[d[2]], sq_scales=[d[3]])
        want = ref.adamw8(p0, g, *state, step=step, seed=0, tensor=0, **KW)
        p0, state = want[0].astype(np.float32), list(want[1:5])
        for got, w_ in zip(d, state):
            got = got.cpu().numpy()
            if got.dtype == np.float32:
                assert np.array_equal(got, w_, equal_nan=True)
            else:   # of blocks with a NaN the scale says it all
                fine = np.repeat(np.isfinite(state[2]), 256)[:n]
                assert np.array_equal(got[fine], w_[fine])
    got = p.cpu().numpy()
    bad = ~np.isfinite(got)
    assert not bad[:512].any() and not bad[1024:].any() and bad[600] and bad[800]
    assert np.allclose(got[256:512], (1 - KW["lr"] * KW["weight_decay"]) ** 2, rtol=4 * tu.U, atol=0)
    # 32 bits: the same gradients touch nothing but their own values.
    p, m, v = (to_dev(x) for x in (np.ones(n, np.float32), *fresh(n, False)))
    pam.adamw_step([p], [to_dev(g)], [m], [v], 1, **KW)
    assert set(np.flatnonzero(~np.isfinite(p.cpu().numpy())).tolist()) <= {600, 800} and not np.isfinite(float(p[800]))
    # A norm that is not finite reaches everything, as its definition has it.
    norm = pam.grad_norm([to_dev(g)])
    assert np.isnan(float(norm))
    pam.adamw_step([p], [to_dev(g)], [m], [v], 2, **KW, norm=norm, max_norm=1.0)
    assert bool(torch.isnan(p).all())


@pytest.mark.parametrize("eight", [False, True])
def test_step_on_the_device_in_a_graph(eight):
    """A captured step counts on, with the norm's limit; replays equal eager steps
    with the integer, to the rounding of 1 - beta^t."""
    import torch
    note(f"adamw in a graph, 8 bits {eight}")
    sizes = [300, 5000, 77]
    host = make(sizes, eight=eight)

    def fresh_state():
        lists = {k: on_device(host[k])[0] for k in ("p", "g")}
        n = [np.zeros(s, np.uint8 if eight else np.float32) for s in sizes]
        lists.update(avg=on_device(n)[0], sq=on_device(n)[0])
        z = [np.zeros(blocks(s), np.float32) for s in sizes]
        lists.update(ms=on_device(z)[0] if eight else None, vs=on_device(z)[0] if eight else None)
        return lists

    def run(s, step):
        norm = pam.grad_norm(s["g"])
        pam.adamw_step(s["p"], s["g"], s["avg"], s["sq"], step, **KW, avg_scales=s["ms"], sq_scales=s["vs"], norm=norm,
                       max_norm=1.0, seed=3)

    eager, replayed = fresh_state(), fresh_state()
    count = torch.ones(1, dtype=torch.int64, device=device())
    run(eager, 1)
    run(replayed, count)
    count += 1
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(replayed, count)
        count += 1
    for step in range(2, 6):
        for s in (eager, replayed):
            for g in s["g"]:
                g.mul_(1.1)
        run(eager, step)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k in ("avg", "sq", "ms", "vs"):
            assert eager[k] is None or all(torch.equal(a, b) for a, b in zip(eager[k], replayed[k])), (step, k)
        for a, b in zip(eager["p"], replayed["p"]):
            assert float((a - b).abs().max()) <= 16 * tu.U * (float(a.abs().max()) + 1)
    del graph


def test_two_streams():
    import torch
    note("adamw on two streams")
    cases = [make([200000, 3], i) for i in range(2)]

    def run(c):
        p, m, v = ([to_dev(t) for t in c[k]] for k in ("p", "avg", "sq"))
        g = [to_dev(t) for t in c["g"]]
        pam.adamw_step(p, g, m, v, 3, **KW, norm=pam.grad_norm(g), max_norm=1.0)
        return p + m + v

    want = [run(c) for c in cases]
    torch.cuda.synchronize()
    got = []
    for c in cases:
        with torch.cuda.stream(torch.cuda.Stream()):
            got.append(run(c))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for x, y in zip(got, want) for a, b in zip(x, y))


def test_steps_count_as_changes_in_place():
    """autograd sees that a parameter changed under a graph that saved it."""
    import torch
    note("adamw, version counters")
    p = torch.ones(4, device=device(), requires_grad=True)
    loss = (p * p).sum()
    pam.adamw_step([p], [torch.ones(4, device=device())], [torch.zeros(4, device=device())],
                   [torch.zeros(4, device=device())], 1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def params(seed=0, shapes=((20, 30), (30,), (7, 300))):
    import torch
    g = torch.Generator().manual_seed(seed)
    return [torch.nn.Parameter(torch.randn(*s, generator=g).to(device())) for s in shapes]


@pytest.mark.parametrize("max_norm", [None, 0.7])
def test_optimizer_against_torch(max_norm):
    """Ten steps of optim.AdamW beside torch's, one parameter now and then without a
    gradient, another group with another rate."""
    import torch
    from paper_2305_17190_amd.optim import AdamW
    note("optim.AdamW against torch")
    mine, other = params(), params()
    groups = [[dict(params=x[:2]), dict(params=x[2:], lr=1e-2, weight_decay=0.0)] for x in (mine, other)]
    a, b = AdamW(groups[0], lr=1e-3, max_norm=max_norm), torch.optim.AdamW(groups[1], lr=1e-3)
    rng = torch.Generator().manual_seed(1)
    for step in range(10):
        for x, y in zip(mine, other):
            x.grad = torch.randn(x.shape, generator=rng).to(device())
            y.grad = x.grad.clone()
        if step % 3 == 1:
            mine[1].grad = other[1].grad = None
        if max_norm is not None:
            torch.nn.utils.clip_grad_norm_([p for p in other if p.grad is not None], max_norm)
        a.step()
        b.step()
    for x, y in zip(mine, other):
        assert torch.allclose(x, y, rtol=1e-5, atol=1e-6)


def test_optimizer_state_goes_on_after_loading():
    import torch
    from paper_2305_17190_amd.optim import AdamW
    note("optim.AdamW, saved and loaded")
    for bits in (8, 32):
        mine, other = params(), params()
        a = AdamW(mine, lr=1e-3, state_bits=bits, seed=4)

        def step(opt, ps, seed):
            g = torch.Generator().manual_seed(seed)
            for p in ps:
                p.grad = torch.randn(p.shape, generator=g).to(device())
            opt.step()

        for i in range(3):
            step(a, mine, i)
        b = AdamW(other, lr=1e-3, state_bits=bits, seed=4)
        b.load_state_dict(a.state_dict())
        with torch.no_grad():
            for x, y in zip(mine, other):
                y.copy_(x)
        for i in range(3, 5):
            step(a, mine, i)
            step(b, other, i)
        assert all(torch.equal(x, y) for x, y in zip(mine, other))
        assert b.state[other[0]]["avg"].dtype == (torch.uint8 if bits == 8 else torch.float32)
