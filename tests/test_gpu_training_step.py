"""The layer-and-step operators together, as a training step uses them: a
feed-forward block forward and back, the gradients' norm and the step."""
import importlib.util
import os

import numpy as np
import pytest

import paper_2305_17190_amd as pam
import training_util as tu
from attention_util import check
from gpu_util import device, note, to_dev
from oracle import pam_ref
from oracle import training_ref as ref

pytestmark = pytest.mark.gpu

KW = dict(lr=2e-3, betas=(0.9, 0.98), eps=1e-8, weight_decay=0.01)


def block(width=48, hidden=160, tokens=130, seed=0):
    rng = np.random.default_rng(seed)
    p = [rng.standard_normal((hidden, width)) / width ** 0.5, 0.1 * rng.standard_normal(hidden),
         rng.standard_normal((width, hidden)) / hidden ** 0.5, 0.1 * rng.standard_normal(width)]
    x, target = (rng.standard_normal((tokens, width)) for _ in range(2))
    return [to_dev(t.astype(np.float32)) for t in p], *(to_dev(t.astype(np.float32)) for t in (x, target))


def gradients(p, x, target, act="gelu"):
    """Of the sum of squares of x + down(act(up(x))) - target, by the operators."""
    w1, b1, w2, b2 = p
    h, z = pam.linear(x, w1, b1, act, save_z=True)
    y = pam.linear(h, w2, b2, residual=x)
    dy, db2 = pam.activation_grad(y - target, None, None)
    dz, db1 = pam.activation_grad(pam.gemm(dy, w2), z, act)
    return y, [pam.gemm(dz, x, trans_a=True), db1, pam.gemm(dy, h, trans_a=True), db2]


def states(p, eight=False):
    import torch
    zeros = [[torch.zeros(t.shape, dtype=torch.uint8 if eight else torch.float32, device=device()) for t in p] for _ in "mv"]
    scales = [[torch.zeros(-(-t.numel() // 256), device=device()) for t in p] for _ in "mv"] if eight else [None, None]
    return *zeros, *scales


def step(p, x, target, s, count, most=1.0, copies=None):
    y, g = gradients(p, x, target)
    norm = pam.grad_norm(g)
    pam.adamw_step(p, g, s[0], s[1], count, **KW, avg_scales=s[2], sq_scales=s[3], norm=norm, max_norm=most, seed=9,
                   copies=copies)
    return y, norm


@pytest.mark.parametrize("eight", [False, True])
def test_autograd_and_optimizer_do_the_same(eight):
    """PAMLinear with activation and residual, and optim.AdamW, are the calls by hand."""
    import torch
    from paper_2305_17190_amd.autograd import PAMLinear
    from paper_2305_17190_amd.optim import AdamW
    note(f"training steps by hand and under autograd, 8 bits {eight}")
    p, x, target = block()
    up, down = PAMLinear(48, 160, device=device(), activation="gelu"), PAMLinear(160, 48, device=device())
    params = [up.weight, up.bias, down.weight, down.bias]
    with torch.no_grad():
        for a, b in zip(params, p):
            a.copy_(b)
    optimizer = AdamW(params, **KW, max_norm=1.0, state_bits=8 if eight else 32, seed=9)
    s = states(p, eight)
    for count in range(1, 6):
        y, norm = step(p, x, target, s, count)
        optimizer.zero_grad()
        out = down(up(x), residual=x)
        out.backward((out - target).detach())
        optimizer.step()
        assert torch.equal(out, y) and torch.equal(optimizer.last_norm, norm)
        for a, b in zip(params, p):
            # Sums and products in the same order: the down layer's bias gradient too.
            assert torch.equal(a, b), count


def test_against_float64():
    """One step's gradients and parameters against the definitions, each product on
    the GPU's own operands (their own error is pam_gemm's)."""
    note("a training step against float64")
    p, x, target = block(seed=1)
    host = [t.cpu().numpy() for t in p]
    w1, b1, w2, b2 = host
    xn = x.cpu().numpy()
    h, z = (t.cpu().numpy() for t in pam.linear(x, p[0], p[1], "gelu", save_z=True))
    y, g = gradients(p, x, target)
    g = [t.cpu().numpy() for t in g]

    def product(a, b, ta, tb, got, extra=0.0, k=None):
        want, size = pam_ref.pam_gemm_ref(a, b, ta, tb)
        check(got, want + extra, 1e-5 * np.sqrt(k) * size + 2 * tu.U * np.abs(want + extra) + tu.TINY, "product")

    product(xn, w1, False, True, z, b1.astype(np.float64), 48)
    check(h, ref.activation(z, "gelu"), tu.activation_error(z, "gelu"), "h")
    product(h, w2, False, True, y.cpu().numpy(), b2.astype(np.float64) + xn, 160)
    dy = (y - target).cpu().numpy()
    dh = pam.gemm(y - target, p[2]).cpu().numpy()
    product(dy, w2, False, False, dh, 0.0, 48)
    dz, db = ref.activation_grad(dh, z, "gelu")
    check(g[1], db, (np.abs(dh) * tu.slope_error(z, "gelu")).sum(0) + 132 * tu.U * np.abs(dz).sum(0), "db1")
    check(g[3], dy.astype(np.float64).sum(0), 132 * tu.U * np.abs(dy).sum(0), "db2")
    product(dy, h, True, False, g[2], 0.0, 130)
    s = states(p)
    _, norm = step(p, x, target, s, 1)
    assert abs(float(norm) - ref.grad_norm(g)) <= 1.01 * tu.U * ref.grad_norm(g)
    limit, err = tu.norm_limit(float(norm), 1.0)
    zero = [np.zeros_like(t) for t in host]
    for j in range(4):
        want = ref.adamw(host[j], g[j], zero[j], zero[j], 1, limit=float(limit), **KW)[0]
        tol = tu.step_errors(host[j], g[j], zero[j], zero[j], err, 1, limit=float(limit), **KW)[0]
        check(p[j].cpu().numpy(), want, tol, f"parameter {j}")


@pytest.mark.parametrize("eight", [False, True])
def test_steps_in_a_graph(eight):
    """A whole step captured: replays on new inputs, eager work between, equal eager
    steps to the rounding of 1 - beta^t (which reaches everything after the first)."""
    import torch
    note(f"training steps in a graph, 8 bits {eight}")
    p, x, target = block(seed=2)
    q = [t.clone() for t in p]
    s, r = states(p, eight), states(p, eight)
    copies = [torch.zeros(t.shape, dtype=torch.bfloat16, device=device()) for t in q]
    count = torch.ones(1, dtype=torch.int64, device=device())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, norm = step(q, x, target, r, count, copies=copies)
        count += 1
    for i in range(1, 5):
        x.mul_(0.9)
        _, want = step(p, x, target, s, i)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        if i == 1:
            assert torch.equal(want, norm)
        assert abs(float(want) - float(norm)) <= 1e-4 * float(want)
        for a, b, c in zip(p, q, copies):
            # A code on the other side of its border moves a parameter by a part of a step.
            far = (a - b).abs()
            assert float(far.mean()) <= 1e-5 and float(far.max()) <= 2 * KW["lr"], i
            assert torch.equal(b.bfloat16(), c)
    assert int(count) == 5
    del graph


def test_backward_pass_in_a_graph():
    """Forward and backward of the layers under autograd, captured with the step: the
    gradients asked for, no eager graph of the same leaves alive; replays equal eager
    passes bit for bit."""
    import torch
    from paper_2305_17190_amd.autograd import pam_linear
    note("layers' backward pass in a graph")
    p, x, target = block(seed=3)

    def passed(leaves):
        h = pam_linear(x, leaves[0], leaves[1], activation="silu")
        y = pam_linear(h, leaves[2], leaves[3], residual=x)
        return y.detach(), torch.autograd.grad(y, leaves, (y - target).detach())

    leaves = [t.clone().requires_grad_() for t in p]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            passed(leaves)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, g = passed(leaves)
    for rep in range(4):
        x.mul_(0.9)
        target.add_(0.1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        again = [t.detach().clone().requires_grad_() for t in leaves]
        want, gw = passed(again)
        torch.cuda.synchronize()
        assert torch.equal(y, want) and all(torch.equal(a, b) for a, b in zip(g, gw)), rep
        with torch.no_grad():
            for t in leaves:
                t.mul_(0.99)
    del graph


@pytest.mark.parametrize("bits", [8, 32])
def test_example_runs_with_either_state(bits):
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decoder.py")
    spec = importlib.util.spec_from_file_location("pam_decoder_example", path)
    decoder = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(decoder)
    note(f"decoder example, states in {bits} bits")
    losses, apart = decoder.main(["--steps", "5", "--new", "2", "--state-bits", str(bits)])
    assert len(losses) == 5 and all(np.isfinite(losses)) and apart < 1e-4
