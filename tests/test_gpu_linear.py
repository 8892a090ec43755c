"""Linear layers with bias, activation and residual: the product is gemm's, sum
for sum where no sum is long, and what is added follows the definition."""
import ctypes
import struct

import numpy as np
import pytest

import paper_2305_17190_amd as pam
import training_util as tu
from attention_util import check
from gpu_util import device, note, to_dev
from oracle import pam_ref
from oracle import training_ref as ref

pytestmark = pytest.mark.gpu

# Few rows of x (4, 8 and 16 at a time, K in parts), few columns, small products,
# every tile, split K, whole and split tiles in one launch; odd sizes; no K.
SIZES = [(1, 1, 1), (1, 512, 2048), (3, 65, 130), (8, 4096, 512), (13, 100, 77), (32, 768, 192), (500, 64, 3),
         (2048, 100, 8), (64, 96, 72), (33, 17, 45), (197, 197, 197), (256, 1024, 256), (1024, 256, 512), (1000, 250, 770),
         (2048, 512, 2048), (1773, 197, 770), (4096, 64, 4096), (128, 8192, 512), (192, 12608, 192), (1, 0, 5), (70, 0, 3)]


def inputs(m, k, n, bf16=False, seed=0, out_bf16=False):
    import torch
    rng = np.random.default_rng([m, k, n, seed])
    x = to_dev(rng.standard_normal((m, k)).astype(np.float32))
    w = to_dev((rng.standard_normal((n, k)) / max(k, 1) ** 0.5).astype(np.float32))
    bias = to_dev(rng.standard_normal(n).astype(np.float32))
    res = to_dev(rng.standard_normal((m, n)).astype(np.float32))
    if bf16:
        x, w = x.bfloat16(), w.bfloat16()
    return x, w, bias, res.bfloat16() if out_bf16 else res


def same(a, b):
    import torch
    kind = torch.int32 if a.dtype == torch.float32 else torch.int16
    return a.dtype == b.dtype and torch.equal(a.view(kind), b.view(kind))


def expect(y, z, name, residual, bf16, what):
    """y from the float32 z."""
    z64 = z.cpu().numpy().astype(np.float64)
    want = ref.activation(z64, name)
    tol = tu.activation_error(z64, name)
    if residual is not None:
        want = want + residual.float().cpu().numpy()
        tol = tol + tu.U * np.abs(want)
    tol = tol * (1 + 2.0 ** -8) + (2.0 ** -8 * np.abs(want) if bf16 else 0)
    check(y.float().cpu().numpy(), want, tol, what)


@pytest.mark.parametrize("m,k,n", SIZES)
@pytest.mark.parametrize("bf16", [False, True])
def test_every_kernel(m, k, n, bf16):
    """All activations, both output types; z is gemm's product plus the bias, bit for
    bit, rounded once."""
    import torch
    for i, name in enumerate(ref.ACTIVATIONS):
        for out_bf16 in (False, True):
            x, w, bias, res = inputs(m, k, n, bf16, i, out_bf16)
            bias = None if (i + out_bf16) % 3 == 2 else bias
            res = None if (i + out_bf16) % 2 else res
            out = torch.bfloat16 if out_bf16 else torch.float32
            note(f"linear {m}x{k}x{n} {name} bias {bias is not None} residual {res is not None} {x.dtype} -> {out}")
            y, z = pam.linear(x, w, bias, name, res, save_z=True, out_dtype=out)
            alone = pam.linear(x, w, bias, name, res, out_dtype=out)
            z32 = pam.gemm(x, w, trans_b=True)
            z32 = z32 if bias is None else z32 + bias
            assert y.dtype == z.dtype == out and y.shape == z.shape == (m, n)
            assert same(z, z32.to(out)) and same(alone, y)
            expect(y, z32, name, res, out_bf16, "y")


@pytest.mark.parametrize("m,k,n", [(5, 33, 70), (130, 250, 200), (300, 2000, 140)])
def test_against_the_definition(m, k, n):
    note(f"linear {m}x{k}x{n} against float64")
    x, w, bias, res = inputs(m, k, n)
    y, z = pam.linear(x, w, bias, "gelu", res, save_z=True)
    want, zr, size = ref.linear(*(t.cpu().numpy() for t in (x, w, bias)), "gelu", res.cpu().numpy())
    dz = 1e-5 * np.sqrt(k) * size + k * 2.0 ** -126 + tu.U * np.abs(zr)
    check(z.cpu().numpy(), zr, dz, "z")
    # gelu's slope stays below 1.13.
    check(y.cpu().numpy(), want, 1.13 * dz + tu.activation_error(zr, "gelu") + tu.U * np.abs(want), "y")


# Whole tiles of every shape and slices whose K is taken in parts, K inside a part,
# at its end and one past it.
@pytest.mark.parametrize("m,k,n", [(1100, 3000, 1300), (4096, 1025, 1024), (2048, 2048, 2048), (2048, 8192, 2048),
                                   (5000, 4097, 260), (700, 8191, 3000), (520, 40000, 140)])
@pytest.mark.parametrize("bf16", [False, True])
def test_long_sums(m, k, n, bf16):
    import torch
    plan, need = pam.plan(m, n, k), [ctypes.c_size_t() for _ in "ab"]
    lib = pam.training._library()
    assert lib.pam_linear_workspace_size(m, n, k, ctypes.byref(need[0])) == 0
    assert lib.pam_gemm_workspace_size(m, n, k, 1, ctypes.byref(need[1])) == 0
    folds = need[0].value > need[1].value + 255
    note(f"linear {m}x{k}x{n} bf16 {bf16}, plan {plan}, in parts {folds}")
    x, w, bias, res = inputs(m, k, n, bf16)
    y, z = pam.linear(x, w, bias, "relu", res, save_z=True)
    rows, cols = (np.unique(np.linspace(0, s - 1, 40).astype(int)) for s in (m, n))
    want, size = pam_ref.pam_gemm_ref(x[rows].float().cpu().numpy(), w[cols].float().cpu().numpy(), False, True)
    z0 = z[rows][:, cols].cpu().numpy()
    whole = want + bias[cols].cpu().numpy().astype(np.float64)
    part = 1024 if folds else k
    check(z0, whole, (part + k / 1024 + 80) * tu.U * size + tu.U * np.abs(whole), "z")
    assert bool((y == torch.relu(z) + res).all())
    if folds:     # shorter chains, smaller errors
        alone = pam.gemm(x, w, trans_b=True)[rows][:, cols].cpu().numpy()
        off = [np.linalg.norm(t.astype(np.float64) - want) for t in (alone, pam.linear(x, w)[rows][:, cols].cpu().numpy())]
        assert off[1] < off[0] or not k > 4000
    again = pam.linear(x, w, bias, "relu", res)
    assert same(again, y)


def test_long_sums_of_many_tiles():
    """More work items than their running sums' memory holds: several launches."""
    import torch
    m, k, n = 16640, 1040, 8192
    assert -(-m // 128) * (n // 128) * 65536 > 512 << 20
    note(f"linear {m}x{k}x{n}, running sums in rounds")
    x, w, bias, _ = inputs(m, k, n, True)
    y = pam.linear(x, w, bias, out_dtype=torch.bfloat16)
    rows, cols = (np.unique(np.linspace(0, s - 1, 50).astype(int)) for s in (m, n))
    want, size = pam_ref.pam_gemm_ref(x[rows].float().cpu().numpy(), w[cols].float().cpu().numpy(), False, True)
    want = want + bias[cols].cpu().numpy().astype(np.float64)
    check(y[rows][:, cols].float().cpu().numpy(), want, 1100 * tu.U * size + 2.0 ** -8 * np.abs(want), "y")
    whole = pam.gemm(x, w, trans_b=True) + bias
    off = (y.float() - whole).abs() - 2.0 ** -8 * whole.abs()
    assert float(off.max()) <= 1e-4          # every output, against the other order of sums


def test_few_rows_at_the_top_of_the_range():
    """Magnitudes about 2^63 and 2^64, whose products reach the largest float32: the
    forms without a range check may not take them."""
    import torch
    note("linear, few rows, magnitudes about 2^64")
    rng = np.random.default_rng(8)
    for bf16 in (False, True):
        for m, n in ((5, 40), (40, 5)):
            x, w = ((2.0 ** rng.integers(61, 66, (r, 64)) * (1 + rng.random((r, 64))) *
                     rng.choice([-1, 1], (r, 64))).astype(np.float32) for r in (m, n))
            x[:, 1:], w[:, 2:] = x[:, 1:] * np.float32(2.0 ** -70), w[:, 2:] * np.float32(2.0 ** -70)
            xd, wd = to_dev(x), to_dev(w)
            if bf16:
                xd, wd = xd.bfloat16(), wd.bfloat16()
                x, w = xd.float().cpu().numpy(), wd.float().cpu().numpy()
            # One term at the top, the others far below: float32 sums are the terms'.
            want, size = pam_ref.pam_gemm_ref(x, w, False, True)
            got = pam.linear(xd, wd).cpu().numpy()
            assert np.isfinite(got).all() and np.abs(want).max() > 1e38
            check(got, want, 70 * tu.U * size, "product")


def test_narrow_mantissas():
    import torch
    note("linear, 7 mantissa bits")
    x, w, bias, _ = inputs(200, 100, 150)
    y, z = pam.linear(x, w, bias, "relu", save_z=True, mantissa_bits=7)
    want = pam.gemm(x, w, trans_b=True, mantissa_bits=7) + bias
    assert same(z, want) and same(y, torch.relu(want))


@pytest.mark.parametrize("m,k,n", [(1, 64, 40), (70, 64, 33), (300, 128, 500)])
def test_views(m, k, n):
    """Rows of wider matrices, at odd offsets."""
    import torch
    note(f"linear of views {m}x{k}x{n}")
    x, w, bias, res = inputs(m, k, n)
    wide = [torch.full((t.shape[0], t.shape[1] + 7), float("nan"), device=device()) for t in (x, w, res)]
    views = []
    for t, big in zip((x, w, res), wide):
        big[:, 3:3 + t.shape[1]] = t
        views.append(big[:, 3:3 + t.shape[1]])
    long_bias = torch.cat((torch.full((1,), float("nan"), device=device()), bias))
    got = pam.linear(views[0], views[1], long_bias[1:], "silu", views[2], save_z=True)
    for a, b in zip(got, pam.linear(x, w, bias, "silu", res, save_z=True)):
        assert same(a, b)


@pytest.mark.parametrize("m,k,n", [(4, 64, 40), (40, 64, 9), (100, 70, 131), (300, 512, 130), (128, 8192, 130)])
@pytest.mark.parametrize("out_bf16", [False, True])
def test_c_call_in_place_with_wide_rows(m, k, n, out_bf16):
    """y on its residual, leading dimensions past n: the columns between stay."""
    import torch
    note(f"pam_linear {m}x{k}x{n} in place, bf16 {out_bf16}")
    x, w, bias, res = inputs(m, k, n, out_bf16=out_bf16)
    want, zw = pam.linear(x, w, bias, "gelu_tanh", res, save_z=True, out_dtype=res.dtype)
    y = torch.full((m, n + 5), 7.0, device=device(), dtype=res.dtype)
    z = torch.full((m, n + 3), 9.0, device=device(), dtype=res.dtype)
    y[:, :n] = res
    lib = pam.training._library()
    need = ctypes.c_size_t()
    assert lib.pam_linear_workspace_size(m, n, k, ctypes.byref(need)) == 0
    ws = torch.empty(max(need.value, 1), dtype=torch.uint8, device=device())
    args = struct.pack("=7q9q4i", x.data_ptr(), w.data_ptr(), bias.data_ptr(), y.data_ptr(), y.data_ptr(), z.data_ptr(),
                       ws.data_ptr(), m, n, k, k, k, n + 5, n + 5, n + 3, need.value, 0, int(out_bf16), 3, 23)
    assert lib.pam_linear(args, torch.cuda.current_stream().cuda_stream) == 0
    assert same(y[:, :n].contiguous(), want) and same(z[:, :n].contiguous(), zw)
    assert bool((y[:, n:] == 7).all()) and bool((z[:, n:] == 9).all())


@pytest.mark.parametrize("name", ref.ACTIVATIONS)
@pytest.mark.parametrize("m", [1, 64, 400])
def test_special_values(name, m):
    """Zeros, infinities, NaN and far values reach the activation through the bias,
    on a product of zeros."""
    note(f"linear specials {name} {m}")
    bias = np.array([0.0, -0.0, np.inf, -np.inf, np.nan, 3e38, -3e38, 1e20, -1e20, 88.5, -88.5, 104.0, -104.0, 16.0,
                     -16.0, 13.5, -13.5, 5.0, -5.0, 1e-30, -1e-30, 1e-3, -1e-3] * 6, np.float32)
    y, z = pam.linear(to_dev(np.zeros((m, 8), np.float32)), to_dev(np.zeros((len(bias), 8), np.float32)), to_dev(bias), name,
                      save_z=True)
    z64 = np.broadcast_to(bias.astype(np.float64), (m, len(bias)))
    check(z.cpu().numpy(), z64, 0, "z")
    want = ref.activation(z64, name)
    with np.errstate(invalid="ignore"):
        check(y.cpu().numpy(), want, np.nan_to_num(tu.activation_error(z64, name), posinf=0), "y")


def test_special_operands():
    """Operands that are inf, NaN, tiny, zero or huge: as in gemm."""
    import torch
    note("linear, special operands")
    for m, k, n in ((5, 300, 40), (150, 300, 140), (600, 300, 1500)):
        x, w, bias, _ = inputs(m, k, n)
        x[0, 0], x[1, 5], w[3, 7], w[4, 9], x[2] = float("inf"), float("nan"), 1e30, 1e-35, 0.0
        z = pam.gemm(x, w, trans_b=True) + bias
        y = pam.linear(x, w, bias, "relu")
        assert torch.equal(torch.isnan(y), torch.isnan(z))
        fine = ~torch.isnan(z)
        assert torch.equal(y[fine], torch.relu(z)[fine])


def test_empty_results():
    import torch
    for m, k, n in ((0, 4, 5), (4, 4, 0), (0, 0, 0)):
        x, w, bias, res = inputs(m, k, n)
        y, z = pam.linear(x, w, bias, "gelu", res, save_z=True)
        assert y.shape == z.shape == (m, n)


def test_streams_and_graphs():
    """A layer's forward pass and the gradient of its additions on two streams at
    once, then captured and replayed with other inputs; the split product among them."""
    import torch
    note("linear and activation_grad on streams and in a graph")
    cases = [inputs(2048, 512, 770, seed=1), inputs(8, 4096, 512, seed=2), inputs(192, 12608, 192, seed=3)]
    assert pam.plan(192, 192, 12608)[2] > 1

    def run(c):
        x, w, bias, res = c
        y, z = pam.linear(x, w, bias, "gelu", res, save_z=True)
        return (y, z, *pam.activation_grad(y, z, "gelu"))

    want = [run(c) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = []
    for s, c in zip(streams, cases):
        with torch.cuda.stream(s):
            got.append(run(c))
    torch.cuda.synchronize()
    assert all(same(a, b) for g, w in zip(got, want) for a, b in zip(g, w))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = [run(c) for c in cases]
    for rep in range(3):
        for x, _, bias, _ in cases:
            x.mul_(1.25)
            bias.add_(0.1)
        want = [run(c) for c in cases]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(same(a, b) for g, w in zip(outs, want) for a, b in zip(g, w)), rep
    del graph


@pytest.mark.parametrize("seed", range(48))
def test_random_layers(seed):
    """Random sizes, types, views and parts, each against gemm and the definition."""
    import random
    import torch
    rng = random.Random(900 + seed)

    def log_uniform(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    m, k, n = log_uniform(1, 5000), log_uniform(1, 3000), log_uniform(1, 3000)
    while m * k * n > 3e9:
        m, k = max(m // 2, 1), max(k // 2, 1)
    bf16, out_bf16 = rng.random() < 0.4, rng.random() < 0.4
    name, pad = rng.choice(ref.ACTIVATIONS), rng.choice((0, 0, 1, 3, 8))
    x, w, bias, res = inputs(m, k, n, bf16, seed, out_bf16)
    if rng.random() < 0.5:
        x = torch.relu(x)
    bias = bias if rng.random() < 0.7 else None
    res = res if rng.random() < 0.5 else None
    wide = [torch.nn.functional.pad(t, (pad, 1 + pad))[:, pad:pad + t.shape[1]] if pad and t is not None else t
            for t in (x, w, res)]
    out = torch.bfloat16 if out_bf16 else torch.float32
    note(f"random layer {seed}: {m}x{k}x{n} {name} {x.dtype} -> {out}, pad {pad}, bias {bias is not None}, "
         f"residual {res is not None}")
    y, z = pam.linear(wide[0], wide[1], bias, name, wide[2], save_z=True, out_dtype=out)
    z32 = pam.gemm(x, w, trans_b=True)
    z32 = z32 if bias is None else z32 + bias
    if k <= 1024:
        assert same(z, z32.to(out))
    else:        # other orders of the same terms, whose magnitudes' sum is at most |x| |w|^T's
        size = x.float().abs().cpu().double() @ w.float().abs().cpu().double().t()
        off = (z.cpu().double() - z32.cpu().double()).abs()
        assert bool((off <= 2 * (k + 2) * tu.U * size + (2.0 ** -8 if out_bf16 else 2 * tu.U) * z32.cpu().double().abs()).all())
        z32 = pam.linear(x, w, bias)
    expect(y, z32, name, res, out_bf16, "y")


def test_host_threads():
    """Layers and their gradients from four host threads, a stream each."""
    import threading
    import torch
    note("linear from 4 host threads")
    cases = [inputs(*s, seed=5) for s in ((2048, 512, 300), (8, 2000, 500), (197, 64, 197), (300, 3000, 700))]

    def run(c):
        y, z = pam.linear(*c[:3], "silu", c[3], save_z=True)
        return (y, z, *pam.activation_grad(y, z, "silu"), pam.grad_norm([y, z]))

    want = [run(c) for c in cases]
    torch.cuda.synchronize()
    got, errors = [None] * len(cases), []

    def work(i):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                for j in range(20):
                    r = run(cases[(i + j) % len(cases)])
                    if (i + j) % len(cases) == i:
                        got[i] = r
            s.synchronize()
        except Exception as e:   # reported below, on the main thread
            errors.append((i, repr(e)))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(cases))]
    for t in threads:
        t.start()
    for t in threads:
        t.join(timeout=60)
    assert not any(t.is_alive() for t in threads) and not errors, errors
    assert all(same(a, b) for g, w in zip(got, want) for a, b in zip(g, w))
