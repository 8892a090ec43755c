"""What the autograd wrappers give and what they refuse, with stand-ins for the
kernels that, like them, record nothing (CPU)."""
import pytest

torch = pytest.importorskip("torch")

from paper_2305_17190_amd import autograd  # noqa: E402

EPS = 1e-5


def plain(x, weight, cos, sin, positions):
    """Norm and rotation of heads in torch."""
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    y = y if weight is None else y * weight
    half = cos.shape[1]
    c, s = cos[positions.long()][:, None], sin[positions.long()][:, None]
    a, b = y[..., :half], y[..., half:]
    return torch.cat((a * c - b * s, b * c + a * s), -1)


@pytest.fixture
def norm_rope(monkeypatch):
    """pam_norm_rope over stand-ins; the gradient's calls."""
    calls = []

    def forward(q, k, positions, cos, sin, qw, kw, eps, interleaved):
        with torch.no_grad():
            return plain(q, qw, cos, sin, positions), plain(k, kw, cos, sin, positions)

    def gradient(dq, dk, q, k, positions, cos, sin, qw, kw, eps, interleaved):
        calls.append(dict(dq=dq, dk=dk, q=q, k=k, q_weight=qw, k_weight=kw))
        out = [None] * 4
        for i, (dz, x, w) in enumerate(((dq, q, qw), (dk, k, kw))):
            if x is None:
                continue
            with torch.enable_grad():
                inputs = [t.detach().requires_grad_() for t in (x, w) if t is not None]
                z = plain(inputs[0], inputs[1] if w is not None else None, cos, sin, positions)
                got = torch.autograd.grad(z, inputs, dz.detach())
            out[i], out[2 + i] = got[0], got[1] if w is not None else None
        return tuple(out)

    monkeypatch.setattr(autograd, "_norm_rope", forward)
    monkeypatch.setattr(autograd, "_norm_rope_grad", gradient)
    return calls


def inputs(seed=0, tokens=5):
    g = torch.Generator().manual_seed(seed)
    q, k = (torch.randn(tokens, h, 8, generator=g, dtype=torch.float64).requires_grad_() for h in (3, 2))
    weights = [(1 + 0.1 * torch.randn(8, generator=g, dtype=torch.float64)).requires_grad_() for _ in "qk"]
    angle = torch.arange(10, dtype=torch.float64)[:, None] * torch.tensor([1.0, 0.3, 0.1, 0.01], dtype=torch.float64)
    return q, k, torch.randint(10, (tokens,), generator=g, dtype=torch.int32), angle.cos(), angle.sin(), *weights


def test_first_derivatives_of_norm_rope(norm_rope):
    q, k, pos, cos, sin, qw, kw = inputs()
    zq, zk = autograd.pam_norm_rope(q, k, pos, cos, sin, qw, kw, EPS)
    got = torch.autograd.grad(zq.pow(2).sum() + zk.exp().sum(), (q, k, qw, kw))
    want = torch.autograd.grad(plain(q, qw, cos, sin, pos).pow(2).sum() + plain(k, kw, cos, sin, pos).exp().sum(),
                               (q, k, qw, kw))
    assert all(torch.allclose(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("loss", [lambda z: z.sum(), lambda z: z.pow(3).sum()])
def test_second_derivatives_of_norm_rope_raise(norm_rope, loss):
    """Also where the loss is linear, so that the gradient reaching the wrapper is
    a constant and the inputs alone would carry the second derivative."""
    q, k, pos, cos, sin, qw, kw = inputs()
    zq, zk = autograd.pam_norm_rope(q, k, pos, cos, sin, qw, kw, EPS)
    total = loss(zq) + loss(zk)
    for x in (q, k, qw, kw):
        (g,) = torch.autograd.grad(total, x, create_graph=True)
        assert torch.allclose(g, torch.autograd.grad(total, x, retain_graph=True)[0])     # itself right, and of use
        with pytest.raises(RuntimeError, match="first derivatives only"):
            (total + g.pow(2).sum()).backward(retain_graph=True)


@pytest.mark.parametrize("needed", [(0,), (1,), (5,), (6,), (0, 5), (0, 1), (1, 5), (0, 1, 5, 6)])
@pytest.mark.parametrize("create_graph", [False, True])
def test_norm_rope_works_on_the_sides_needed_alone(norm_rope, needed, create_graph):
    """Queries (inputs 0 and 5) or keys (1 and 6) that need no gradient are not worked on."""
    args = [t.detach() for t in inputs()]
    for i in needed:
        args[i].requires_grad_()
    zq, zk = autograd.pam_norm_rope(*args, EPS)
    got = torch.autograd.grad(zq.pow(2).sum() + zk.exp().sum(), [args[i] for i in needed], create_graph=create_graph)
    q, k, pos, cos, sin, qw, kw = args
    total = plain(q, qw, cos, sin, pos).pow(2).sum() + plain(k, kw, cos, sin, pos).exp().sum()
    want = torch.autograd.grad(total, [args[i] for i in needed])
    assert all(torch.allclose(a, b) for a, b in zip(got, want))
    (call,) = norm_rope
    for side, at in (("q", (0, 5)), ("k", (1, 6))):
        given = bool(set(at) & set(needed))
        assert all((call[name] is not None) == given for name in (side, "d" + side, side + "_weight"))


@pytest.fixture
def products(monkeypatch):
    """The wrappers of the products over stand-ins with ordinary products."""
    def turned(t, trans):
        return t.transpose(-1, -2) if trans else t

    def product(a, b, trans_a=False, trans_b=False, mantissa_bits=23):
        with torch.no_grad():
            return turned(a, trans_a) @ turned(b, trans_b)

    for name in ("_gemm", "_bmm"):
        monkeypatch.setattr(autograd, name, product)
    monkeypatch.setattr(autograd, "_exact_grad", lambda a, b, mod, trans_a=False: product(a, b, trans_a))


def floats(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).requires_grad_()


@pytest.mark.parametrize("derivative", ["approximate", "exact"])
def test_second_derivatives_of_linear_raise(products, derivative):
    x, w, bias = floats(0, 4, 6), floats(1, 5, 6), floats(2, 5)
    y = autograd.pam_linear(x, w, bias, derivative=derivative)
    want = torch.autograd.grad((x @ w.T + bias).pow(2).sum(), (x, w, bias))
    got = torch.autograd.grad(y.pow(2).sum(), (x, w, bias), create_graph=True)
    assert all(torch.allclose(a, b, rtol=1e-5) for a, b in zip(got, want))
    for g in got[:2]:
        with pytest.raises(RuntimeError, match="first derivatives only"):
            (y.sum() + g.pow(2).sum()).backward(retain_graph=True)
    got[2].sum().backward(retain_graph=True, inputs=[bias])       # torch's own sum
    # Gradients that depend on no other tracked tensor are constants, as they should be.
    y = autograd.pam_linear(x, w.detach(), derivative=derivative)
    (g,) = torch.autograd.grad(y.sum(), x, create_graph=True)
    assert not g.requires_grad


def test_second_derivatives_of_matmul_raise(products):
    a, b = floats(3, 2, 4, 6), floats(4, 2, 6, 5)
    c = autograd.pam_matmul(a, b)
    want = torch.autograd.grad((a @ b).pow(2).sum(), (a, b))
    got = torch.autograd.grad(c.pow(2).sum(), (a, b), create_graph=True)
    assert all(torch.allclose(x, y, rtol=1e-5) for x, y in zip(got, want))
    for g in got:
        with pytest.raises(RuntimeError, match="first derivatives only"):
            (c.sum() + g.pow(2).sum()).backward(retain_graph=True)
