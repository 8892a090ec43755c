"""The layer-and-step side of a PAM transformer at the sizes it is used at: linear layers with bias, activation
and residual, the gradient of what they add to their product, and the optimizer's step over all parameters.

``run`` computes each of them through the library (``own``) or in its plain form: elementary torch operations
in float32.  ``exact`` evaluates the definitions in float64: the PAM terms by Sec. 2.3's identity
``paexp2(palog2|a| + palog2|b|)``, the activations' gradient by differentiating them, the optimizer's moments
without rounding, or, where they are held in 8 bits, rounded where their definition rounds.

Kinds of case:

  linear   act(x .^ w^T + bias) + residual of `m` tokens, `k` -> `n`; ``z``: what the activation took, too
  grad     from the gradient of a layer's output that of its product, and the bias's
  adamw    one step over a model's parameters: `layers` layers of a decoder, or `tensors` ragged ones;
           ``clip``: the gradients' common norm first, and the step with its limit

The optimizer's state in 8 bits (blocks of 256 values of a tensor, one float32 scale a block, its largest
magnitude): the first moment as a sign and 7 bits, code c > 0 standing for the float32 of encoding (c + 889) <<
20 times the scale, the second as 8 bits, (c + 761) << 20; 0 is 0.  Codes come by adding 16 random bits below
the kept ones to the encoding of |value| / scale and dropping those, bits that a hash of seed, step, tensor and
element gives.  A code next to a border goes by the last bit of a moment, so that each operation on the way
there is rounded to float32 by itself, and gradients of these cases come unscaled.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16}
LR, BETA1, BETA2, EPS, DECAY, STEP, SEED = 3e-4, 0.9, 0.999, 1e-8, 0.01, 100, 1234
MAX_NORM = 1.0
BLOCK = 256


# ---------------------------------------------------------------------------
# The cases
# ---------------------------------------------------------------------------

def listed():
    return [
        # One token through the first layer of a transformer-base feed-forward block: the smallest call.
        dict(name="linear_token", kind="linear", m=1, k=512, n=2048, act="relu", bias=True, residual=False, z=False,
             dtype="float32", out="float32"),
        # A decoding step of 8 sequences through a large layer with bfloat16 weights, onto the residual stream.
        dict(name="linear_decode", kind="linear", m=8, k=4096, n=4096, act="none", bias=True, residual=True, z=False,
             dtype="bfloat16", out="bfloat16"),
        # Training: the first layer of a transformer-base feed-forward block, its pre-activations kept for the
        # backward pass.
        dict(name="linear_up", kind="linear", m=8192, k=512, n=2048, act="gelu", bias=True, residual=False, z=True,
             dtype="float32", out="float32"),
        # The second one, back onto the residual stream.
        dict(name="linear_down", kind="linear", m=8192, k=2048, n=512, act="none", bias=True, residual=True, z=False,
             dtype="float32", out="float32"),
        # Ragged: a batch of images' tokens through a narrow layer whose width no tile divides.
        dict(name="linear_ragged", kind="linear", m=1773, k=197, n=770, act="gelu_tanh", bias=True, residual=True, z=True,
             dtype="float32", out="bfloat16"),
        # A large layer.
        dict(name="linear_large", kind="linear", m=4096, k=4096, n=4096, act="silu", bias=False, residual=False, z=True,
             dtype="float32", out="float32"),
        # The backward pass of linear_up's additions.
        dict(name="grad_up", kind="grad", m=8192, n=2048, act="gelu", dtype="float32"),
        # Of a few odd rows: the smallest one.
        dict(name="grad_ragged", kind="grad", m=197, n=771, act="relu", dtype="float32"),
        # Of the large layer on bfloat16 activations.
        dict(name="grad_large", kind="grad", m=16384, n=4096, act="silu", dtype="bfloat16"),
        # The example decoder's 23 tensors: launches and host time count.
        dict(name="adamw_small", kind="adamw", layers=2, width=128, hidden=512, vocabulary=64, bits=32, clip=True,
             dtype="float32", copies=False),
        # A transformer-base decoder of 6 layers: bfloat16 gradients, and bfloat16 copies for the next step's products.
        dict(name="adamw_base", kind="adamw", layers=6, width=512, hidden=2048, vocabulary=8192, bits=32, clip=True,
             dtype="bfloat16", copies=True),
        # One large layer, the moments in 8 bits.
        dict(name="adamw_large", kind="adamw", layers=1, width=4096, hidden=16384, vocabulary=512, bits=8, clip=False,
             dtype="float32", copies=False),
    ]


ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
MOST_MACS = 4096 ** 3
MOST_OUT = 16384 * 4096
MOST_PARAMS = 1 << 26


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("linear", "linear", "grad", "adamw", "adamw"))
    if kind == "adamw":
        bits = rng.choice((8, 32))
        count = _log(rng, 1, 100)
        return dict(kind=kind, tensors=count, largest=_log(rng, 1, MOST_PARAMS // count), bits=bits,
                    clip=bits == 32 and rng.random() < 0.5, dtype=rng.choice(("float32", "bfloat16")),
                    copies=rng.random() < 0.3)
    act = rng.choice(ACTS)
    even = rng.choice((1, 1, 8, 64))
    m, n = _log(rng, 1, 16384), -(-_log(rng, 1, 8192) // even) * even
    if kind == "grad":
        return dict(kind=kind, m=min(m, MOST_OUT // n), n=n, act=act if act != "none" else "gelu",
                    dtype=rng.choice(("float32", "bfloat16")))
    k = -(-_log(rng, 1, 8192) // even) * even
    return dict(kind=kind, m=max(1, min(m, MOST_MACS // 2 // (k * n))), k=k, n=n, act=act, bias=rng.random() < 0.7,
                residual=rng.random() < 0.4, z=act != "none" and rng.random() < 0.5,
                dtype=rng.choice(("float32", "bfloat16")), out=rng.choice(("float32", "float32", "bfloat16")))


def _sizes(case):
    """Values of each tensor, by the case alone."""
    if "layers" not in case:
        rng = random.Random(case["tensors"] * 1000003 + case["largest"])
        return [case["largest"]] + [_log(rng, 1, case["largest"]) for _ in range(case["tensors"] - 1)]
    w, h, v = case["width"], case["hidden"], case["vocabulary"]
    # Embedding and the last norm and head; of a layer the norms, qkv, out, up and down with biases, and the
    # weights of the norms of queries and keys.
    return [v * w, w, v * w] + case["layers"] * [w, w, 2 * w * w, w * w, h * w, h, w * h, w, 32, 32]


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    dtype = TYPES[case["dtype"]]

    def normal(*shape, scale=1.0, dtype=dtype):
        return torch.empty(shape, device=DEV, dtype=dtype).normal_(0.0, scale, generator=g)

    if case["kind"] == "adamw":
        return _prepare_step(case, g, normal)
    m, n = case["m"], case["n"]
    if case["kind"] == "grad":
        return dict(case=case, dy=normal(m, n, scale=1e-3), z=normal(m, n))
    k, out = case["k"], TYPES[case["out"]]
    x = normal(m, k)
    if case["residual"] and case["act"] == "none":
        x.clamp_(min=0)                  # what comes back from a feed-forward block's middle
    return dict(case=case, x=x, w=normal(n, k, scale=1 / math.sqrt(k)),
                bias=normal(n, scale=0.1, dtype=torch.float32) if case["bias"] else None,
                residual=normal(m, n, dtype=out) if case["residual"] else None)


def _prepare_step(case, g, normal):
    """Parameters, gradients and moments as one allocation each, every tensor a view of it."""
    sizes = _sizes(case)
    total = sum(sizes)
    state = dict(case=case, step=STEP, p=normal(total, scale=0.02, dtype=torch.float32), g=normal(total, scale=1e-3))
    if case["bits"] == 32:
        state["m"] = normal(total, scale=3e-4, dtype=torch.float32)
        state["v"] = normal(total, scale=1e-3, dtype=torch.float32).square_().clamp_(min=1e-8)
    else:
        # Codes of magnitudes within about 2^5 of the block's largest.
        state["m"] = torch.randint(88, 128, (total,), device=DEV, dtype=torch.uint8, generator=g)
        state["m"] |= torch.randint(2, (total,), device=DEV, dtype=torch.uint8, generator=g) << 7
        state["v"] = torch.randint(190, 256, (total,), device=DEV, dtype=torch.uint8, generator=g)
        blocks = [-(-n // BLOCK) for n in sizes]
        for name, scale in (("ms", 1e-3), ("vs", 1e-6)):
            state[name] = scale * (0.5 + torch.rand(sum(blocks), device=DEV, generator=g))
            state[name + "_each"] = list(state[name].split(blocks))
    if case["copies"]:
        state["copy"] = torch.zeros(total, dtype=torch.bfloat16, device=DEV)
    for name in ("p", "g", "m", "v", "copy"):
        if name in state:
            state[name + "_each"] = list(state[name].split(sizes))
    return state


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(state):
    case = state["case"]
    if case["kind"] == "adamw":
        state["step"] += 1
    if own:
        return _run_own(case, state)
    if case["kind"] == "adamw":
        return _step(case, state)
    return _linear(case, state) if case["kind"] == "linear" else _grad(case, state)


def _run_own(case, s):
    import paper_2305_17190_amd as pam

    act = None if case.get("act") == "none" else case.get("act")
    if case["kind"] == "linear":
        return pam.linear(s["x"], s["w"], s["bias"], activation=act, residual=s["residual"], save_z=case["z"],
                          out_dtype=TYPES[case["out"]])
    if case["kind"] == "grad":
        return pam.activation_grad(s["dy"], s["z"], act)
    norm = pam.grad_norm(s["g_each"]) if case["clip"] else None
    pam.adamw_step(s["p_each"], s["g_each"], s["m_each"], s["v_each"], s["step"], lr=LR, betas=(BETA1, BETA2), eps=EPS,
                   weight_decay=DECAY, avg_scales=s.get("ms_each"), sq_scales=s.get("vs_each"),
                   copies=s.get("copy_each"), norm=norm, max_norm=MAX_NORM if case["clip"] else None, seed=SEED)
    return _stepped(case, s, norm)


def _stepped(case, s, norm):
    """What a step leaves, the moments as the values they stand for."""
    m, v = s["m"], s["v"]
    if case["bits"] == 8:
        m = torch.cat([_values(c, x, 889, 127) for c, x in zip(s["m_each"], s["ms_each"])])
        v = torch.cat([_values(c, x, 761, 255) for c, x in zip(s["v_each"], s["vs_each"])])
    return s["p"], m, v, s.get("copy"), norm


# Plain forms ------------------------------------------------------------

MIN_NORMAL, BIAS, MAGNITUDE = 0x00800000, 0x3F800000, 0x7FFFFFFF
SOME = 1 << 24       # terms of a product at once


def _pam_product(x, w):
    """x .^ w^T of float32 matrices: the sums of the magnitudes' encodings less one bias, zero below the normal
    range or for an operand that is zero, with the product of the signs.  Operands stay far from the top of the
    float32 range, so that nothing saturates."""
    mx, mw = (t.view(torch.int32) & MAGNITUDE for t in (x, w))
    sx, sw = (t.sign() * (m >= MIN_NORMAL) for t, m in ((x, mx), (w, mw)))
    mw = mw - BIAS
    out = torch.empty(x.shape[0], w.shape[0], device=x.device)
    rows = max(1, SOME // w.numel())
    for r in range(0, x.shape[0], rows):         # all terms at once would not fit
        t = mx[r:r + rows, None] + mw
        t.masked_fill_(t < MIN_NORMAL, 0)
        out[r:r + rows] = t.view(torch.float32).mul_(sx[r:r + rows, None]).mul_(sw).sum(-1)
    return out


TANH0, TANH1 = math.sqrt(2 / math.pi), math.sqrt(2 / math.pi) * 0.044715


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, 0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(z * (TANH0 + TANH1 * z * z)))
    return z / (1 + torch.exp(-z)) if act == "silu" else z


def _linear(case, s):
    z = _pam_product(s["x"].float(), s["w"].float())
    if s["bias"] is not None:
        z = z + s["bias"]
    y = _act(z, case["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out = TYPES[case["out"]]
    return (y.to(out), z.to(out)) if case["z"] else y.to(out)


def _grad(case, s):
    dy, z = s["dy"].float(), s["z"].float()
    if case["act"] == "relu":
        d = torch.where(z > 0, 1.0, 0.0)
    elif case["act"] == "gelu":
        d = 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    elif case["act"] == "gelu_tanh":
        t = torch.tanh(z * (TANH0 + TANH1 * z * z))
        d = 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * (TANH0 + 3 * TANH1 * z * z)
    else:
        t = 1 / (1 + torch.exp(-z))
        d = t + z * t * (1 - t)
    dz = dy * d
    return dz.to(s["dy"].dtype), dz.sum(0)


def _mix(x):
    """A 32-bit hash (xor-shifts and two odd factors)."""
    x = ((x ^ (x >> 16)) * 0x7FEB352D) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x846CA68B) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random(step, tensor, n):
    """Two sets of random bits for each element of a tensor, 20 bits whose low four are 8."""
    key = _mix((_mix((SEED + step * 0x9E3779B9) & 0xFFFFFFFF) + tensor) & 0xFFFFFFFF)
    h = _mix((torch.arange(n, device=DEV) + key) & 0xFFFFFFFF)
    return ((h & 0xFFFF) << 4) + 8, ((h >> 16) << 4) + 8


def _values(code, scale, low, most):
    """The values that 8-bit codes stand for, in float32."""
    c = code.int()
    x = torch.where((c & most) > 0, ((c & most) + low) << 20, 0).view(torch.float32)
    x = x * scale.repeat_interleave(BLOCK)[:x.numel()]
    return torch.where(c > most, -x, x)


def _coded(x, low, least, bits):
    """Codes of magnitudes x and their blocks' scales."""
    n = x.numel()
    blocks = torch.nn.functional.pad(x, (0, -n % BLOCK)).view(-1, BLOCK)
    scale = blocks.amax(1)
    part = (blocks / scale.clamp(min=1e-37)[:, None]).flatten()[:n]
    code = ((part.view(torch.int32) + bits) >> 20) - low
    return code.clamp_(min=0).maximum((least & (x > 0)).to(code.dtype)), scale


def _moments8(s, t, g):
    """The moments of tensor t after its gradient g, and their codes and scales in place of the old ones."""
    m = _values(s["m_each"][t], s["ms_each"][t], 889, 127) * BETA1 + g * (1 - BETA1)
    v = _values(s["v_each"][t], s["vs_each"][t], 761, 255) * BETA2 + g * (1 - BETA2) * g
    rm, rv = _random(s["step"], t, g.numel())
    code, scale = _coded(m.abs(), 889, False, rm)
    s["m_each"][t].copy_(code | ((m < 0) & (code > 0)).to(code.dtype) << 7)
    s["ms_each"][t].copy_(scale)
    code, scale = _coded(v, 761, True, rv)
    s["v_each"][t].copy_(code)
    s["vs_each"][t].copy_(scale)
    return m, v


def _moved(p, m, v, step):
    """Parameters after their moments."""
    c1, c2 = 1 - BETA1 ** step, 1 - BETA2 ** step
    return p * (1 - LR * DECAY) - LR / c1 * (m / (v.sqrt() / math.sqrt(c2) + EPS))


def _step(case, s):
    step, g, norm = s["step"], s["g"].float(), None
    if case["clip"]:
        norm = (g * g).sum().sqrt()
        g = g * (MAX_NORM / (norm + 1e-6)).clamp(max=1.0)
    if case["bits"] == 32:
        m, v = s["m"] * BETA1 + g * (1 - BETA1), s["v"] * BETA2 + g * (1 - BETA2) * g
        s["m"].copy_(m)
        s["v"].copy_(v)
    else:
        each = [_moments8(s, t, x.float()) for t, x in enumerate(s["g_each"])]
        m, v = (torch.cat(x) for x in zip(*each))
    s["p"].copy_(_moved(s["p"], m, v, step))
    if case["copies"]:
        s["copy"].copy_(s["p"])
    return _stepped(case, s, norm)


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------

def _palog2(x):
    f, e = torch.frexp(x.abs())
    return torch.where(x == 0, 0.0, e - 1 + (2 * f - 1))


def _power(e):
    """2^e for whole e, without a rounding."""
    return (e.long() + 1023 << 52).view(torch.float64)


def _exact_product(x, w):
    lx, lw, sx, sw = _palog2(x), _palog2(w), x.sign(), w.sign()
    out = torch.empty(x.shape[0], w.shape[0], dtype=torch.float64, device=DEV)
    rows = max(1, SOME // w.numel())
    for r in range(0, x.shape[0], rows):
        s = lx[r:r + rows, None] + lw
        whole = s.floor()
        s.sub_(whole).add_(1).mul_(_power(whole))
        out[r:r + rows] = s.mul_(sx[r:r + rows, None]).mul_(sw).sum(-1)
    return out


def _exact_act(z, act):
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "gelu_tanh":
        return z * torch.sigmoid(2 * TANH0 * (z + 0.044715 * z ** 3))
    return z * torch.sigmoid(z) if act == "silu" else z.relu() if act == "relu" else z


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "linear":
        z = _exact_product(s["x"].double(), s["w"].double())
        if s["bias"] is not None:
            z = z + s["bias"].double()
        y = _exact_act(z, case["act"])
        if s["residual"] is not None:
            y = y + s["residual"].double()
        return (y, z) if case["z"] else y
    if case["kind"] == "grad":
        z = s["z"].double().requires_grad_()
        dz, = torch.autograd.grad(_exact_act(z, case["act"]), z, s["dy"].double())
        return dz, dz.sum(0)
    return _exact_step(case, s)


def _f32(x):
    return x.float().double()


def _exact_value(code, scale, most):
    """What codes stand for, by the octave and the eighth of it."""
    c = code.double() % (most + 1)
    place = c + (1016 - most)
    octave = (place / 8).floor()
    size = (1 + place / 8 - octave) * _power(octave - 127)
    x = _f32(size * scale.double().repeat_interleave(BLOCK)[:c.numel()])
    return torch.where(c > 0, torch.where(code > most, -x, x), 0.0)


def _exact_held(x, most, least, bits):
    """Magnitudes as their blocks hold them."""
    n = x.numel()
    top = torch.nn.functional.pad(x, (0, -n % BLOCK)).view(-1, BLOCK).amax(1).repeat_interleave(BLOCK)[:n]
    part = _f32(x / top)
    code = (8 * (_palog2(part) + 127) + bits.double() / 2 ** 20).floor() - (1016 - most)
    code = torch.where(part > 0, code.clamp(min=least), 0.0).clamp(min=0)
    place = code + (1016 - most)
    octave = (place / 8).floor()
    return torch.where(code > 0, _f32((1 + place / 8 - octave) * _power(octave - 127) * top), 0.0)


def _exact_step(case, s):
    s["step"] += 1
    g, norm = s["g"].double(), None
    if case["clip"]:
        norm = torch.linalg.vector_norm(g)
        g = g * torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0)
    if case["bits"] == 32:
        m, v = s["m"].double().lerp(g, 1 - BETA1), s["v"].double().lerp(g * g, 1 - BETA2)
        p = _moved(s["p"].double(), m, v, s["step"])
        return p, m, v, p if case["copies"] else None, norm
    b1, c1, b2, c2 = (torch.tensor(b, dtype=torch.float32).item() for b in (BETA1, 1 - BETA1, BETA2, 1 - BETA2))
    each = []
    for t, g in enumerate(s["g_each"]):
        g = g.double()
        m = _f32(_f32(_exact_value(s["m_each"][t], s["ms_each"][t], 127) * b1) + _f32(g * c1))
        v = _f32(_f32(_exact_value(s["v_each"][t], s["vs_each"][t], 255) * b2) + _f32(_f32(g * c2) * g))
        rm, rv = _random(s["step"], t, g.numel())
        each.append((m, v, m.sign() * _exact_held(m.abs(), 127, 0, rm), _exact_held(v, 255, 1, rv)))
    m, v, held_m, held_v = (torch.cat(x) for x in zip(*each))
    p = _moved(s["p"].double(), m, v, s["step"])
    return p, held_m, held_v, p if case["copies"] else None, None


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    size = {"float32": 4, "bfloat16": 2}
    each = size[case["dtype"]]
    if case["kind"] == "linear":
        m, k, n, out = case["m"], case["k"], case["n"], size[case["out"]]
        # A PAM and an addition for each term.
        return {"bytes": each * (m + n) * k + 4 * n * case["bias"] + out * m * n * (1 + case["residual"] + case["z"]),
                "flops": 2 * m * n * k + 10 * m * n}
    if case["kind"] == "grad":
        return {"bytes": 3 * each * case["m"] * case["n"] + 4 * case["n"], "flops": 20 * case["m"] * case["n"]}
    sizes = _sizes(case)
    held = sum(sizes) * (16 if case["bits"] == 32 else 4) + (0 if case["bits"] == 32 else 16 * sum(-(-n // BLOCK) for n in sizes))
    return {"bytes": held + sum(sizes) * (8 + each + 2 * case["copies"]), "flops": sum(sizes) * 20}
