"""The attention-side operators of a PAM transformer at the sizes they are used at: norms of queries and
keys with the position rotation (forward and gradient), appending to a paged key/value cache, and PAM
attention over that cache, for single tokens and for chunks.

``run`` computes each of them through the library (``own``) or in its plain form: elementary torch
operations in float32.  ``exact`` evaluates the definitions in float64, the PAM terms in their value form
``2^(E_A + E_B + c) (1 + M_A + M_B - c)`` and the gradient by differentiating the forward formula.

Kinds of case:

  norm_rope   queries and keys of `tokens` tokens; ``grad``: the gradient of the same
  append      keys and values of `tokens` new tokens into the cache, with their queries normed and rotated
  attention   `batch` sequences of up to `kv` cached keys, each with up to `chunk` new tokens
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
EPS = 1e-6
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16}


# ---------------------------------------------------------------------------
# The cases
# ---------------------------------------------------------------------------

def listed():
    return [
        # Training a transformer-base layer (8 heads of 64, 8192 tokens): queries and keys on their way to the
        # attention products, and the gradient on the way back.
        dict(name="norm_rope_base", kind="norm_rope", grad=False, tokens=8192, hq=8, hk=8, d=64, rot=64,
             interleaved=False, dtype="float32"),
        dict(name="norm_rope_grad_base", kind="norm_rope", grad=True, tokens=8192, hq=8, hk=8, d=64, rot=64,
             interleaved=False, dtype="float32"),
        # Training a large layer (16384 tokens, width 4096 = 32 heads of 128, 8 key heads) on bfloat16 activations.
        dict(name="norm_rope_grad_large", kind="norm_rope", grad=True, tokens=16384, hq=32, hk=8, d=128, rot=128,
             interleaved=False, dtype="bfloat16"),
        # One decoding step of 8 sequences: a single small launch, latency counts.
        dict(name="append_decode", kind="append", tokens=8, hq=32, hk=8, d=128, rot=128, page=16, interleaved=False,
             dtype="float32", cache="bfloat16"),
        # 64 images of 197 tokens, 3 heads of 64, half of each head rotated in adjacent pairs, float32 cache.
        dict(name="append_vit", kind="append", tokens=12608, hq=3, hk=3, d=64, rot=32, page=32, interleaved=True,
             dtype="float32", cache="float32"),
        # Filling the cache with a long prompt of the large layer.
        dict(name="append_prompt", kind="append", tokens=16384, hq=32, hk=8, d=128, rot=128, page=64,
             interleaved=False, dtype="float32", cache="bfloat16"),
        # One user's next token: a short context, the smallest call.
        dict(name="decode_one", kind="attention", batch=1, kv=1000, chunk=1, hq=32, hk=8, d=128, page=16, window=0,
             dtype="float32", cache="bfloat16"),
        # A translation decoder (8 heads of 64, 32 sequences of up to 256 tokens), float32 cache.
        dict(name="decode_base", kind="attention", batch=32, kv=256, chunk=1, hq=8, hk=8, d=64, page=16, window=0,
             dtype="float32", cache="float32"),
        # Serving: 128 sequences of different lengths at once.
        dict(name="decode_batch", kind="attention", batch=128, kv=8192, chunk=1, hq=32, hk=8, d=128, page=16,
             window=0, dtype="float32", cache="bfloat16"),
        # One very long context: few rows, all the work along the keys.
        dict(name="decode_long", kind="attention", batch=1, kv=131071, chunk=1, hq=32, hk=8, d=128, page=64,
             window=0, dtype="bfloat16", cache="bfloat16"),
        # Ragged chunks of several prompts, every head with its own keys, a sliding window.
        dict(name="chunk_ragged", kind="attention", batch=5, kv=1777, chunk=333, hq=8, hk=8, d=64, page=48,
             window=1024, dtype="float32", cache="float32"),
        # A chunk of a long prompt of the large layer.
        dict(name="chunk_large", kind="attention", batch=1, kv=4096, chunk=512, hq=32, hk=8, d=128, page=64,
             window=0, dtype="float32", cache="bfloat16"),
    ]


MOST_ELEMENTS = 16384 * 40 * 128      # of norm_rope_grad_large / append_prompt
MOST_MACS = 4096 * 512 * 32 * 128     # score products of chunk_large (before the causal mask)
HEADS = ((1, 1), (3, 3), (8, 8), (8, 2), (16, 4), (32, 8), (32, 32), (12, 1), (15, 5))


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("norm_rope", "append", "attention", "attention"))
    hq, hk = rng.choice(HEADS)
    d = rng.choice((32, 64, 64, 80, 96, 128, 128, 192, 256))
    dtype = rng.choice(("float32", "bfloat16"))
    if kind != "attention":
        most = min(16384, MOST_ELEMENTS // ((hq + 2 * hk) * d))
        case = dict(kind=kind, tokens=_log(rng, 1, most), hq=hq, hk=hk, d=d, rot=rng.choice((d, d, d // 2)),
                    interleaved=rng.random() < 0.3, dtype=dtype)
        if kind == "norm_rope":
            return dict(case, grad=rng.random() < 0.5)
        return dict(case, page=rng.choice((16, 32, 48, 64, 128)), cache=rng.choice(("float32", "bfloat16")))
    if rng.random() < 0.5:
        chunk, batch = 1, _log(rng, 1, 128)
    else:
        chunk, batch = _log(rng, 2, 512), _log(rng, 1, 8)
    most = MOST_MACS // 2 // (batch * chunk * hq * d)
    kv = _log(rng, max(chunk, 64), max(chunk, 64, min(131072, most)))
    while batch > 1 and batch * chunk * kv * hq * d > MOST_MACS:
        batch -= 1
    while chunk > 1 and batch * chunk * kv * hq * d > MOST_MACS:
        chunk = max(1, chunk * 3 // 4)
    return dict(kind=kind, batch=batch, kv=kv, chunk=chunk, hq=hq, hk=hk, d=d,
                page=rng.choice((16, 32, 48, 64, 128)), window=rng.choice((0, 0, 0, max(1, kv // 3))), dtype=dtype,
                cache=rng.choice(("float32", "bfloat16")))


def _lengths(case):
    """(new tokens, cached keys with them) of each sequence: ragged, the first one the longest; by the case's
    sizes alone."""
    rng = random.Random(case["batch"] * 1000003 + case["kv"] * 1009 + case["chunk"])
    new = [case["chunk"]] + [rng.randint(max(1, case["chunk"] // 2), case["chunk"]) for _ in range(case["batch"] - 1)]
    kv = [case["kv"]] + [max(n, rng.randint(case["kv"] // 4 + 1, case["kv"])) for n in new[1:]]
    return new, kv


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _tables(positions, rot):
    """cos and sin of every position's angles, one column for each rotated pair."""
    freq = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * freq
    return angle.cos().float().to(DEV), angle.sin().float().to(DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    kind, d, hq, hk = case["kind"], case["d"], case["hq"], case["hk"]
    dtype = TYPES[case["dtype"]]

    def normal(*shape, scale=1.0, dtype=dtype):
        return torch.empty(shape, device=DEV, dtype=dtype).normal_(0.0, scale, generator=g)

    if kind == "attention":
        new, kv = _lengths(case)
        page = case["page"]
        pages = [-(-n // page) for n in kv]
        order = torch.randperm(sum(pages), generator=g, device=DEV).to(torch.int32)
        table = torch.zeros(len(kv), max(pages), dtype=torch.int32, device=DEV)
        at = 0
        for b, n in enumerate(pages):
            table[b, :n] = order[at:at + n]
            at += n
        shape = (sum(pages), page, hk, d)
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        return dict(case=case, q=normal(starts[-1], hq, d, scale=2.0), k_cache=normal(*shape, dtype=TYPES[case["cache"]]),
                    v_cache=normal(*shape, dtype=TYPES[case["cache"]]), table=table,
                    kv_lens=torch.tensor(kv, dtype=torch.int32, device=DEV),
                    q_starts=torch.tensor(starts, dtype=torch.int32, device=DEV), max_q=max(new), max_kv=max(kv))

    t = case["tokens"]
    # Queries, keys and values are views of one projection's output, as a layer has them.
    qkv = normal(t, hq + 2 * hk, d, scale=1.5)
    state = dict(case=case, q=qkv[:, :hq], k=qkv[:, hq:hq + hk], v=qkv[:, hq + hk:],
                 q_weight=1 + normal(d, scale=0.2, dtype=torch.float32),
                 k_weight=1 + normal(d, scale=0.2, dtype=torch.float32))
    state["cos"], state["sin"] = _tables(4096, case["rot"])
    state["positions"] = torch.randint(4096, (t,), generator=g, device=DEV, dtype=torch.int32)
    if kind == "norm_rope":
        if case["grad"]:
            state["dq"], state["dk"] = normal(t, hq, d, scale=1e-2), normal(t, hk, d, scale=1e-2)
        return state
    pages = -(-t // case["page"]) * 5 // 4 + 1
    state["k_cache"], state["v_cache"] = (normal(pages, case["page"], hk, d, dtype=TYPES[case["cache"]]) for _ in "kv")
    state["slots"] = torch.randperm(pages * case["page"], generator=g, device=DEV)[:t]
    return state


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(state):
    case = state["case"]
    if own:
        return _run_own(case, state)
    if case["kind"] == "attention":
        return _attention(case, state)
    if case["kind"] == "append":
        return _append(case, state)
    return _norm_rope_grad(case, state) if case["grad"] else _norm_rope(case, state)


def _run_own(case, s):
    import paper_2305_17190_amd as pam

    if case["kind"] == "attention":
        return pam.paged_attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["kv_lens"],
                                   q_starts=s["q_starts"], max_q=s["max_q"], max_kv=s["max_kv"],
                                   window=case["window"])
    norm = dict(q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS, interleaved=case["interleaved"])
    if case["kind"] == "append":
        q = pam.append_kv(s["k"], s["v"], s["k_cache"], s["v_cache"], s["slots"], positions=s["positions"],
                          cos=s["cos"], sin=s["sin"], q=s["q"], **norm)
        return q, s["k_cache"], s["v_cache"]
    if case["grad"]:
        return pam.norm_rope_grad(s["dq"], s["dk"], s["q"], s["k"], s["positions"], s["cos"], s["sin"], **norm)
    return pam.norm_rope(s["q"], s["k"], s["positions"], s["cos"], s["sin"], **norm)


# Plain forms ------------------------------------------------------------

def _halves(x, rot, interleaved):
    """The two members of each rotated pair, and the values that stay."""
    if interleaved:
        return x[..., 0:rot:2], x[..., 1:rot:2], x[..., rot:]
    return x[..., :rot // 2], x[..., rot // 2:rot], x[..., rot:]


def _joined(a, b, rest, interleaved):
    pair = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((pair, rest), -1)


def _normed(x, weight):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight


def _rotated(x, cos, sin, case):
    a, b, rest = _halves(x, case["rot"], case["interleaved"])
    return _joined(a * cos - b * sin, b * cos + a * sin, rest, case["interleaved"])


def _norm_rope(case, s):
    cos, sin = (s[name][s["positions"]][:, None] for name in ("cos", "sin"))
    return tuple(_rotated(_normed(s[x].float(), s[x + "_weight"]), cos, sin, case).to(s[x].dtype) for x in "qk")


def _norm_rope_grad(case, s):
    cos, sin = (s[name][s["positions"]][:, None] for name in ("cos", "sin"))
    dx, dw = [], []
    for name in "qk":
        x, w = s[name].float(), s[name + "_weight"]
        grad = _rotated(s["d" + name].float(), cos, -sin, case)
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        xr, u = x * r, grad * w
        dw.append((grad * xr).sum((0, 1)))
        dx.append((r * (u - xr * (u * xr).mean(-1, keepdim=True))).to(s[name].dtype))
    return (*dx, *dw)


def _append(case, s):
    q, k = _norm_rope(case, dict(s, q=s["q"].float(), k=s["k"].float()))
    page, at = s["slots"] // case["page"], s["slots"] % case["page"]
    s["k_cache"][page, at] = k.to(s["k_cache"].dtype)
    s["v_cache"][page, at] = s["v"].to(s["v_cache"].dtype)
    return q.to(s["q"].dtype), s["k_cache"], s["v_cache"]


MIN_NORMAL, BIAS, MAGNITUDE = 0x00800000, 0x3F800000, 0x7FFFFFFF


def _pam_sum(a, b, dim):
    """Sum over `dim` of the PAM of two broadcast float32 tensors: the sum of the magnitudes' encodings less one
    bias, zero where that falls below the normal range or an operand is zero, with the product of the signs.
    Activations stay far from the top of the float32 range, so nothing saturates."""
    ma, mb = (x.contiguous().view(torch.int32) & MAGNITUDE for x in (a, b))
    t = ma + (mb - BIAS)
    t.masked_fill_(t < MIN_NORMAL, 0)
    value = t.view(torch.float32)
    for x, m in ((a, ma), (b, mb)):
        value *= torch.where(m < MIN_NORMAL, 0.0, x.sign())
    return value.sum(dim)


def _visible(case, new, kv, rows, keys):
    """Which keys the rows (positions among a sequence's new tokens) see; new and kv broadcast over sequences."""
    p = kv - new + rows
    ok = (keys < kv) & (keys <= p) & (rows < new)
    return ok & (keys > p - case["window"]) if case["window"] else ok


def _attention(case, s):
    hq, hk, d = case["hq"], case["hk"], case["d"]
    g, b, most_q, most_kv = hq // hk, case["batch"], s["max_q"], s["max_kv"]
    starts = s["q_starts"].long()
    new = (starts[1:] - starts[:-1])[:, None]
    rows = torch.arange(most_q, device=DEV)
    at = (starts[:-1, None] + rows).clamp_(max=s["q"].shape[0] - 1)
    q = s["q"][at].float().view(b, most_q, hk, g, d).transpose(1, 2)                          # b hk row g d
    k, v = (s[c][s["table"].long()].float().flatten(1, 2)[:, :most_kv].transpose(1, 2) for c in ("k_cache", "v_cache"))
    scores = _pam_sum(q.reshape(b, hk, most_q * g, 1, d), k.unsqueeze(2), -1) / math.sqrt(d)  # b hk (row g) key
    seen = _visible(case, new[:, :, None], s["kv_lens"].long()[:, None, None], rows[:, None],
                    torch.arange(most_kv, device=DEV))
    seen = seen.repeat_interleave(g, 1).unsqueeze(1)
    scores = scores.masked_fill(~seen, -math.inf)
    p = (scores - scores.amax(-1, keepdim=True).clamp_(min=-1e30)).exp()
    p = p / p.sum(-1, keepdim=True).clamp_(min=1e-30)
    out = _pam_sum(p.unsqueeze(-1), v.unsqueeze(2), -2)                                       # b hk (row g) d
    out = out.view(b, hk, most_q, g, d).transpose(1, 2).reshape(b, most_q, hq, d)
    token = torch.arange(s["q"].shape[0], device=DEV)
    seq = torch.searchsorted(starts, token, right=True) - 1
    return out[seq, token - starts[seq]]


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------

def _exact_rotated(x, weight, cos, sin, case):
    """Norm and rotation of one head-major tensor as a complex product of each pair with its angle."""
    y = x / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + EPS) * weight
    a, b, rest = _halves(y, case["rot"], case["interleaved"])
    z = torch.complex(a, b) * torch.complex(cos, sin)[:, None]
    return _joined(z.real, z.imag, rest, case["interleaved"])


def _exact_pam_sum(a, b, dim):
    fa, ea = torch.frexp(a.abs())
    fb, eb = torch.frexp(b.abs())
    frac = (2 * fa - 1) + (2 * fb - 1)
    value = torch.ldexp(torch.where(frac >= 1, 2 * frac, 1 + frac), ea + eb - 2)
    return (value * a.sign() * b.sign()).sum(dim)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "attention":
        return _exact_attention(case, s)
    cos, sin = (s[name].double()[s["positions"].long()] for name in ("cos", "sin"))
    if case["kind"] == "norm_rope" and case["grad"]:
        out = []
        for name in "qk":
            x, w = (t.double().detach().requires_grad_() for t in (s[name], s[name + "_weight"]))
            y = _exact_rotated(x, w, cos, sin, case)
            out.append(torch.autograd.grad(y, (x, w), s["d" + name].double()))
        return out[0][0], out[1][0], out[0][1], out[1][1]
    q, k = (_exact_rotated(s[name].double(), s[name + "_weight"].double(), cos, sin, case) for name in "qk")
    if case["kind"] == "norm_rope":
        return q, k
    caches = []
    for name, new in (("k_cache", k), ("v_cache", s["v"].double())):
        cache = s[name].double()
        cache.view(-1, case["hk"], case["d"])[s["slots"]] = new
        caches.append(cache)
    return (q, *caches)


def _exact_attention(case, s):
    hq, hk, d, page = case["hq"], case["hk"], case["d"], case["page"]
    g = hq // hk
    new, kv = _lengths(case)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    first = 0
    for b, (n, length) in enumerate(zip(new, kv)):
        at = torch.arange(length, device=DEV)
        page_of, slot = s["table"][b].long()[at // page], at % page
        k, v = (s[c][page_of, slot].double() for c in ("k_cache", "v_cache"))                  # key hk d
        some = max(1, (1 << 27) // (length * hq * d))
        for r in range(0, n, some):
            rows = torch.arange(r, min(n, r + some), device=DEV)
            q = s["q"][first + rows].double().view(-1, hk, g, 1, d)
            scores = _exact_pam_sum(q, k.transpose(0, 1)[:, None], -1) / math.sqrt(d)          # row hk g key
            scores = scores.masked_fill(~_visible(case, n, length, rows[:, None], at)[:, None, None], -math.inf)
            p = scores.softmax(-1).unsqueeze(-1)
            out[first + rows] = _exact_pam_sum(p, v.transpose(0, 1)[:, None], -2).view(-1, hq, d)
        first += n
    return out


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    size = {"float32": 4, "bfloat16": 2}
    hq, hk, d = case["hq"], case["hk"], case["d"]
    act = size[case["dtype"]]
    if case["kind"] == "attention":
        new, kv = _lengths(case)
        pairs = keys = 0
        for n, length in zip(new, kv):
            lo = [max(0, length - n + i + 1 - case["window"]) if case["window"] else 0 for i in range(n)]
            pairs += sum(length - n + i + 1 - a for i, a in enumerate(lo))
            keys += length - lo[0]
        # Keys and values once, queries in their type, float32 outputs; a PAM and an addition for each term.
        return {"bytes": keys * hk * 2 * d * size[case["cache"]] + sum(new) * hq * d * (act + 4),
                "flops": 4 * pairs * hq * d}
    t = case["tokens"]
    table = min(t, 4096) * case["rot"] * 4
    if case["kind"] == "append":
        moved = t * d * ((2 * hq + 2 * hk) * act + 2 * hk * size[case["cache"]])
        return {"bytes": moved + table + 12 * t, "flops": 10 * t * (hq + hk) * d}
    moved = t * (hq + hk) * d * act * (3 if case["grad"] else 2)
    return {"bytes": moved + table + 4 * t, "flops": (20 if case["grad"] else 10) * t * (hq + hk) * d}
