"""A small decoder whose products are PAM: trained with whole sequences, answering
from a paged key/value cache.

    python examples/decoder.py [--steps N] [--new TOKENS] [--state-bits 8]

Training runs the linear layers through ``PAMLinear``, the activation and the
residual stream in their products' launches, queries and keys through
``pam_norm_rope`` and the attention through ``pam_matmul`` with a softmax between,
under autograd; ``AdamW`` steps over all parameters at once.  Answering runs the same weights over ``append_kv`` and
``paged_attention``: the prompts in chunks of different lengths at once, then one
token a sequence.  The two are the same function, so the logits agree to
float32 rounding; the example checks that and says how far they are apart.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch
from torch import nn

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2305_17190_amd as pam  # noqa: E402
from paper_2305_17190_amd.autograd import PAMLinear, pam_matmul, pam_norm_rope  # noqa: E402
from paper_2305_17190_amd.optim import AdamW  # noqa: E402


class Cache:
    """The pages of all layers and who holds which: keys and values of a layer are
    (pages, page, heads, d); a sequence owns the pages in its row of the table."""

    def __init__(self, layers, sequences, tokens, heads, d, page=16, dtype=torch.float32, device="cuda"):
        self.page = page
        each = -(-tokens // page)
        shape = (layers, sequences * each, page, heads, d)
        self.k, self.v = (torch.empty(shape, dtype=dtype, device=device) for _ in "kv")
        # Pages in no order, as a pool that has been in use for a while gives them out.
        self.table = torch.randperm(sequences * each, device=device).to(torch.int32).view(sequences, each)
        self.lens = [0] * sequences

    def extend(self, counts):
        """Room for counts[b] new tokens of each sequence: their positions and slots,
        the lengths with them, and where each sequence's tokens start."""
        seq = torch.tensor([b for b, n in enumerate(counts) for _ in range(n)])
        pos = torch.tensor([self.lens[b] + i for b, n in enumerate(counts) for i in range(n)])
        self.lens = [have + n for have, n in zip(self.lens, counts)]
        device = self.table.device
        pos, seq = pos.to(device), seq.to(device)
        slots = self.table[seq, pos // self.page].long() * self.page + pos % self.page
        starts = torch.tensor([0] + counts).cumsum(0)
        return (pos.to(torch.int32), slots, torch.tensor(self.lens, dtype=torch.int32, device=device),
                starts.to(torch.int32).to(device))


class Layer(nn.Module):
    def __init__(self, width, heads, kv_heads, d, hidden, device):
        super().__init__()
        self.heads, self.kv_heads, self.d = heads, kv_heads, d
        self.norm1, self.norm2 = (nn.RMSNorm(width, device=device) for _ in range(2))
        self.qkv = PAMLinear(width, (heads + 2 * kv_heads) * d, bias=False, device=device)
        self.out = PAMLinear(heads * d, width, bias=False, device=device)
        self.up = PAMLinear(width, hidden, device=device, activation="relu")
        self.down = PAMLinear(hidden, width, device=device)
        self.q_weight, self.k_weight = (nn.Parameter(torch.ones(d, device=device)) for _ in range(2))

    def heads_of(self, x):
        """Queries, keys and values as views of one projection."""
        qkv = self.qkv(self.norm1(x)).view(-1, self.heads + 2 * self.kv_heads, self.d)
        return qkv.split((self.heads, self.kv_heads, self.kv_heads), 1)

    def rest(self, x, attended):
        x = self.out(attended.reshape(x.shape[0], -1), residual=x)
        return self.down(self.up(self.norm2(x)), residual=x)

    def whole(self, x, batch, positions, cos, sin):
        """All tokens of `batch` sequences of one length, differentiable."""
        q, k, v = self.heads_of(x)
        q, k = pam_norm_rope(q, k, positions, cos, sin, self.q_weight, self.k_weight)
        n, g = x.shape[0] // batch, self.heads // self.kv_heads

        def by_head(t, repeat):
            t = t.reshape(batch, n, -1, self.d).transpose(1, 2)
            return t.repeat_interleave(repeat, 1).reshape(-1, n, self.d)

        s = pam_matmul(by_head(q, 1), by_head(k, g).transpose(1, 2)) / math.sqrt(self.d)
        s = s.masked_fill(torch.ones(n, n, dtype=torch.bool, device=s.device).triu(1), -math.inf)
        o = pam_matmul(torch.softmax(s, -1), by_head(v, g))
        return self.rest(x, o.view(batch, self.heads, n, self.d).transpose(1, 2).reshape(x.shape[0], -1))

    def cached(self, x, k_cache, v_cache, table, positions, slots, lens, starts, max_q, max_kv, cos, sin):
        """New tokens of all sequences, over the cache."""
        q, k, v = self.heads_of(x)
        q = pam.append_kv(k, v, k_cache, v_cache, slots, positions, cos, sin, self.k_weight.detach(), q,
                          self.q_weight.detach())
        return self.rest(x, pam.paged_attention(q, k_cache, v_cache, table, lens, starts, max_q, max_kv))


class Decoder(nn.Module):
    def __init__(self, vocabulary=64, width=128, layers=2, heads=4, kv_heads=2, d=32, positions=256, device="cuda"):
        super().__init__()
        self.embed = nn.Embedding(vocabulary, width, device=device)
        self.layers = nn.ModuleList(Layer(width, heads, kv_heads, d, 4 * width, device) for _ in range(layers))
        self.norm = nn.RMSNorm(width, device=device)
        self.head = PAMLinear(width, vocabulary, bias=False, device=device)
        angle = torch.arange(positions)[:, None] * 10000.0 ** (-torch.arange(0, d, 2) / d)
        self.register_buffer("cos", angle.cos().to(device))
        self.register_buffer("sin", angle.sin().to(device))
        self.kv_heads, self.d = kv_heads, d

    def forward(self, tokens):
        """Logits of whole sequences (batch, n), differentiable."""
        batch, n = tokens.shape
        positions = torch.arange(n, dtype=torch.int32, device=tokens.device).repeat(batch)
        x = self.embed(tokens.reshape(-1))
        for layer in self.layers:
            x = layer.whole(x, batch, positions, self.cos, self.sin)
        return self.head(self.norm(x)).view(batch, n, -1)

    @torch.no_grad()
    def step(self, tokens, cache, counts):
        """Logits of counts[b] new tokens of each sequence, which join the cache."""
        positions, slots, lens, starts = cache.extend(counts)
        x = self.embed(tokens)
        for i, layer in enumerate(self.layers):
            x = layer.cached(x, cache.k[i], cache.v[i], cache.table, positions, slots, lens, starts, max(counts),
                             max(cache.lens), self.cos, self.sin)
        return self.head(self.norm(x))


def batch_of(rng, size, half, vocabulary):
    """Sequences that say the same random tokens twice."""
    first = torch.randint(vocabulary, (size, half), generator=rng)
    return torch.cat((first, first), 1).cuda()


def train(model, steps, half=12, size=32, state_bits=32):
    rng = torch.Generator().manual_seed(0)
    optimizer = AdamW(model.parameters(), lr=2e-3, weight_decay=0.01, state_bits=state_bits)
    losses = []
    for _ in range(steps):
        tokens = batch_of(rng, size, half, model.embed.num_embeddings)
        logits = model(tokens)[:, half - 1:-1]
        loss = nn.functional.cross_entropy(logits.reshape(-1, logits.shape[-1]), tokens[:, half:].reshape(-1))
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(float(loss.detach()))
    return losses


@torch.no_grad()
def answer(model, prompts, new, chunk=7, dtype=torch.float32):
    """Greedy continuations of prompts of different lengths: each prompt in chunks,
    then token by token, all sequences at once.  Also the logits each new token was
    chosen from."""
    cache = Cache(len(model.layers), len(prompts), max(map(len, prompts)) + new, model.kv_heads, model.d, dtype=dtype)
    left = [list(p) for p in prompts]
    last = [None] * len(prompts)
    while any(left):
        counts = [min(chunk, len(p)) for p in left]
        logits = model.step(torch.tensor([t for p, n in zip(left, counts) for t in p[:n]], device="cuda"), cache, counts)
        at = 0
        for b, n in enumerate(counts):
            at += n
            if n:
                last[b] = logits[at - 1]
            left[b] = left[b][n:]
    chosen, seen = [], []
    logits = torch.stack(last)
    for i in range(new):
        seen.append(logits)
        token = logits.argmax(-1)
        chosen.append(token)
        if i + 1 < new:
            logits = model.step(token, cache, [1] * len(prompts))
    return torch.stack(chosen, 1), torch.stack(seen, 1)


def main(argv=None):
    parser = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    parser.add_argument("--steps", type=int, default=300)
    parser.add_argument("--new", type=int, default=12)
    parser.add_argument("--state-bits", type=int, default=32, choices=(8, 32))
    args = parser.parse_args(argv)
    torch.manual_seed(0)
    model = Decoder()
    losses = train(model, args.steps, state_bits=args.state_bits)
    if losses:
        print(f"loss {losses[0]:.3f} -> {losses[-1]:.3f} in {len(losses)} steps")
    tokens = batch_of(torch.Generator().manual_seed(1), 4, 12, 64)
    prompts = [t[:12 + b].tolist() for b, t in enumerate(tokens)]
    got, seen = answer(model, prompts, args.new)
    # The same sequences, whole.
    apart = 0.0
    for b, prompt in enumerate(prompts):
        text = torch.tensor([prompt + got[b].tolist()], device="cuda")
        with torch.no_grad():
            whole = model(text)[0, len(prompt) - 1:-1]
        apart = max(apart, float((whole - seen[b]).abs().max() / whole.abs().max()))
        print(f"prompt {prompt} -> {got[b].tolist()}")
    print(f"logits from the cache and from whole sequences differ by at most {apart:.1e} of the largest")
    return losses, apart


if __name__ == "__main__":
    main()
