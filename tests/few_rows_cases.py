"""Calls of PAM attention with few rows a key head, by the form they take:
"whole" (one launch) or "split" (scores, values, join), in waves of 16 keys
("fine") or of 64.  The library decides by the bounds ``max_q`` and ``max_kv``,
so a table that could reach far takes short sequences to any of them.
``test_attention_forms.py`` holds every case to its form on the CPU."""
from __future__ import annotations

import numpy as np

import attention_util as au


class Case:
    """`seqs`: (new tokens, keys) of each sequence; reach: keys of the table, at
    least those of the longest sequence; rows, lanes: what the kernel works in."""

    def __init__(self, form, fine, seqs, page, heads, group, d, bf16, reach=0, causal=True, window=0):
        self.form, self.fine, self.seqs, self.page = form, fine, seqs, page
        self.heads, self.group, self.d, self.bf16 = heads, group, d, bf16
        self.causal, self.window = causal, window
        self.counts = [n for n, _ in seqs]
        self.kv_lens = [kv for _, kv in seqs]
        self.width = -(-max(reach, max(self.kv_lens), 1) // page)

    def __repr__(self):
        return (f"{self.form}-{'fine' if self.fine else 'wide'}-{len(self.seqs)}x{max(self.counts)}-page{self.page}-"
                f"{self.heads}x{self.group}x{self.d}-{'bf16' if self.bf16 else 'f32'}-reach{self.width * self.page}-"
                f"{'causal' if self.causal else 'all'}-{self.window}")

    def cache(self, rng, spare=2):
        cache = au.Paged(rng, self.kv_lens, self.page, self.heads, self.d, self.bf16, spare)
        wide = np.full((len(self.seqs), self.width), -1, np.int32)
        wide[:, :cache.table.shape[1]] = cache.table
        cache.table = wide
        return cache

    def queries(self, rng):
        return rng.standard_normal((sum(self.counts), self.heads * self.group, self.d)).astype(np.float32) * 2

    def kw(self):
        return dict(causal=self.causal, window=self.window)


def sequences(new, lengths):
    """`new` tokens at most, fewer in every third sequence, more than its keys in none."""
    return [(max(new - (i % 3 == 2), 1), max(kv, new) if kv else 0) for i, kv in enumerate(lengths)]


SHORT = [256, 0, 1, 63, 64, 65, 130, 17] + [3 + 7 * i % 61 for i in range(36)]     # 44 sequences: 132 units of 3 heads
LONG = [700, 64, 0, 333]

# What lies outside the sequences' own keys.
OUTSIDE = [
    Case(form, fine, sequences(new, lengths), 16, heads, 2, 64, bf16, reach)
    for new in (1, 3) for bf16 in (False, True)
    for form, fine, lengths, heads, reach in (
        ("whole", True, [250, 77, 16, 3], 1, 0), ("whole", False, SHORT, 3, 0), ("split", True, [300, 77], 2, 0),
        ("split", False, LONG, 2, 4500))
]

# Bounds whose workspace passes a round's: the units take turns in it.
ROUNDS = [
    Case("split", False, sequences(1, LONG), 16, 2, 8, 64, True, 4000000),
    Case("split", False, sequences(2, [300, 5, 1200]), 1024, 3, 2, 128, False, 9000000, window=50),
]
