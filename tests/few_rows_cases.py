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

# Head sizes by the lanes a key takes: (d, bfloat16 cache), whole and with a part of
# the last lanes' 16 bytes past the head's end.
HEADS = [(16, False), (8, True), (32, False), (64, True), (56, True), (64, False), (48, False), (128, True), (72, True),
         (128, False), (96, False), (256, True), (200, True), (256, False), (136, False)]
# (new tokens, query heads a key head): every count of rows a unit can have, 5 and 7
# among those that a unit of the next one takes.
ROWS = [(1, 1), (2, 1), (1, 3), (2, 2), (1, 5), (3, 2), (1, 7), (2, 4)]


def every_kernel(fine, layouts):
    """One case for each lane count, type and count of rows in both forms; every
    second with a window, every third without the causal mask."""
    return [Case(form, fine, sequences(new, lengths), pages[i % 3], heads, group, d, bf16, reach[i % 2], i % 3 != 1,
                 (0, 50)[i // 2 % 2])
            for form, heads, lengths, pages, reach in layouts
            for i, (d, bf16, new, group) in enumerate((d, bf16, new, group) for d, bf16 in HEADS for new, group in ROWS)]


FINE = every_kernel(True, (("whole", 1, [250, 77, 16, 3], (16, 1, 32), (0, 0)), ("split", 2, [300, 77], (16, 1, 48), (0, 3000))))
# The far bounds give splits of 256 and of 1024 keys.
WIDE = every_kernel(False, (("whole", 3, SHORT, (16, 1, 32), (0, 0)), ("split", 2, LONG, (16, 1, 48), (4500, 140000))))
# Many units whose scores fit half of LDS take one launch past 256 keys as well.
WIDE += [Case("whole", False, sequences(1, [1000, 3, 0, 64] + SHORT * 2), 16, 3, group, d, bf16)
         for d, bf16 in ((64, False), (128, True)) for group in (1, 4)]

# Where it goes wrong most easily, in one and in three launches, float32 and bfloat16.
CORNERS = [case for case in WIDE if case.form == "split" and case.d in (64, 128) and max(case.counts) * case.group in (3, 8)]
CORNERS += [case for case in WIDE if case.form == "whole" and case.d in (64, 128) and max(case.counts) * case.group in (2, 7)]
