"""Linear layers whose sums are taken in parts: one of each kernel form that the
planner chooses for them, as (m, k, n, form)."""
from __future__ import annotations

# form: tile, k-groups, K split, whole tiles among the launch's, launches of the tiled kernel
CASES = [
    (38, 61010, 2303, ((64, 64), 1, True, False, 1)), (150, 1061, 14705, ((64, 64), 1, True, True, 1)),
    (37, 34179, 3995, ((64, 64), 4, True, False, 1)), (166, 4485, 10673, ((64, 64), 4, False, True, 1)),
    (2136, 64546, 38, ((128, 64), 1, True, False, 1)), (39381, 1048, 35, ((128, 64), 1, True, True, 1)),
    (25164, 1061, 266, ((128, 64), 1, False, True, 1)), (3782, 33153, 34, ((128, 64), 2, True, False, 1)),
    (20225, 16787, 391, ((128, 64), 2, True, False, 2)), (2708, 2150, 1421, ((128, 64), 2, False, True, 1)),
    (65, 68028, 1106, ((128, 128), 1, True, False, 1)), (18030, 69289, 77, ((128, 128), 1, True, False, 2)),
    (135, 1041, 16413, ((128, 128), 1, True, True, 1)), (4493, 3198, 4538, ((128, 128), 1, True, True, 2)),
    (24509, 1095, 521, ((128, 128), 1, False, True, 1)), (16640, 1040, 8192, ((128, 128), 1, False, True, 2))]
