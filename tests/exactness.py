"""What separates 32-bit arithmetic from 16-bit arithmetic at any width: the RMS of the error in relation to the RMS of the result.

Worst cases grow with the number of terms, typical errors with its root: every one of n additions is off by at most half a step, 2^-24 of the running
sum, which is no larger than the result's own scale, in directions of their own.  A value rounded to fp16 is off by 2^-11 / sqrt(12) and more of itself,
and so is a sum over such values, whatever their number."""
from __future__ import annotations

import numpy as np

from tests import tree_reference as tr

STEP = 2.0 ** -24


def rms(x):
    return float(np.sqrt(np.mean(np.square(x))))


def product_limit(n_in: int) -> float:
    """n_in additions, twice over; 16 roundings for scales, parts, joining and, of a head, the norm."""
    return STEP * (16 + 2 * np.sqrt(n_in))


def attention_limit(d: int, s: float, positions: int) -> float:
    """A score is a chain of d additions in relation to s, its products' magnitudes, and shifts its weight by that; as many additions as positions; 16
    roundings for the exponential, rescaling and the quotient.  Twice what is expected of the chains."""
    return STEP * (16 + np.sqrt(d) * s + np.sqrt(positions))


# fp32 products: shapes of every form of the kernel, split contractions and operands in and out of LDS among them
PRODUCTS = [(130, 64, 32, (1, 20)), (2304, 208, 64, (2, 11, 33, 70)), (8192, 96, 128, (1, 4, 9, 17, 32)), (8400, 206, 32, (1, 9, 24)), (8400, 206, 64, (33,)),
            (300, 4104, 128, (1, 8, 30)), (2000, 8200, 64, (1, 4, 12)), (384, 66000, 128, (9, 20))]
HEADS = [(1024, 4104, 64, 24), (8448, 1000, 64, 21), (512, 9000, 32, 40)]
# (query heads, kv heads, d, contexts, nodes): whole contexts and such that are cut into runs
ATTENTION = [(8, 2, 64, [40], [5]), (4, 1, 64, [20, 3], [100, 256]), (2, 1, 128, [3000], [2]), (4, 1, 64, [2100, 5, 1000], [13, 16, 2]), (8, 1, 128, [1500, 0, 700], [26, 20, 30]),
             (2, 1, 64, [4000], [1]), (16, 4, 128, [2048, 1900], [8, 5]), (8, 8, 64, [600] * 4, [8] * 4)]


def attention_rows(seq_inputs, lens, trees):
    """seq_inputs: per sequence (q, k_ctx, v_ctx, k, v) in float64.  (result, largest product magnitude of a score) of all rows."""
    found = [tr.attention(*x, t) for x, t in zip(seq_inputs, trees) if t]
    return np.concatenate([f[0] for f in found]), max(float(f[2].max()) for f in found)
