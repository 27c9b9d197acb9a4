"""Drafted trees in 64 bits on the CPU, from their definition: what a node attends, its attention, the accepted path."""
from __future__ import annotations

import random

import numpy as np
import torch

UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}      # half a step: what one rounding is off at most, relative
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def random_tree(n: int, seed: int, width: int = 0):
    """Parents of n nodes: width 0 a random tree, 1 a chain, otherwise at most that many children a node."""
    r = random.Random(seed)
    if width == 1:
        return [i - 1 for i in range(n)]
    if width == 0:
        return [-1] * min(n, 1) + [r.randrange(i) for i in range(1, n)]
    return [-1] * min(n, 1) + [(i - 1) // width for i in range(1, n)]


def ancestors(parents, x):
    """x, its parent, ..., the root."""
    out = []
    while x >= 0:
        out.append(x)
        x = parents[x]
    return out


def depth(parents, x):
    return len(ancestors(parents, x)) - 1


def attention(q, k_ctx, v_ctx, k, v, parents):
    """One sequence, float64: q [n, hq, d], k_ctx / v_ctx [len, hkv, d], k / v [n, hkv, d].  Returns (o, a, s): the result [n, hq, d], the
    weighted sum of |v| and the largest sum |q_i k_i| / sqrt(d) of a row, which the error bounds are made of."""
    n, hq, d = q.shape
    hkv, c = k.shape[1], k_ctx.shape[0]
    o, a, s = np.zeros((n, hq, d)), np.zeros((n, hq, d)), np.zeros((n, hq, 1))
    for x in range(n):
        at = list(range(c)) + [c + y for y in ancestors(parents, x)]
        keys, values = np.concatenate([k_ctx, k])[at], np.concatenate([v_ctx, v])[at]
        for h in range(hq):
            kk, vv = keys[:, h // (hq // hkv)], values[:, h // (hq // hkv)]
            score = kk @ q[x, h] / np.sqrt(d)
            w = np.exp(score - score.max())
            w /= w.sum()
            o[x, h], a[x, h] = w @ vv, w @ np.abs(vv)
            s[x, h] = (np.abs(kk) @ np.abs(q[x, h])).max() / np.sqrt(d)
    return o, a, s


def attention_bound(o, a, s, dtype, d, positions):
    """How far a row may be off: the result's rounding; for 16 bits the rounding of every weight in front of the second product; the
    32-bit arithmetic, (d + 8) roundings a score (in relation to the sum of its products' magnitudes, twice: numerator and sum) and one for
    every position that is added up, on the weighted magnitudes."""
    u = UNIT[dtype]
    f32 = UNIT["f32"] * (2 * (d + 8) * s + 2 * positions + 64)
    return u * np.abs(o) + (u if dtype != "f32" else 0.0) * a + f32 * a * (1 + u)


def accept(parents, draft, chosen):
    """(path, tokens) of one sequence."""
    if not parents:
        return [], []
    path = [0]
    while True:
        fits = [x for x in range(len(parents)) if parents[x] == path[-1] and draft[x] == chosen[path[-1]]]
        if not fits:
            return path, [chosen[x] for x in path]
        path.append(fits[0])
