"""Windowed rows and eviction in 64 bits on the CPU, from their definition: what a row attends, its attention, the weights' sums, the slots that stay."""
from __future__ import annotations

import numpy as np

from oracle import stage_oracle as so
from tests import tree_reference as tr


def visible(p, window, sinks):
    """Slots that the row at slot p attends; window None: all of them."""
    w = window if window is not None else p + 1
    return [j for j in range(p + 1) if p - j < w or j < sinks]


def attention(q, k_ctx, v_ctx, k, v, window, sinks):
    """One sequence, float64: q [n, hq, d], k_ctx / v_ctx [len, hkv, d], k / v [n, hkv, d].  Returns (o, a, s, w, e): the result, the weighted sum of |v|,
    the largest sum |q_i k_i| / sqrt(d) of a row, the weights' sums [hkv, len + n] and the same sums with each weight times its row's s."""
    n, hq, d = q.shape
    hkv, c = k_ctx.shape[1], k_ctx.shape[0]
    o, a, s = np.zeros((n, hq, d)), np.zeros((n, hq, d)), np.zeros((n, hq, 1))
    sums, scaled = np.zeros((hkv, c + n)), np.zeros((hkv, c + n))
    keys, values = np.concatenate([k_ctx, k]), np.concatenate([v_ctx, v])
    for x in range(n):
        at = visible(c + x, window, sinks)
        for h in range(hq):
            g = h // (hq // hkv)
            kk, vv = keys[at, g], values[at, g]
            score = kk @ q[x, h] / np.sqrt(d)
            w = np.exp(score - score.max())
            w /= w.sum()
            o[x, h], a[x, h] = w @ vv, w @ np.abs(vv)
            s[x, h] = (np.abs(kk) @ np.abs(q[x, h])).max() / np.sqrt(d)
            sums[g, at] += w
            scaled[g, at] += w * s[x, h]
    return o, a, s, sums, scaled


def weights_bound(sums, scaled, before, d, positions, terms):
    """How far an accumulated weight may be off: of every weight the score's (d + 8) roundings in relation to s, once for it and once for the sum it is
    divided by, that sum's additions, 64 for exponential, quotient and joining; and one rounding for each of the terms that are added up, on what there is at the end."""
    return tr.UNIT["f32"] * (2 * (d + 8) * scaled + (2 * positions + 64) * sums + (terms + 8) * (sums + np.abs(before)))


def chosen(n, keep, sinks, recent, weights=None):
    """The slots of a context of n that stay, in order."""
    if n <= keep:
        return list(range(n))
    middle = list(range(sinks, n - recent))
    if weights is None:
        middle = middle[::-1]
    else:
        key = [(-np.inf if np.isnan(w) else w, 0 if np.isnan(w) else 1) for w in weights]       # NaN below everything, -inf among it
        middle = sorted(middle, key=lambda i: (-key[i][0], -key[i][1], i))
    return sorted(list(range(sinks)) + middle[:keep - sinks - recent] + list(range(n - recent, n)))


def turned_back(k, distance, theta):
    """Keys [n, hkv, d] whose positions fall by distance[n]."""
    return so.rope(np.asarray(k, dtype=np.float64), -np.asarray(distance), theta)


class WindowOracle(so.OracleStage):
    """The stage whose rows attend a window and the first positions; gathers the weights' sums per layer and sequence."""
    window, sinks = None, 0

    def attn_partial(self, layer, cache, h, seq_of_row):
        W = self.layers[layer]
        T = h.shape[0]
        n = so.rmsnorm(h, W["g_attn"], self.eps)
        q, k, v = ((n @ W[x]).reshape(T, -1, self.d) for x in ("wq", "wk", "wv"))
        o = np.zeros_like(q)
        for s in sorted(set(seq_of_row)):
            rows = [i for i, x in enumerate(seq_of_row) if x == s]
            first = cache.length(layer, s)
            pos = np.arange(first, first + len(rows))
            qs, ks = so.rope(q[rows], pos, self.theta), so.rope(k[rows], pos, self.theta)
            o[rows], _, _, sums, _ = attention(qs, cache.k[layer][s], cache.v[layer][s], ks, v[rows], self.window, self.sinks)
            cache.append(layer, s, ks, v[rows])
            before = self.gathered.setdefault((layer, s), np.zeros((self.hkv_l, 0)))
            full = np.zeros((self.hkv_l, first + len(rows)))
            full[:, :before.shape[1]] = before
            self.gathered[layer, s] = full + sums
        return o.reshape(T, -1) @ W["wo"]


def window_oracle(cfg, weights, window, sinks, rank=0):
    from tests.helpers import ORDER
    st = WindowOracle(cfg.hidden, cfg.n_heads, cfg.n_kv_heads, cfg.ffn, cfg.n_layers, cfg.tp_degree, rank, cfg.rms_eps, cfg.rope_theta)
    st.window, st.sinks, st.gathered = window, sinks, {}
    for layer in range(cfg.n_layers):
        st.load_layer(layer, *[weights[layer][k] for k in ORDER])
    return st
