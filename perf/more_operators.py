"""Operators of long requests in a cache of bounded size, as cases that can be timed and checked.

  kind "window"  attention of new rows over the KV cache with a sliding window and a few first positions that stay visible: the rows' keys
                 and values join the cache behind each sequence's context (`KVCache.window_attention`); with `weights` every position's
                 attention weights, summed over the rows and the query heads of its kv head, are added to an accumulator as well
  kind "evict"   a context shrinks to `keep` slots per layer and kv head (`KVCache.evict`): the first ones, the most recent ones and of the others the
                 heaviest (or, without weights, the newest) move to a cache of that size, their keys possibly rotated to their new positions;
                 behind it the next step's attention of one row per sequence over what is left, in every layer

Contexts and new rows of a batch are ragged: `lo` .. `hi` positions and `rows_lo` .. `rows_hi` rows, spread evenly over these ranges in a
fixed order, so that a case's work does not depend on the seed.  `window` 0: none, every earlier position is visible.
"""
from __future__ import annotations

import math

import torch

own = False

TORCH_TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
THETA = 10000.0
WIDE = 1 << 30         # a window that nothing reaches


def _window(dtype, batch, heads, kv_heads, d, lo, hi, rows_lo, rows_hi, window, sinks, weights):
    return dict(kind="window", dtype=dtype, batch=batch, heads=heads, kv_heads=kv_heads, d=d, lo=lo, hi=hi, rows_lo=rows_lo, rows_hi=rows_hi,
                window=window, sinks=sinks, weights=weights)


def _evict(dtype, layers, batch, heads, kv_heads, d, lo, hi, keep, sinks, recent, weights, rotate):
    return dict(kind="evict", dtype=dtype, layers=layers, batch=batch, heads=heads, kv_heads=kv_heads, d=d, lo=lo, hi=hi, keep=keep, sinks=sinks,
                recent=recent, weights=weights, rotate=rotate)


def listed():
    return [
        # one token of a tiny full-precision model: the smallest call, latency counts
        dict(_window("f32", 1, 8, 2, 64, 40, 40, 1, 1, 24, 4, False), name="window_f32_tiny"),
        # one interactive request on the narrowest shard of the 70B shape, far into a long conversation
        dict(_window("bf16", 1, 8, 1, 128, 4000, 4000, 1, 1, 1024, 4, False), name="window_b1"),
        # a small fp16 model with 64-wide heads: seven ragged requests, from one new row to sixteen, contexts shorter and longer than the window
        dict(_window("f16", 7, 32, 8, 64, 11, 330, 1, 16, 100, 3, False), name="window_f16_ragged"),
        # a batched step of the full-width layer that gathers weights for a later eviction
        dict(_window("bf16", 32, 64, 8, 128, 240, 4027, 1, 1, 2048, 4, True), name="window_b32_weights"),
        # full precision, odd sizes: three short prompts behind short contexts, a check of a 16-bit deployment
        dict(_window("f32", 3, 16, 4, 128, 0, 203, 90, 301, 128, 1, True), name="window_f32_prompt"),
        # a whole prompt of the full-width layer under a window
        dict(_window("bf16", 1, 64, 8, 128, 0, 0, 4096, 4096, 1024, 4, False), name="window_prompt"),
        # chunks of eight long prompts without a window, gathering weights
        dict(_window("bf16", 8, 32, 4, 128, 1000, 3500, 512, 512, 0, 0, True), name="window_chunks_weights"),
        # one short fp16 request of a small model that is over its budget by a little
        dict(_evict("f16", 1, 1, 32, 8, 64, 333, 333, 256, 4, 32, True, False), name="evict_small"),
        # full precision, odd sizes, some contexts within the budget already
        dict(_evict("f32", 2, 5, 16, 4, 64, 100, 700, 301, 2, 50, True, True), name="evict_f32_odd"),
        # sixteen endless streams on the narrowest shard: first and most recent positions, keys rotated to their new places
        dict(_evict("bf16", 2, 16, 8, 1, 128, 4000, 4000, 2048, 4, 2044, False, True), name="evict_stream"),
        # prompts of the full-width layers compressed to the positions that were attended most
        dict(_evict("bf16", 2, 8, 64, 8, 128, 1500, 4000, 1024, 4, 64, True, False), name="evict_heavy"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["window", "window", "window", "evict", "evict"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f16", "f16", "f32"])
    d, group, kv_heads = rng.choice([64, 128]), rng.choice([1, 2, 3, 4, 8, 8, 16]), rng.choice([1, 2, 4, 8])
    while group * kv_heads * d % 128:
        kv_heads *= 2
    heads, hi, weights = group * kv_heads, _log_int(rng, 1, 4096), rng.random() < 0.5
    lo, sinks = int(hi * rng.uniform(0.0, 1.0)), rng.choice([0, 1, 4, 4, rng.randrange(0, 70)])
    if kind == "evict":
        layers, batch = rng.choice([1, 1, 2, 3]), _log_int(rng, 1, 16)
        while layers * batch * kv_heads * hi > 2 * 8 * 8 * 4000:
            batch = (batch + 1) // 2
            hi, lo = (hi, lo) if batch > 1 else (hi // 2, lo // 2)
        keep = max(1, int(hi * rng.uniform(0.1, 1.1)))
        sinks = min(sinks, keep)
        recent = int((keep - sinks) * rng.choice([0.0, 0.1, 0.5, 1.0]))
        return _evict(dtype, layers, batch, heads, kv_heads, d, max(1, lo), max(1, hi), keep, sinks, recent, weights, rng.random() < 0.5)
    shape = rng.choice(["step", "step", "chunk", "prompt"])
    rows = 1 if shape == "step" else _log_int(rng, 2, 64) if shape == "chunk" else _log_int(rng, 64, 4096)
    rows_lo = 1 if shape == "step" else max(0 if shape == "chunk" else 1, int(rows * rng.uniform(0.1, 1.0)))
    if shape == "prompt" and rng.random() < 0.5:
        lo, hi = 0, 0
    window = 0 if rng.random() < 0.25 else _log_int(rng, 1, 2048)
    batch = _log_int(rng, 1, 32)
    most = 8 * 32 * 512 * 2250 // (8 if dtype == "f32" else 1)      # (sequence, head, row, position): the largest listed case
    while batch * heads * rows * (hi + rows) > most or batch * kv_heads * (hi + rows) > 32 * 8 * 2100:
        if batch > 1:
            batch = (batch + 1) // 2
        else:
            rows, rows_lo = max(1, rows // 2), max(1, rows_lo // 2)
            hi, lo = hi // 2, lo // 2
    return _window(dtype, batch, heads, kv_heads, d, lo, hi, min(rows_lo, rows), rows, window, sinks, weights)


def _spread(n, lo, hi, step):
    return [lo + int(round((hi - lo) * (((i + 1) * step) % 1.0))) for i in range(n)]


def _contexts(case):
    return _spread(case["batch"], case["lo"], case["hi"], 0.6180339887498949)


def _rows(case):
    if case["kind"] == "evict":
        return [1] * case["batch"]
    counts = _spread(case["batch"], case["rows_lo"], case["rows_hi"], 0.41421356237309515)
    return counts if sum(counts) else [1] + counts[1:]


# ---- inputs -------------------------------------------------------------------------------------------------------
def _generator(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1009 + salt)
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _gathered(g, *shape):
    """Accumulated weights: a few heavy positions, many light ones, and some that were never seen (equal: the lowest slot goes first)."""
    w = torch.exp(1.5 * _normal(g, *shape) - 2)
    return w * (torch.rand(shape, generator=g, device="cuda") >= 0.15)


def _drawn(case, seed):
    """Cache [layers, batch, slots, kv heads, d], the new rows of every layer, the accumulated weights [layers, batch, kv heads, slots]."""
    td, hkv, d = TORCH_TYPE[case["dtype"]], case["kv_heads"], case["d"]
    layers, lens, counts = case.get("layers", 1), _contexts(case), _rows(case)
    size = max(n + c for n, c in zip(lens, counts))
    g = _generator(seed, 1)
    kc, vc = [_normal(g, layers, case["batch"], size, hkv, d).to(td) for _ in range(2)]
    q, k, v = [_normal(g, layers, sum(counts), heads, d).to(td) for heads in (case["heads"], hkv, hkv)]
    weights = _gathered(g, layers, case["batch"], hkv, size) if case["weights"] else None
    if weights is not None and case["kind"] == "window":
        weights = weights[0] * (torch.arange(size, device="cuda") < torch.tensor(lens, device="cuda")[:, None, None])
    return kc, vc, q, k, v, weights


def prepare(case, seed):
    kc, vc, q, k, v, weights = _drawn(case, seed)
    lens, counts = _contexts(case), _rows(case)
    state = {"case": dict(case), "q": q, "k": k, "v": v, "weights": weights}
    if case["kind"] == "window":
        state.update(q=q[0], k=k[0], v=v[0])
    if not own:
        n = torch.tensor(counts)
        return dict(state, k_cache=kc, v_cache=vc, lens=torch.tensor(lens, device="cuda"), seq=torch.repeat_interleave(torch.arange(len(counts)), n).cuda(),
                    row=torch.cat([torch.arange(c) for c in counts]).cuda())
    import paper_2311_11514_amd as hx

    stage = hx.Stage(case["heads"] * case["d"], case["heads"], case["kv_heads"], 256, kc.shape[0], 1, 0, case["dtype"])
    kv = stage.kv_cache_create(case["batch"], kc.shape[2])
    for layer in range(kc.shape[0]):
        for b, n in enumerate(lens):
            if n:
                kv.fill(layer, b, kc[layer, b, :n], vc[layer, b, :n])
    kv.set_lengths(lens)
    state.update(stage=stage, kv=kv, counts=None if set(counts) == {1} else counts)
    if case["kind"] == "evict":
        state["small"] = stage.kv_cache_create(case["batch"], case["keep"] + 1)
    return state


# ---- the operators ------------------------------------------------------------------------------------------------
def _plain_attention(q, k_cache, v_cache, lens, seq, row, most, window, sinks):
    """Rows q [rows, heads, d] of sequence `seq`, number `row` of at most `most`, over caches [batch, slots, kv heads, d] that hold them already:
    the results in 32 bits, and the weights of every slot summed over rows and query heads [batch, kv heads, slots]."""
    batch, slots, hkv, d = k_cache.shape
    group = q.shape[1] // hkv
    k = k_cache.float().permute(0, 2, 3, 1).contiguous()                         # [batch, kv head, d, slot]
    v = v_cache.float().permute(0, 2, 1, 3).contiguous()
    padded = torch.zeros(batch, most, hkv * group, d, device="cuda")
    padded[seq, row] = q.float()
    there = torch.zeros(batch, most, dtype=torch.bool, device="cuda")
    there[seq, row] = True
    padded = padded.view(batch, most, hkv, group, d).permute(0, 2, 1, 3, 4).reshape(batch, hkv, most * group, d)
    at = (lens[:, None] + torch.arange(most, device="cuda"))[:, :, None]         # [batch, row, 1]: a row's own slot
    slot = torch.arange(slots, device="cuda")
    sees = (slot <= at) & ((at - slot < window) | (slot < sinks)) & there[:, :, None]
    score = (padded @ k / math.sqrt(d)).view(batch, hkv, most, group, slots).masked_fill(~sees[:, None, :, None], -math.inf)
    e = torch.exp(score - score.amax(-1, keepdim=True).clamp(min=-3e38))         # rows of the padding see nothing
    p = e / e.sum(-1, keepdim=True).clamp(min=1e-30)
    o = (p.view(batch, hkv, most * group, slots) @ v).view(batch, hkv, most, group, d).permute(0, 2, 1, 3, 4).reshape(batch, most, hkv * group, d)
    return o[seq, row], p.sum((2, 3))


def _plain_window(s):
    case = s["case"]
    at = s["lens"][s["seq"]] + s["row"]
    k, v = s["k_cache"][0], s["v_cache"][0]
    k[s["seq"], at] = s["k"]
    v[s["seq"], at] = s["v"]
    o, gathered = _plain_attention(s["q"], k, v, s["lens"], s["seq"], s["row"], max(1, case["rows_hi"]), case["window"] or WIDE, case["sinks"])
    o = o.to(s["q"].dtype)
    return o if s["weights"] is None else {"out": o, "weights": s["weights"] + gathered}


def _plain_evict(s):
    case = s["case"]
    keep, sinks, recent, w = case["keep"], case["sinks"], case["recent"], s["weights"]
    layers, batch, slots, hkv, d = s["k_cache"].shape
    index = torch.arange(slots, device="cuda")
    n = s["lens"][:, None, None]                                                 # [batch, 1, 1]
    value = index.float().expand(layers, batch, hkv, slots) if w is None else w
    always = (index < sinks) | (index >= n - recent) | (n <= keep)
    value = torch.where(always, math.inf, value).masked_fill(index >= n, -math.inf)
    order = torch.sort(value, dim=-1, descending=True, stable=True).indices      # of equal ones the lowest slot first
    size = keep + 1
    kept = torch.clamp(s["lens"], max=keep)
    inside = torch.arange(size, device="cuda") < kept[:, None, None]             # [batch, 1, size]
    order = torch.nn.functional.pad(order, (0, max(0, size - slots)), value=slots)[..., :size]
    order = torch.where(inside, order, slots).sort(-1).values                    # the kept ones, in the order of their slots
    at = order.clamp(max=slots - 1)
    k, v = [torch.gather(c, 2, at.permute(0, 1, 3, 2)[..., None].expand(-1, -1, -1, -1, d)) for c in (s["k_cache"], s["v_cache"])]
    if case["rotate"]:
        moved = (order - torch.arange(size, device="cuda")).clamp(min=0).permute(0, 1, 3, 2).double()       # [layers, batch, size, kv heads]
        angle = moved[..., None] * THETA ** (-2 * torch.arange(d // 2, device="cuda", dtype=torch.float64) / d)
        c, sn = torch.cos(angle).float(), torch.sin(angle).float()
        a, b = k.float().split(d // 2, -1)
        k = torch.cat((a * c + b * sn, b * c - a * sn), -1).to(k.dtype)
    mine = torch.where(inside, order, -1).int()
    # the next row of every sequence, in every layer
    lens = kept.repeat(layers)
    every = torch.arange(layers * batch, device="cuda")
    k, v = k.reshape(-1, size, hkv, d), v.reshape(-1, size, hkv, d)
    k[every, lens], v[every, lens] = s["k"].flatten(0, 1), s["v"].flatten(0, 1)
    o, _ = _plain_attention(s["q"].flatten(0, 1), k, v, lens, every, torch.zeros_like(every), 1, WIDE, 0)
    out = {"slots": mine, "out": o.to(s["q"].dtype).view_as(s["q"])}
    if w is not None:
        out["weights"] = torch.where(inside, torch.gather(w, 3, at), 0.0)
    return out


def run(state):
    case = state["case"]
    if not own:
        return _plain_window(state) if case["kind"] == "window" else _plain_evict(state)
    if case["kind"] == "window":
        window = case["window"] or None
        if state["weights"] is None:
            return state["kv"].window_attention(0, state["q"], state["k"], state["v"], state["counts"], window=window, sinks=case["sinks"])
        weights = state["weights"].clone()
        o = state["kv"].window_attention(0, state["q"], state["k"], state["v"], state["counts"], window=window, sinks=case["sinks"], weights=weights)
        return {"out": o, "weights": weights}
    slots, weights = state["kv"].evict(case["keep"], sinks=case["sinks"], recent=case["recent"], weights=state["weights"], rotate=case["rotate"],
                                       into=state["small"])
    o = torch.empty_like(state["q"])
    for layer in range(case["layers"]):
        state["small"].window_attention(layer, state["q"][layer], state["k"][layer], state["v"][layer], out=o[layer])
    out = {"slots": slots, "out": o}
    return out if weights is None else dict(out, weights=weights)


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    lens, counts = _contexts(case), _rows(case)
    hq, hkv, d = case["heads"], case["kv_heads"], case["d"]
    edge = sum(counts) * (2 * hq + 4 * hkv) * d * e                                 # q and o; the new k and v, read and appended
    if case["kind"] == "evict":
        layers, keep = case["layers"], case["keep"]
        kept, batch = sum(min(n, keep) for n in lens), case["batch"]
        rows = kept * hkv * d * e
        moved = 4 * rows + 2 * rows + edge                                         # K and V read and written; read by the attention
        marks = 4 * hkv * batch * (keep + 1) + (4 * hkv * (sum(lens) + batch * (keep + 1)) if case["weights"] else 0)
        return {"bytes": layers * (moved + marks), "flops": layers * 4 * d * hq * (kept + batch)}
    window, sinks = case["window"] or WIDE, case["sinks"]
    pairs = reach = 0
    for n, c in zip(lens, counts):
        if not c:
            continue
        first = max(0, n - window + 1)                                             # of the cached positions that some row's window reaches
        reach += max(0, n - first) + min(sinks, first, n)
        pairs += sum(min(p + 1, window) + min(sinks, max(0, p + 1 - window)) for p in range(n, n + c))
    total = 2 * reach * hkv * d * e + edge
    if case["weights"]:
        total += 8 * hkv * (reach + sum(counts))
    return {"bytes": total, "flops": (6 if case["weights"] else 4) * d * hq * pairs}


# ---- the same in 64 bits ------------------------------------------------------------------------------------------
def _exact_rows(q, keys, values, first, window, sinks):
    """One head: rows q [n, d] at positions first .. over keys, values [m, d].  Returns the rows and the weights' sums."""
    p = first + torch.arange(q.shape[0], device="cuda")[:, None]
    j = torch.arange(keys.shape[0], device="cuda")[None]
    seen = torch.logical_and(j <= p, torch.logical_or(j > p - window, j < sinks))
    weight = torch.softmax(torch.where(seen, q @ keys.T / q.shape[1] ** 0.5, -math.inf), 1)
    return weight @ values, weight.sum(0)


def _exact_window(case, seed):
    kc, vc, q, k, v, weights = _drawn(case, seed)
    kc, vc, q, k, v = [x[0].double() for x in (kc, vc, q, k, v)]
    out, row, group = torch.empty_like(q), 0, case["heads"] // case["kv_heads"]
    total = None if weights is None else weights.double()
    for b, (n, c) in enumerate(zip(_contexts(case), _rows(case))):
        for h in range(case["heads"] if c else 0):
            kvh = h // group
            keys, values = torch.cat((kc[b, :n, kvh], k[row:row + c, kvh])), torch.cat((vc[b, :n, kvh], v[row:row + c, kvh]))
            out[row:row + c, h], w = _exact_rows(q[row:row + c, h], keys, values, n, case["window"] or WIDE, case["sinks"])
            if total is not None:
                total[b, kvh, :n + c] += w
        row += c
    return out if total is None else {"out": out, "weights": total}


def _chosen(case, n, weights):
    """The slots of a context of n that stay."""
    keep, sinks, recent = case["keep"], case["sinks"], case["recent"]
    if n <= keep:
        return list(range(n))
    middle = range(sinks, n - recent)
    by = sorted(middle, key=(lambda i: -i) if weights is None else (lambda i: (-weights[i], i)))
    return list(range(sinks)) + sorted(by[:keep - sinks - recent]) + list(range(n - recent, n))


def _exact_evict(case, seed):
    kc, vc, q, k, v, weights = _drawn(case, seed)
    td, d, keep, group = TORCH_TYPE[case["dtype"]], case["d"], case["keep"], case["heads"] // case["kv_heads"]
    layers, batch, hkv = kc.shape[0], case["batch"], case["kv_heads"]
    slots = torch.full((layers, batch, hkv, keep + 1), -1, dtype=torch.int32)
    left = None if weights is None else torch.zeros(layers, batch, hkv, keep + 1, dtype=torch.float64)
    host = None if weights is None else weights.double().cpu()
    out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    for layer in range(layers):
        for b, n in enumerate(_contexts(case)):
            for h in range(hkv):
                at = _chosen(case, n, None if host is None else host[layer, b, h].tolist())
                slots[layer, b, h, :len(at)] = torch.tensor(at, dtype=torch.int32)
                if left is not None:
                    left[layer, b, h, :len(at)] = host[layer, b, h, at]
                pick = torch.tensor(at, device="cuda")
                keys, values = kc[layer, b, pick, h].double(), vc[layer, b, pick, h].double()
                if case["rotate"]:
                    back = (pick - torch.arange(len(at), device="cuda")).double()[:, None]
                    turn = torch.polar(torch.ones_like(back), -back * THETA ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d))
                    turned = torch.complex(keys[:, :d // 2], keys[:, d // 2:]) * turn
                    keys = torch.cat((turned.real, turned.imag), 1).to(td).double()    # the cache holds its type
                keys, values = torch.cat((keys, k[layer, b, h][None].double())), torch.cat((values, v[layer, b, h][None].double()))
                mine = slice(h * group, (h + 1) * group)
                out[layer, b, mine] = torch.softmax(q[layer, b, mine].double() @ keys.T / d ** 0.5, 1) @ values
    got = {"slots": slots, "out": out}
    return got if left is None else dict(got, weights=left)


def exact(case, seed):
    return _exact_window(case, seed) if case["kind"] == "window" else _exact_evict(case, seed)
