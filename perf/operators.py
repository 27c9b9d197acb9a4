"""Operators of speculative decoding, as cases that can be timed and checked.

  kind "attention"  attention of a tree of drafted tokens over the KV cache: the nodes' keys and values join the cache behind each
                    sequence's context, and every node attends the context, its ancestors and itself (`KVCache.tree_attention`)
  kind "accept"     greedy acceptance: the longest path from the root along which each drafted token is the one the model chose for its
                    parent (`Tree.accept`)
  kind "project"    rows times a matrix of 4-bit weights with scales, and possibly zero points, per group of input features (`Q4Matrix.project`)
  kind "head"       final norm, 4-bit LM head and arg-max over the rows of a step (`Head.greedy` after `Head.load_q4`)

Contexts and trees of a batch are ragged: `lo` .. `hi` positions and `nodes_lo` .. `nodes_hi` nodes, spread evenly over these ranges in a
fixed order, so that a case's work does not depend on the seed.  The trees' shapes, the tokens and all values are drawn from it.
"""
from __future__ import annotations

import math
import random

import torch

own = False

TORCH_TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5
VOCAB = 32000          # drafted tokens are drawn from a vocabulary of this size


def _attention(dtype, batch, heads, kv_heads, d, lo, hi, nodes_lo, nodes_hi):
    return dict(kind="attention", dtype=dtype, batch=batch, heads=heads, kv_heads=kv_heads, d=d, lo=lo, hi=hi, nodes_lo=nodes_lo, nodes_hi=nodes_hi)


def _project(dtype, rows, n_in, n_out, group, zeros):
    return dict(kind="project", dtype=dtype, rows=rows, n_in=n_in, n_out=n_out, group=group, zeros=zeros)


def _head(dtype, rows, hidden, vocab, group, zeros):
    return dict(kind="head", dtype=dtype, rows=rows, hidden=hidden, vocab=vocab, group=group, zeros=zeros)


def listed():
    return [
        # the tiny full-precision stage of workloads/configs.py drafting five tokens: the smallest call, latency counts
        dict(_attention("f32", 1, 8, 2, 64, 40, 40, 5, 5), name="attention_f32_tiny"),
        # one interactive request on the narrowest shard of the 70B shape: one kv head, a tree of 26
        dict(_attention("bf16", 1, 8, 1, 128, 2048, 2048, 26, 26), name="attention_b1"),
        # a small fp16 model with 64-wide heads: seven ragged requests, from one token to sixteen
        dict(_attention("f16", 7, 32, 8, 64, 11, 330, 1, 16), name="attention_f16_ragged"),
        # batched verification of short drafts on the narrowest shard, 16 sequences at context 2048
        dict(_attention("bf16", 16, 8, 1, 128, 2048, 2048, 8, 8), name="attention_b16"),
        # the full-width layer: 32 ragged contexts up to 4096, trees of 8 to 64 nodes
        dict(_attention("bf16", 32, 64, 8, 128, 240, 4027, 8, 64), name="attention_b32_wide"),
        # acceptance for one request, and for a full batch of large trees
        dict(kind="accept", batch=1, nodes_lo=26, nodes_hi=26, name="accept_b1"),
        dict(kind="accept", batch=64, nodes_lo=4, nodes_hi=64, name="accept_b64"),
        # full precision, odd sizes, a last group that is not full: a check of a quantised model
        dict(_project("f32", 3, 1000, 1410, 64, True), name="project_f32_odd"),
        # one token through the fused query / key / value projection of the 70B shape
        dict(_project("bf16", 1, 8192, 10240, 128, False), name="project_b1"),
        # twelve sequences through its gate and up projections, the widest matrix
        dict(_project("f16", 12, 8192, 57344, 128, True), name="project_f16_b12"),
        # a drafting step's next token: the 70B LM head in 4 bits, one row
        dict(_head("bf16", 1, 8192, 32000, 128, False), name="head_b1"),
        # the same for a batch on a 4096-wide model with a larger vocabulary
        dict(_head("f16", 24, 4096, 50304, 64, True), name="head_f16_b24"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attention", "attention", "attention", "attention", "project", "project", "project", "accept", "head"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f16", "f16", "f32"])
    if kind == "accept":
        hi = _log_int(rng, 2, 128)
        return dict(kind="accept", batch=_log_int(rng, 1, 64), nodes_lo=_log_int(rng, 1, hi), nodes_hi=hi)
    if kind == "project":
        # widths of models from small to the 70B shape, or odd ones
        n_in = rng.choice([512, 1408, 2048, 4096, 5632, 8192, 28672, _log_int(rng, 65, 9000)])
        n_out = rng.choice([512, 1024, 2560, 4096, 10240, 22016, 2 * _log_int(rng, 40, 6000)])
        return _project(dtype, _log_int(rng, 1, 64 if dtype != "f32" else 24), n_in, n_out, rng.choice([32, 64, 128, 128, 256]), rng.random() < 0.5)
    if kind == "head":
        return _head(dtype, _log_int(rng, 1, 64), rng.choice([512, 1024, 2048, 4096]), rng.choice([1000, 32000, 32000, 50304]), rng.choice([32, 64, 128]), rng.random() < 0.5)
    d, group = rng.choice([64, 128]), rng.choice([1, 2, 3, 4, 8, 8, 16])
    kv_heads = rng.choice([1, 2, 4, 8])
    while group * kv_heads * d % 128:
        kv_heads *= 2
    batch, hi, nodes = _log_int(rng, 1, 32), _log_int(rng, 1, 4096), _log_int(rng, 1, 96)
    lo, nodes_lo = int(hi * rng.uniform(0.0, 1.0)), max(1, int(nodes * rng.uniform(0.1, 1.0)))
    most = 32 * 64 * 40 * 2100                  # (sequence, head, node, position) quadruples: about the largest listed case
    if dtype == "f32":
        most //= 8
    while batch * group * kv_heads * nodes * hi > most or batch * kv_heads * hi > 32 * 8 * 2100:
        if batch > 1:
            batch = (batch + 1) // 2
        else:
            hi, lo = hi // 2, lo // 2
    return _attention(dtype, batch, group * kv_heads, kv_heads, d, lo, hi, nodes_lo, nodes)


def _spread(n, lo, hi, step):
    return [lo + int(round((hi - lo) * (((i + 1) * step) % 1.0))) for i in range(n)]


def _contexts(case):
    return _spread(case["batch"], case["lo"], case["hi"], 0.6180339887498949)


def _nodes(case):
    return _spread(case["batch"], case["nodes_lo"], case["nodes_hi"], 0.41421356237309515)


# ---- inputs -------------------------------------------------------------------------------------------------------
def _generator(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1009 + salt)
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _trees(case, seed):
    """Per sequence the parents of its nodes, -1 for the root, every parent in front of its children: bushy, a few tokens deep."""
    r = random.Random(seed * 7 + 3)
    return [[-1] + [r.randrange(0, max(1, (i + 1) // 2)) for i in range(1, n)] for n in _nodes(case)]


def _tokens(trees, seed):
    """Drafted tokens, some of them drafted twice below one parent, and for each node the token the model chooses behind it: for most
    nodes one that a child of theirs carries."""
    r = random.Random(seed * 11 + 5)
    draft, chosen = [], []
    for parents in trees:
        mine = [r.randrange(VOCAB) for _ in parents]
        for i in range(2, len(parents)):
            if parents[i] == parents[i - 1] and r.random() < 0.1:
                mine[i] = mine[i - 1]
        children = {}
        for i, p in enumerate(parents):
            children.setdefault(p, []).append(i)
        chosen += [mine[r.choice(children[i])] if i in children and r.random() < 0.8 else r.randrange(VOCAB) for i in range(len(parents))]
        draft += mine
    return draft, chosen


def _plan(trees):
    """Where the packed rows sit in a batch padded to the largest tree, the ancestors (each node among its own), the parents."""
    counts = torch.tensor([len(t) for t in trees])
    n = int(counts.max())
    parent = torch.full((len(trees), n), -1)
    ancestors = torch.zeros(len(trees), n, n, dtype=torch.bool)
    for b, t in enumerate(trees):
        for i, p in enumerate(t):
            parent[b, i] = p
            if p >= 0:
                ancestors[b, i] = ancestors[b, p]
            ancestors[b, i, i] = True
    seq = torch.repeat_interleave(torch.arange(len(trees)), counts)
    node = torch.cat([torch.arange(len(t)) for t in trees])
    return {"seq": seq.cuda(), "node": node.cuda(), "counts": counts.cuda(), "parent": parent.cuda(), "ancestors": ancestors.cuda()}


def _tree_handle(trees):
    import paper_2311_11514_amd as hx

    tree = hx.Tree(len(trees), sum(len(t) for t in trees))
    tree.set([len(t) for t in trees], [p for t in trees for p in t])
    return tree


def _weights(case, seed, n_in, n_out):
    """4-bit weights, two neighbouring columns a byte, and their groups' scales (products of about unit size) and zero points."""
    g = _generator(seed, 3)
    groups = -(-n_in // case["group"])
    w4 = torch.randint(0, 256, (n_in, n_out // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = ((1 + 0.2 * torch.rand(groups, n_out, generator=g, device="cuda")) / (5 * math.sqrt(n_in))).to(TORCH_TYPE[case["dtype"]])
    zeros = torch.randint(0, 256, (groups, n_out // 2), generator=g, device="cuda", dtype=torch.uint8) if case["zeros"] else None
    return w4, scales, zeros


def prepare(case, seed):
    if case["kind"] == "accept":
        trees = _trees(case, seed)
        draft, chosen = _tokens(trees, seed)
        state = {"draft": torch.tensor(draft, dtype=torch.int32, device="cuda"), "chosen": torch.tensor(chosen, dtype=torch.int32, device="cuda")}
        if own:
            state["tree"] = _tree_handle(trees)
        else:
            state["plan"] = _plan(trees)
        return dict(state, kind="accept")
    td = TORCH_TYPE[case["dtype"]]
    if case["kind"] == "attention":
        trees, lens = _trees(case, seed), _contexts(case)
        g = _generator(seed, 1)
        batch, hkv, d = case["batch"], case["kv_heads"], case["d"]
        rows, size = sum(len(t) for t in trees), max(n + len(t) for n, t in zip(lens, trees))
        cache = [_normal(g, batch, size, hkv, d).to(td) for _ in range(2)]
        new = {x: _normal(g, rows, heads, d).to(td) for x, heads in (("q", case["heads"]), ("k", hkv), ("v", hkv))}
        state = dict(new, kind="attention")
        if not own:
            return dict(state, k_cache=cache[0], v_cache=cache[1], lens=torch.tensor(lens, device="cuda"), plan=_plan(trees))
        import paper_2311_11514_amd as hx

        hidden = case["heads"] * d
        stage = hx.Stage(hidden, case["heads"], hkv, 256, 1, 1, 0, case["dtype"])
        kv = stage.kv_cache_create(batch, size)
        for b, n in enumerate(lens):
            if n:
                kv.fill(0, b, cache[0][b, :n], cache[1][b, :n])
        kv.set_lengths(lens)
        return dict(state, stage=stage, kv=kv, tree=_tree_handle(trees))
    if case["kind"] == "project":
        w4, scales, zeros = _weights(case, seed, case["n_in"], case["n_out"])
        state = {"kind": "project", "x": _normal(_generator(seed, 2), case["rows"], case["n_in"]).to(td)}
        if not own:
            return dict(state, w4=w4, scales=scales, zeros=zeros, group=case["group"])
        import paper_2311_11514_amd as hx

        matrix = hx.Q4Matrix(case["n_in"], case["n_out"], case["group"], case["dtype"])
        matrix.load(w4, scales, zeros)
        return dict(state, matrix=matrix)
    w4, scales, zeros = _weights(case, seed, case["hidden"], case["vocab"])
    g = _generator(seed, 2)
    gain = (1 + 0.02 * _normal(g, case["hidden"])).to(td)
    state = {"kind": "head", "a": _normal(g, case["rows"], case["hidden"]).to(td), "b": _normal(g, case["rows"], case["hidden"]).to(td)}
    if not own:
        return dict(state, gain=gain, w4=w4, scales=scales, zeros=zeros, group=case["group"])
    import paper_2311_11514_amd as hx

    head = hx.Head(case["hidden"], case["vocab"], 1, 0, case["dtype"], EPS)
    head.load_q4(gain, w4, scales, zeros, group=case["group"])
    return dict(state, head=head)


# ---- the operators ------------------------------------------------------------------------------------------------
def _nibbles(w):
    return torch.stack((w & 15, w >> 4), dim=-1).flatten(-2)


def _plain_weights(s, n_in):
    groups = s["scales"].shape[0]
    scale = s["scales"].float()
    zero = _nibbles(s["zeros"]).float() if s["zeros"] is not None else torch.full_like(scale, 8.0)
    w = _nibbles(s["w4"]).float()
    full = n_in // s["group"] * s["group"]
    if full == n_in:
        w = w.view(groups, s["group"], -1)
        return ((w - zero[:, None]) * scale[:, None]).view(n_in, -1)
    at = torch.arange(n_in, device="cuda") // s["group"]
    return (w - zero[at]) * scale[at]


def _plain_attention(s):
    p, dtype = s["plan"], s["q"].dtype
    batch, hkv, d = s["k_cache"].shape[0], s["k_cache"].shape[2], s["k_cache"].shape[3]
    nodes, group = p["parent"].shape[1], s["q"].shape[1] // hkv
    at = s["lens"][p["seq"]] + p["node"]
    s["k_cache"][p["seq"], at] = s["k"]
    s["v_cache"][p["seq"], at] = s["v"]
    k = s["k_cache"].float().permute(0, 2, 3, 1).contiguous()                   # [batch, kv head, d, position]
    v = s["v_cache"].float().permute(0, 2, 1, 3).contiguous()
    q = torch.zeros(batch, nodes, hkv * group, d, device="cuda")
    q[p["seq"], p["node"]] = s["q"].float()
    q = q.view(batch, nodes, hkv, group, d).permute(0, 2, 1, 3, 4).reshape(batch, hkv, nodes * group, d)
    drafted = torch.arange(k.shape[3], device="cuda")[None] - s["lens"][:, None]  # [batch, position]: index among the drafted ones
    ancestor = torch.gather(p["ancestors"], 2, drafted.clamp(0, nodes - 1)[:, None].expand(batch, nodes, -1))
    sees = (drafted < 0)[:, None] | (ancestor & (drafted < nodes)[:, None])
    score = (q @ k / math.sqrt(d)).view(batch, hkv, nodes, group, -1).masked_fill(~sees[:, None, :, None], -math.inf)
    e = torch.exp(score - score.amax(-1, keepdim=True).clamp(min=-3e38))         # rows of the padding see nothing, or their context
    o = e.view(batch, hkv, nodes * group, -1) @ v / e.sum(-1).view(batch, hkv, nodes * group, 1)
    o = o.view(batch, hkv, nodes, group, d).permute(0, 2, 1, 3, 4).reshape(batch, nodes, hkv * group, d)
    return o[p["seq"], p["node"]].to(dtype)


def _plain_accept(s):
    p = s["plan"]
    batch, nodes = p["parent"].shape
    draft = torch.full((batch, nodes), -1, dtype=torch.int32, device="cuda")
    draft[p["seq"], p["node"]] = s["draft"]
    chosen = torch.full((batch, nodes), -1, dtype=torch.int32, device="cuda")
    chosen[p["seq"], p["node"]] = s["chosen"]
    index = torch.arange(nodes, device="cuda")
    there = index[None] < p["counts"][:, None]
    wanted = torch.gather(chosen, 1, p["parent"].clamp(min=0))
    twin = (p["parent"][:, :, None] == p["parent"][:, None]) & (draft[:, :, None] == draft[:, None]) & (index[None] < index[:, None])
    fits = there & ((draft == wanted) & ~twin.any(2) | (p["parent"] < 0))        # of twins the first
    kept = there & ~(p["ancestors"] & ~fits[:, None]).any(2)
    order = torch.where(kept, index, nodes + index).argsort(1)                   # the kept ones in front: every parent before its children
    count = kept.sum(1)
    inside = index[None] < count[:, None]
    path = torch.where(inside, order, -1)
    tokens = torch.where(inside, torch.gather(chosen, 1, order), -1)
    at = (p["seq"], p["node"])
    return {"kept": count.int(), "path": path[at].int(), "tokens": tokens[at].int()}


def _plain_head(s):
    x = s["a"].float() + s["b"].float()
    x = x * torch.rsqrt((x * x).mean(1, keepdim=True) + EPS) * s["gain"].float()
    logits = x @ _plain_weights(s, x.shape[1])
    best = logits.amax(1)
    index = torch.arange(logits.shape[1], device="cuda")
    token = torch.where(logits == best[:, None], index, logits.shape[1]).amin(1)
    return {"token": token.int(), "logit": best}


def run(state):
    if state["kind"] == "attention":
        if own:
            return state["kv"].tree_attention(0, state["tree"], state["q"], state["k"], state["v"])
        return _plain_attention(state)
    if state["kind"] == "accept":
        if own:
            kept, path, tokens = state["tree"].accept(state["draft"], state["chosen"])
            return {"kept": kept, "path": path, "tokens": tokens}
        return _plain_accept(state)
    if state["kind"] == "project":
        if own:
            return state["matrix"].project(state["x"])
        return (state["x"].float() @ _plain_weights(state, state["x"].shape[1])).to(state["x"].dtype)
    if own:
        token, logit = state["head"].greedy(state["a"], state["b"])
        return {"token": token, "logit": logit}
    return _plain_head(state)


def work(case):
    e = 4 if case.get("dtype") == "f32" else 2
    if case["kind"] == "accept":
        rows = sum(_nodes(case))
        return {"bytes": 4 * (5 * rows + 2 * case["batch"]), "flops": rows}      # parents, drafted and chosen tokens; path and tokens
    if case["kind"] == "attention":
        lens, nodes = _contexts(case), _nodes(case)
        hq, hkv, d = case["heads"], case["kv_heads"], case["d"]
        rows = sum(nodes)
        moved = 2 * sum(lens) * hkv * d + 2 * rows * hq * d + 4 * rows * hkv * d     # context; q and o; the drafted k and v, read and appended
        return {"bytes": e * moved, "flops": 4 * d * hq * sum(n * (c + 1) for n, c in zip(nodes, lens))}
    head = case["kind"] == "head"
    n_in, n_out = (case["hidden"], case["vocab"]) if head else (case["n_in"], case["n_out"])
    groups = -(-n_in // case["group"])
    weights = n_in * n_out / 2 + groups * n_out * (e + (0.5 if case["zeros"] else 0))
    rows = case["rows"]
    edge = e * (2 * rows * n_in + n_in) + 8 * rows if head else e * rows * (n_in + n_out)
    return {"bytes": weights + edge, "flops": 2 * rows * n_in * n_out}


# ---- the same in 64 bits ------------------------------------------------------------------------------------------
def _exact_matrix(case, seed, n_in, n_out):
    w4, scales, zeros = _weights(case, seed, n_in, n_out)
    w = torch.empty(n_in, n_out, dtype=torch.float64, device="cuda")
    for first in range(0, n_in, case["group"]):
        at, last = first // case["group"], min(first + case["group"], n_in)
        for odd in (0, 1):
            shift = 16 if odd else 1
            zero = 8.0 if zeros is None else (zeros[at] // shift % 16).double()
            w[first:last, odd::2] = ((w4[first:last] // shift % 16).double() - zero) * scales[at, odd::2].double()
    return w


def _exact_attention(case, seed):
    td = TORCH_TYPE[case["dtype"]]
    trees, lens = _trees(case, seed), _contexts(case)
    g = _generator(seed, 1)
    hkv, d = case["kv_heads"], case["d"]
    rows, size = sum(len(t) for t in trees), max(n + len(t) for n, t in zip(lens, trees))
    kc, vc = [_normal(g, case["batch"], size, hkv, d).to(td) for _ in range(2)]
    q, k, v = [_normal(g, rows, heads, d).to(td).double() for heads in (case["heads"], hkv, hkv)]
    out, row = torch.empty(rows, case["heads"], d, dtype=torch.float64, device="cuda"), 0
    for b, parents in enumerate(trees):
        n, c = len(parents), lens[b]
        hidden = torch.ones(n, c + n, dtype=torch.bool)
        hidden[:, :c] = False
        for i in range(n):
            a = i
            while a >= 0:
                hidden[i, c + a] = False
                a = parents[a]
        hidden = hidden.cuda()
        for h in range(case["heads"]):
            kv = h // (case["heads"] // hkv)
            keys = torch.cat((kc[b, :c, kv].double(), k[row:row + n, kv]))
            values = torch.cat((vc[b, :c, kv].double(), v[row:row + n, kv]))
            weight = torch.softmax((q[row:row + n, h] @ keys.T / d ** 0.5).masked_fill(hidden, -math.inf), 1)
            out[row:row + n, h] = weight @ values
        row += n
    return out


def _exact_accept(case, seed):
    trees = _trees(case, seed)
    draft, chosen = _tokens(trees, seed)
    kept, path, tokens, first = [], [], [], 0
    for parents in trees:
        n, walk = len(parents), [0]
        while True:
            here = walk[-1]
            nexts = [i for i in range(n) if parents[i] == here and draft[first + i] == chosen[first + here]]
            if not nexts:
                break
            walk.append(nexts[0])
        kept.append(len(walk))
        path += walk + [-1] * (n - len(walk))
        tokens += [chosen[first + i] for i in walk] + [-1] * (n - len(walk))
        first += n
    return {name: torch.tensor(x, dtype=torch.int32) for name, x in (("kept", kept), ("path", path), ("tokens", tokens))}


def exact(case, seed):
    if case["kind"] == "attention":
        return _exact_attention(case, seed)
    if case["kind"] == "accept":
        return _exact_accept(case, seed)
    td = TORCH_TYPE[case["dtype"]]
    g = _generator(seed, 2)
    if case["kind"] == "project":
        x = _normal(g, case["rows"], case["n_in"]).to(td).double()
        return x @ _exact_matrix(case, seed, case["n_in"], case["n_out"])
    gain = (1 + 0.02 * _normal(g, case["hidden"])).to(td).double()
    x = sum(_normal(g, case["rows"], case["hidden"]).to(td).double() for _ in range(2))
    x = x / torch.sqrt((x ** 2).sum(1, keepdim=True) / case["hidden"] + EPS) * gain
    logit, token = torch.max(x @ _exact_matrix(case, seed, case["hidden"], case["vocab"]), 1)
    return {"token": token.int(), "logit": logit}
