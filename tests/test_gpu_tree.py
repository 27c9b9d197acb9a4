"""Drafted trees on the GPU against 64 bits: attention over the cache, acceptance, the rows that are kept, a stage's layers, and the
three together as speculative decoding, which has to say what plain decoding says."""
import math

import numpy as np
import pytest
import torch

import paper_2311_11514_amd as hx
from tests import tree_reference as tr
from tests.helpers import TOL, check, make_gpu_stage, make_oracle, to_dev
from workloads import StageConfig, generate

pytestmark = pytest.mark.gpu


class Case:
    """A cache with contexts, trees, and rows for them; values as they are stored, in float64."""

    def __init__(self, dtype, hq, hkv, d, lens, trees, max_seq=None, layers=1, seed=0, fill=True):
        self.dtype, self.hq, self.hkv, self.d, self.lens, self.trees = dtype, hq, hkv, d, lens, trees
        self.stage = hx.Stage(hq * d, hq, hkv, 256, layers, 1, 0, dtype)
        self.kv = self.stage.kv_cache_create(len(lens), max_seq or max(n + len(t) for n, t in zip(lens, trees)))
        g = torch.Generator().manual_seed(seed)
        td = tr.TORCH[dtype]
        self.ctx = [[[torch.randn(n, hkv, d, generator=g).to(td) for _ in range(2)] for n in lens] for _ in range(layers)]
        if fill:
            for layer in range(layers):
                for b, n in enumerate(lens):
                    if n:
                        self.kv.fill(layer, b, *self.ctx[layer][b])
        self.kv.set_lengths(lens)
        self.rows = sum(len(t) for t in trees)
        self.q = torch.randn(self.rows, hq, d, generator=g).to(td)
        self.k, self.v = (torch.randn(self.rows, hkv, d, generator=g).to(td) for _ in range(2))
        self.tree = hx.Tree(len(lens), max(1, self.rows))
        self.tree.set([len(t) for t in trees], [p for t in trees for p in t])

    def attend(self, layer=0, **kw):
        out = self.kv.tree_attention(layer, self.tree, self.q.cuda(), self.k.cuda(), self.v.cuda(), **kw)
        torch.cuda.synchronize()
        return out

    def reference(self, layer=0):
        """Per sequence (o, bound)."""
        row, found = 0, []
        for b, t in enumerate(self.trees):
            n = len(t)
            part = [x[row:row + n].double().numpy() for x in (self.q, self.k, self.v)]
            ctx = [x.double().numpy() for x in self.ctx[layer][b]]
            o, a, s = tr.attention(part[0], ctx[0], ctx[1], part[1], part[2], t)
            found.append((o, tr.attention_bound(o, a, s, self.dtype, self.d, self.lens[b] + n)))
            row += n
        return np.concatenate([x[0] for x in found]), np.concatenate([x[1] for x in found])

    def check(self, out, layer=0):
        o, bound = self.reference(layer)
        off = np.abs(out.double().cpu().numpy() - o) / bound
        print(f"{self.dtype} {self.lens} {[len(t) for t in self.trees]}: {off.max():.3f} of the bound", flush=True)
        assert off.max() <= 1, np.unravel_index(off.argmax(), off.shape)


def _trees(counts, seed=1, width=0):
    return [tr.random_tree(n, seed + i, width) for i, n in enumerate(counts)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,lens,counts", [
    (2, 2, 64, [0], [1]),                            # one node, nothing before it
    (8, 2, 64, [40], [5]),
    (2, 1, 64, [31, 32, 33, 0], [1, 1, 1, 2]),       # around the end of a tile
    (8, 1, 128, [63, 64, 1], [3, 0, 4]),             # a sequence without a tree
    (4, 4, 128, [100, 7], [8, 33]),                  # one head a group, the tree over a tile's end
    (6, 2, 64, [129], [17]),                         # groups of three
    (16, 1, 128, [50], [7]),                         # the widest group
    (8, 1, 128, [300, 31, 5], [16, 9, 40]),
    (8, 8, 64, [95], [64]),                          # a mask of more than a word, shifted by 31
    (4, 1, 64, [20, 3], [100, 256]),                 # the largest tree
])
def test_attention_matches_64_bits(dtype, hq, hkv, d, lens, counts):
    c = Case(dtype, hq, hkv, d, lens, _trees(counts))
    c.check(c.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,lens,counts", [
    (2, 1, 128, [3000], [2]),                        # 32 rows or fewer a block: four tiles a step, cut into runs
    (4, 1, 64, [2100, 5, 1000], [13, 16, 2]),        # two row groups; a context that is shorter than one run
    (8, 1, 128, [1500, 0, 700], [26, 20, 30]),       # four row groups
    (2, 1, 64, [4000], [1]),                         # the single token
])
def test_long_contexts_in_runs_match_64_bits(dtype, hq, hkv, d, lens, counts):
    c = Case(dtype, hq, hkv, d, lens, _trees(counts, seed=7), seed=3)
    c.check(c.attend())


WIDE = [                                             # enough tiles that blocks share them
    (64, 8, 128, [2148, 2099, 2181, 2148, 2200, 2147, 2149, 2144], [16] * 7 + [9]),                        # 64 rows a block, in runs
    (64, 8, 64, [2148, 2099, 2181, 2148, 2200, 2147, 2149, 2144], [16] * 7 + [9]),
    (64, 8, 128, [860 + 9 * i for i in range(15)] + [3], [20] * 12 + [0, 1, 33, 18]),                       # 64 rows, whole contexts
    (64, 8, 128, [230 + 9 * i for i in range(16)], [64 - (i % 4) for i in range(16)]),                      # 128 rows
    (64, 8, 64, [230 + 9 * i for i in range(16)], [64 - (i % 4) for i in range(16)]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hkv,d,lens,counts", WIDE)
def test_blocks_that_share_tiles_match_64_bits(dtype, hq, hkv, d, lens, counts):
    c = Case(dtype, hq, hkv, d, lens, _trees(counts, seed=5), seed=8)
    out = c.attend()
    c.check(out)
    assert torch.equal(c.attend(), out)                # the same bits, from rows that are in the cache by now as well


@pytest.mark.parametrize("hq,hkv,d,lens,counts", WIDE)
def test_blocks_that_share_tiles_and_slots_that_are_nobodys(hq, hkv, d, lens, counts):
    """NaN behind every tree, and an infinity in the rows of the last node of each, which no other node attends."""
    c = Case("bf16", hq, hkv, d, lens, _trees(counts, seed=6), max_seq=max(lens) + 128, seed=9, fill=False)
    for b, n in enumerate(lens):
        pad = torch.full((128, hkv, d), float("nan"))
        c.kv.fill(0, b, *[torch.cat([x.float(), pad]) for x in c.ctx[0][b]])
    c.kv.set_lengths(lens)
    c.check(c.attend())
    last = np.cumsum([len(t) for t in c.trees])[[len(t) > 0 for t in c.trees]] - 1
    c.v[last] = float("inf")
    out = c.attend().double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        o, bound = c.reference()
    good = np.setdiff1d(np.arange(c.rows), last)
    assert (np.abs(out[good] - o[good]) <= bound[good]).all() and not np.isfinite(out[last]).any()


def test_more_sequences_than_the_plan_orders():
    """Sequences beyond the 64 that are dispatched by length."""
    for dtype in ("bf16", "f32"):
        c = Case(dtype, 4, 2, 64, [(37 * i) % 150 for i in range(75)], _trees([(i % 5) + (i % 7 == 0) for i in range(75)], seed=2), seed=4)
        c.check(c.attend())


@pytest.mark.parametrize("width", [1, 2, 255])
def test_tree_shapes(width):
    """A chain (plain causal attention), a binary tree, a star."""
    c = Case("bf16", 4, 2, 64, [37], _trees([70], width=width))
    c.check(c.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_what_a_node_does_not_attend_has_no_influence(dtype):
    """Infinities and NaN in the keys and values of siblings, and in slots behind the tree that an earlier, larger tree left."""
    parents = [-1, 0, 0, 1, 2, 2, 4, 0]
    big = Case(dtype, 4, 2, 64, [45], [parents], max_seq=64, seed=11)
    big.k[5], big.v[5] = math.nan, math.inf             # nobody's ancestor
    big.k[7], big.v[7] = -math.inf, math.nan
    out = big.attend().double().cpu().numpy()
    good = [0, 1, 2, 3, 4, 6]
    assert np.isnan(out[[5, 7]]).all()                  # they attend themselves
    o, bound = big.reference()                          # per row over its own ancestors only
    assert (np.abs(out[good] - o[good]) <= bound[good]).all()
    big.trees = [parents[:5]]
    big.tree.set([5], parents[:5])
    big.rows, big.q, big.k, big.v = 5, big.q[:5], big.k[:5], big.v[:5]
    big.check(big.attend())                             # slots 45 + 5 and 45 + 7 still hold what was there
    # a visible infinity arrives
    big.v[1, 0, 3] = math.inf
    out = big.attend().double().cpu().numpy()
    assert np.isinf(out[[1, 3], :2, 3]).all() and np.isfinite(out[[0, 2, 4]]).all() and np.isfinite(out[[1, 3], 2:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_extreme_scores(dtype):
    """Scores far apart, and a context whose scores are all of the type's lowest value: the weights still sum to one."""
    c = Case(dtype, 4, 1, 64, [70], _trees([6]), seed=5)
    c.q = c.q * 60
    c.check(c.attend())
    low = torch.finfo(tr.TORCH[dtype]).min
    c = Case(dtype, 2, 2, 64, [40], [[-1]], seed=6, fill=False)
    c.q, c.k, keys = torch.zeros_like(c.q), torch.zeros_like(c.k), torch.zeros(40, 2, 64, dtype=tr.TORCH[dtype])
    c.q[..., 0], c.k[..., 0], keys[..., 0] = 1.0, low, low
    c.kv.fill(0, 0, keys, c.ctx[0][0][1])
    c.kv.set_lengths([40])
    values = np.concatenate([c.ctx[0][0][1].double().numpy(), c.v.double().numpy()])      # equal scores, and exactly: the mean
    o, a = values.mean(0)[None], np.abs(values).mean(0)[None]
    assert (np.abs(c.attend().double().cpu().numpy() - o) <= tr.attention_bound(o, a, 0.0, dtype, 64, 41)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_rows_join_the_cache_and_nothing_else_changes(dtype):
    c = Case(dtype, 4, 2, 64, [30, 5], _trees([6, 3]), max_seq=64, layers=2)
    before = [[c.kv.read(layer, b, 0, 64) for b in range(2)] for layer in range(2)]
    c.attend(layer=1)
    row = 0
    for b, (n, t) in enumerate(zip(c.lens, c.trees)):
        k, v = c.kv.read(1, b, 0, 64)
        want = [x.clone() for x in before[1][b]]
        want[0][n:n + len(t)], want[1][n:n + len(t)] = c.k[row:row + len(t)].float(), c.v[row:row + len(t)].float()
        assert torch.equal(k, want[0]) and torch.equal(v, want[1])
        assert all(torch.equal(x, y) for x, y in zip(c.kv.read(0, b, 0, 64), before[0][b]))
        row += len(t)
    assert c.kv.get_lengths(2) == [30, 5]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_contexts_from_device_memory_are_those_from_the_host(dtype):
    st = hx.Stage(512, 4, 2, 256, 1, 1, 0, dtype)
    kv = st.kv_cache_create(2, 64)
    k, v = (torch.randn(45, 2, 128, generator=torch.Generator().manual_seed(i)).to(tr.TORCH[dtype]) for i in range(2))
    kv.fill(0, 0, k, v)
    kv.fill(0, 1, k.cuda(), v.cuda())
    kv.set_lengths([45, 45])
    for a, b, want in zip(kv.read(0, 0, 0, 45), kv.read(0, 1, 0, 45), (k, v)):
        assert torch.equal(a, want.float()) and torch.equal(b, a)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_parts_of_a_fused_projection_and_an_output_of_the_callers(dtype):
    c = Case(dtype, 8, 2, 64, [100, 3], _trees([9, 4]))
    want = c.attend()
    fused = torch.cat([c.q.flatten(1), c.k.flatten(1), c.v.flatten(1)], 1).cuda()
    q, k, v = fused.split([512, 128, 128], 1)
    guard = torch.full((c.rows + 2, 8, 64), 7.0, dtype=tr.TORCH[dtype], device="cuda")
    got = c.kv.tree_attention(0, c.tree, q, k, v, out=guard[1:-1])
    assert torch.equal(got, want)
    assert (guard[0] == 7).all() and (guard[-1] == 7).all()
    wide = torch.zeros(c.rows, 16, 64, dtype=tr.TORCH[dtype], device="cuda")
    wide[:, :8] = c.q.cuda()
    assert torch.equal(c.kv.tree_attention(0, c.tree, wide[:, :8], k, v), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_another_stream_and_the_same_bits_again(dtype):
    c = Case(dtype, 8, 1, 128, [1500, 40], _trees([20, 12]))
    want = c.attend()
    s = torch.cuda.Stream()
    args = [x.cuda() for x in (c.q, c.k, c.v)]
    s.wait_stream(torch.cuda.current_stream())
    got = [c.kv.tree_attention(0, c.tree, *args, stream=s) for _ in range(5)]
    s.synchronize()
    assert all(torch.equal(x, want) for x in got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_recorded_and_replayed(dtype):
    """Replays take the rows, the trees and the lengths of that moment."""
    c = Case(dtype, 8, 1, 128, [700, 40], _trees([10, 30]), max_seq=1024)
    args = [x.cuda() for x in (c.q, c.k, c.v)]
    c.kv.tree_attention(0, c.tree, *args)
    torch.cuda.synchronize()
    out = torch.empty_like(args[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.kv.tree_attention(0, c.tree, *args, out=out)
    for k in range(4):
        fresh = [torch.randn_like(x.float()).to(x.dtype) for x in args]
        lens = [600 + 100 * k, 7 * k]
        parents = [p for t in _trees([10, 30], seed=50 + k) for p in t]
        c.kv.set_lengths(lens)
        c.tree.set([10, 30], parents)
        want = c.kv.tree_attention(0, c.tree, *fresh)
        for x, y in zip(args, fresh):
            x.copy_(y)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        # (an eager call may cut the contexts elsewhere: the 32-bit sums are in another order, a result may round the other way)
        off = (out.double() - want.double()).abs().max().item() / want.double().abs().max().item()
        assert off <= 2 * tr.UNIT[dtype] + 2 ** -18, (k, off)


def test_attention_refusals():
    c = Case("bf16", 4, 2, 64, [30, 40], _trees([3, 4]), max_seq=44)
    q, k, v = c.q.cuda(), c.k.cuda(), c.v.cuda()

    def status(f, *a, **kw):
        with pytest.raises(hx.HexgenError) as e:
            f(*a, **kw)
        return e.value.status

    raw = hx.lib.hexgen_kv_tree_attention
    good = [c.kv.handle, 0, c.tree.handle, q.data_ptr(), 256, k.data_ptr(), 128, v.data_ptr(), 128, q.data_ptr()]
    for at, bad in ((1, 1), (1, -1), (3, None), (5, None), (7, None), (9, None), (3, q.data_ptr() + 2), (4, 248), (4, 260), (6, 120), (8, 127)):
        args = list(good)
        args[at] = bad
        assert raw(*args, None) == 1, (at, bad)
    assert raw(*good[:2], None, *good[3:], None) == 1
    c.kv.set_lengths([30, 41])
    assert status(c.kv.tree_attention, 0, c.tree, q, k, v) == 4
    c.kv.set_lengths([30])
    assert status(c.kv.tree_attention, 0, c.tree, q, k, v) == 3          # trees of two sequences, a batch of one
    c.kv.reset()
    assert status(c.kv.tree_attention, 0, c.tree, q, k, v) == 3
    empty = hx.Tree(2, 4)
    assert raw(*good[:2], empty.handle, *good[3:], None) == 3
    assert hx.lib.hexgen_stage_decode_tree(c.stage.handle, c.kv.handle, c.tree.handle, q.data_ptr(), q.data_ptr(), None, None) == 3   # no weights
    with pytest.raises(ValueError, match="^q"):
        c.kv.tree_attention(0, c.tree, q[:-1], k, v)
    with pytest.raises(ValueError, match="^k"):
        c.kv.tree_attention(0, c.tree, q, k.cpu(), v)
    # a refused set leaves the trees that were there
    c.kv.set_lengths([30, 40])
    want = c.kv.tree_attention(0, c.tree, q, k, v)
    with pytest.raises(hx.HexgenError):
        c.tree.set([2, 2], [-1, 0, 0, 0])
    assert torch.equal(c.kv.tree_attention(0, c.tree, q, k, v), want)


# ---- acceptance ---------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("counts,width,vocab", [([1], 0, 2), ([26], 0, 3), ([0, 5, 0, 1], 0, 2), ([256, 255, 64, 65], 1, 1), ([256, 130, 63], 2, 2),
                                                ([256], 255, 300), ([40] * 70, 0, 3), ([7, 200], 0, 1)])
def test_accept(counts, width, vocab):
    """Small vocabularies: drafted twins and long paths."""
    trees = _trees(counts, seed=31, width=width)
    tree = hx.Tree(len(counts), sum(counts))
    tree.set(counts, [p for t in trees for p in t])
    for seed in range(3):
        r = np.random.default_rng(seed)
        draft, chosen = (r.integers(0, vocab, sum(counts)).astype(np.int32) for _ in range(2))
        kept, path, tokens = (x.cpu().tolist() for x in tree.accept(torch.tensor(draft).cuda(), torch.tensor(chosen).cuda()))
        row = 0
        for b, t in enumerate(trees):
            n = len(t)
            p, tok = tr.accept(t, draft[row:row + n].tolist(), chosen[row:row + n].tolist())
            assert kept[b] == len(p)
            assert path[row:row + n] == p + [-1] * (n - len(p)) and tokens[row:row + n] == tok + [-1] * (n - len(p))
            row += n


# ---- keeping ------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_keep_moves_the_path_behind_the_context(dtype):
    trees = [[-1, 0, 0, 2, 1, 3, 3, 6, 7, 8, 9, 10, 11, 12, 13, 14], [-1, 0, 0], [-1, 0], [], [-1]]
    paths = [[0, 2, 3, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15], [0], [], [], [0]]
    lens = [29, 32, 3, 4, 31]
    c = Case(dtype, 4, 2, 64, lens, trees, max_seq=64, layers=3)
    for layer in range(3):
        c.attend(layer=layer)
    before = [[c.kv.read(layer, b, 0, 64) for b in range(5)] for layer in range(3)]
    flat = [x for t, p in zip(trees, paths) for x in p + [-1] * (len(t) - len(p))]
    c.kv.keep(c.tree, [len(p) for p in paths], flat)
    assert c.kv.get_lengths(5) == [n + len(p) for n, p in zip(lens, paths)]
    for layer in range(3):
        for b in range(5):
            n, p = lens[b], paths[b]
            for got, old in zip(c.kv.read(layer, b, 0, 64), before[layer][b]):
                assert torch.equal(got[:n], old[:n]) and torch.equal(got[n:n + len(p)], old[[n + x for x in p]])
                assert torch.equal(got[n + len(trees[b]):], old[n + len(trees[b]):])
    # the device has the same lengths: the next trees' attention reads the kept rows as context
    ctx = [[x[:n + len(p)].to(tr.TORCH[dtype]) for x in c.kv.read(0, b, 0, 64)] for b, (n, p) in enumerate(zip(lens, paths))]
    c.lens, c.ctx = [n + len(p) for n, p in zip(lens, paths)], [ctx]
    c.check(c.attend())


def test_keep_refusals():
    c = Case("f32", 2, 1, 64, [10, 10], [[-1, 0, 1, 0], [-1]], max_seq=16)
    c.attend()
    for kept, path in (([2, 1], [0, 2, 0, 0, 0]), ([2, 0], [1, 2, 0, 0, 0]), ([5, 0], [0, 1, 2, 0, 0]), ([-1, 0], [0] * 5), ([3, 0], [0, 1, 3, 0, 0]),
                       ([2, 0], [0, 4, 0, 0, 0]), ([2, 0], [0, -1, 0, 0, 0])):
        with pytest.raises(hx.HexgenError) as e:
            c.kv.keep(c.tree, kept, path)
        assert e.value.status == 2
    assert c.kv.get_lengths(2) == [10, 10]
    for kept, path in (([1], [0] * 5), ([1, 1], [0] * 4)):
        with pytest.raises(ValueError):
            c.kv.keep(c.tree, kept, path)
    c.kv.keep(c.tree, [4 - 2, 1], [0, 3, -1, -1, 0])
    assert c.kv.get_lengths(2) == [12, 11]
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        with pytest.raises(hx.HexgenError) as e:
            c.kv.keep(c.tree, [1, 1], [0, -1, -1, -1, 0], stream=stream)
        assert e.value.status == 6
        with pytest.raises(hx.HexgenError) as e:
            c.tree.set([1, 1], [-1, -1], stream=stream)
        assert e.value.status == 6
    assert c.kv.get_lengths(2) == [12, 11]


# ---- a stage's layers ---------------------------------------------------------------------------------------------
def _stage(dtype, heads=8, kv=2, layers=2, tp=1, rank=0, hidden=1024, ffn=2816):
    cfg = StageConfig("tree", dtype, hidden, heads, kv, ffn, layers, tp, (rank,), batch=2, seed=77)
    w = [generate.layer_weights(cfg, l) for l in range(layers)]
    return cfg, make_gpu_stage(cfg, rank, w), make_oracle(cfg, rank, w)


@pytest.mark.parametrize("dtype,counts,tp", [("f32", [5, 9], 1), ("f32", [30, 25], 2), ("bf16", [1, 1], 1), ("bf16", [7, 12], 2), ("bf16", [40, 27], 1),
                                             ("f16", [2, 0], 1), ("f16", [20, 12], 1), ("f16", [100, 57], 2)])
def test_decode_tree_equals_decoding_every_path(dtype, counts, tp):
    """Each node's output is the last row of its sequence's prompt and path in the oracle; the decode kernels up to 32 rows, the prefill
    kernels beyond."""
    cfg, st, ora = _stage(dtype, heads=16, kv=4, tp=tp, rank=tp - 1)
    lens, trees = [19, 33], _trees(counts, seed=3)
    prompt, nodes = generate.hidden_rows(cfg, sum(lens)), generate.hidden_rows(cfg, sum(counts), stream_id=1)
    kv = st.kv_cache_create(2, 200)
    x = to_dev(prompt, cfg)
    st.prefill(kv, x, lens, torch.empty_like(x), torch.empty_like(x))
    tree = hx.Tree(2, 200)
    tree.set(counts, [p for t in trees for p in t])
    xin = to_dev(nodes, cfg)
    outp, outr = torch.empty_like(xin), torch.empty_like(xin)
    st.decode_tree(kv, tree, xin, outp, outr)
    again = torch.empty_like(xin)
    st.decode_tree(kv, tree, xin, again)                  # lengths unchanged, no residual asked for: the same once more
    torch.cuda.synchronize()
    assert torch.equal(again, outp) and kv.get_lengths(2) == lens
    ref_p, ref_r, row, first = [], [], 0, 0
    for b, t in enumerate(trees):
        for n in range(len(t)):
            path = tr.ancestors(t, n)[::-1]
            rows = np.concatenate([prompt[first:first + lens[b]].numpy(), nodes[[row + i for i in path]].numpy()])
            p, h = ora.prefill(ora.new_cache(1), rows, [len(rows)])
            ref_p.append(p[-1])
            ref_r.append(h[-1])
        row += len(t)
        first += lens[b]
    check("partial", outp.float().cpu().numpy(), np.stack(ref_p), TOL[dtype])
    check("residual", outr.float().cpu().numpy(), np.stack(ref_r), TOL[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_tree_recorded_and_replayed(dtype):
    cfg, st, _ = _stage(dtype)
    kv, tree = st.kv_cache_create(2, 100), hx.Tree(2, 64)
    prompt = to_dev(generate.hidden_rows(cfg, 30), cfg)
    st.prefill(kv, prompt, [10, 20], torch.empty_like(prompt))
    tree.set([6, 9], [p for t in _trees([6, 9]) for p in t])
    xs = [to_dev(generate.hidden_rows(cfg, 15, stream_id=2 + i), cfg) for i in range(4)]
    want = []
    for x in xs:
        want.append((torch.empty_like(x), torch.empty_like(x)))
        st.decode_tree(kv, tree, x, *want[-1])
    torch.cuda.synchronize()
    x, p, r = (torch.empty_like(xs[0]) for _ in range(3))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st.decode_tree(kv, tree, x, p, r)
    for _ in range(2):
        for y, (wp, wr) in zip(xs, want):
            x.copy_(y)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(p, wp) and torch.equal(r, wr)


def test_decode_tree_checks():
    cfg, st, _ = _stage("bf16")
    kv, tree = st.kv_cache_create(2, 40), hx.Tree(2, 64)
    tree.set([6, 9], [p for t in _trees([6, 9]) for p in t])
    x = to_dev(generate.hidden_rows(cfg, 15), cfg)
    with pytest.raises(hx.HexgenError) as e:
        st.decode_tree(kv, tree, x, torch.empty_like(x))
    assert e.value.status == 3
    kv.set_lengths([30, 32])
    with pytest.raises(hx.HexgenError) as e:
        st.decode_tree(kv, tree, x, torch.empty_like(x))
    assert e.value.status == 4
    with pytest.raises(ValueError, match="hidden_in"):
        st.decode_tree(kv, tree, x[:3], torch.empty_like(x))
    kv.set_lengths([3, 3])
    hx.lib.hexgen_stage_set_params(st.handle, 1e-5, 5e5)
    with pytest.raises(hx.HexgenError) as e:
        st.decode_tree(kv, tree, x, torch.empty_like(x))
    assert e.value.status == 3


# ---- together -----------------------------------------------------------------------------------------------------
def test_speculative_decoding_says_what_plain_decoding_says():
    """Embedding, stage and head of a tiny model: 24 tokens one by one, then the same prompt with drafted trees that hold the right
    continuation for a while, among wrong branches.  Ordinary decode steps go on from the kept rows."""
    cfg = StageConfig("spec", "f32", 512, 8, 2, 1408, 2, 1, (0,), batch=2, seed=9, vocab=500)
    st = make_gpu_stage(cfg, 0, [generate.layer_weights(cfg, l) for l in range(2)])
    hw = generate.head_weights(cfg)
    table = hw["embedding"].cuda()
    head = hx.Head(512, 500, 1, 0, "f32", cfg.rms_eps)
    head.load(hw["g_final"], hw["w_lm"])
    lens = [11, 23]
    prompt = torch.randint(0, 500, (sum(lens),), generator=torch.Generator().manual_seed(2), dtype=torch.int32).cuda()

    def prefill(kv):
        x = hx.embed_rows(table, prompt)
        p, r = torch.empty_like(x), torch.empty_like(x)
        st.prefill(kv, x, lens, p, r)
        last = [lens[0] - 1, sum(lens) - 1]
        return head.greedy(p[last].contiguous(), r[last].contiguous())[0]

    def decode(kv, step, tok):
        x = hx.embed_rows(table, tok)
        p, r = torch.empty_like(x), torch.empty_like(x)
        st.decode(kv, step, x, p, r)
        return head.greedy(p, r)[0]

    kv = st.kv_cache_create(2, 80)
    tok, plain = prefill(kv), []
    for step in range(24):
        plain.append(tok.cpu().tolist())
        tok = decode(kv, step, tok)
    plain.append(tok.cpu().tolist())
    plain = np.array(plain).T.tolist()                     # [sequence][token]

    kv2, tree = st.kv_cache_create(2, 80), hx.Tree(2, 32)
    tok = prefill(kv2).cpu().tolist()
    said = [[tok[0]], [tok[1]]]
    rng = np.random.default_rng(0)
    steps = 0
    while min(len(s) for s in said) < 16:
        counts, parents, draft = [], [], []
        for b in range(2):
            right = plain[b][len(said[b]):][:int(rng.integers(0, 5))]      # the true continuation, as far as this draft knows it
            par, toks, at = [-1], [said[b][-1]], 0
            for t in right:
                for _ in range(int(rng.integers(0, 3))):
                    par.append(at)
                    toks.append((t + 1 + int(rng.integers(0, 400))) % 500)
                par.append(at)
                toks.append(t)
                at = len(par) - 1
            counts.append(len(par))
            parents += par
            draft += toks
        tree.set(counts, parents)
        d = torch.tensor(draft, dtype=torch.int32, device="cuda")
        x = hx.embed_rows(table, d)
        p, r = torch.empty_like(x), torch.empty_like(x)
        st.decode_tree(kv2, tree, x, p, r)
        chosen, _ = head.greedy(p, r)
        kept, path, tokens = (v.cpu().tolist() for v in tree.accept(d, chosen))
        kv2.keep(tree, kept, path)
        row = 0
        for b in range(2):
            said[b] += tokens[row:row + kept[b]]
            row += counts[b]
        steps += 1
    assert steps < 15, "the drafted tokens were not taken"
    for b in range(2):
        n = min(len(said[b]), len(plain[b]))
        assert said[b][:n] == plain[b][:n]
    assert kv2.get_lengths(2) == [n + len(s) - 1 for n, s in zip(lens, said)]
    tok = torch.tensor([s[-1] for s in said], dtype=torch.int32, device="cuda")
    nxt = decode(kv2, 0, tok).cpu().tolist()
    for b in range(2):
        if len(said[b]) < len(plain[b]):
            assert nxt[b] == plain[b][len(said[b])]
