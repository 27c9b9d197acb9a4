"""Eviction on the GPU: which slots stay, that their rows and weights move as they are (keys turned back where asked), in place and into another cache."""
import numpy as np
import pytest
import torch

import paper_2311_11514_amd as hx
from tests import tree_reference as tr
from tests import window_reference as wr

pytestmark = pytest.mark.gpu

THETA = 10000.0


class Case:
    def __init__(self, dtype, layers, hq, hkv, d, lens, max_seq, seed=0, kind="random"):
        self.dtype, self.layers, self.hkv, self.d, self.lens, self.max_seq = dtype, layers, hkv, d, lens, max_seq
        self.stage = hx.Stage(hq * d, hq, hkv, 256, layers, 1, 0, dtype)
        self.kv = self.stage.kv_cache_create(len(lens), max_seq)
        g = torch.Generator().manual_seed(seed)
        shape = (layers, len(lens), max_seq, hkv, d)
        self.k, self.v = (torch.randn(*shape, generator=g).to(tr.TORCH[dtype]).float() for _ in range(2))
        for layer in range(layers):
            for b in range(len(lens)):
                self.kv.fill(layer, b, self.k[layer, b], self.v[layer, b])
        self.kv.set_lengths(lens)
        shape = (layers, len(lens), hkv, max_seq)
        w = torch.exp(2 * torch.randn(*shape, generator=g) - 3)
        if kind == "ties":                                   # few values: equal ones at every border
            w = torch.randint(0, 3, shape, generator=g).float()
        elif kind == "equal":
            w = torch.full(shape, 0.25)
        elif kind == "close":                                # neighbours in the last bits, every byte of the number decides somewhere
            w = (torch.randint(0x3f7fff00, 0x3f800100, shape, generator=g, dtype=torch.int32)).view(torch.float32)
        elif kind == "wild":
            w = torch.randint(-1 << 31, (1 << 31) - 1, shape, generator=g, dtype=torch.int64).to(torch.int32).view(torch.float32)
            w[..., ::7] = 0.0
            w[..., 1::7] = -0.0
            w[..., 2::11] = float("nan")
            w[..., 3::13] = float("inf")
            w[..., 4::13] = -float("inf")
        self.w = w

    def check(self, keep, sinks, recent, weights=True, rotate=False, into=None):
        """into: None in place, else the positions of the other cache."""
        batch, size = len(self.lens), self.max_seq if into is None else into
        dst = None if into is None else self.stage.kv_cache_create(batch + (into % 2), into)
        if dst is not None:
            for layer in range(self.layers):
                for b in range(dst.max_batch):
                    dst.fill(layer, b, torch.full((into, self.hkv, self.d), 5.0), torch.full((into, self.hkv, self.d), 6.0))
        w = self.w.cuda() if weights else None
        slots, left = self.kv.evict(keep, sinks=sinks, recent=recent, weights=w, rotate=rotate, into=dst)
        assert slots.shape == (self.layers, batch, self.hkv, size) and slots.dtype == torch.int32
        assert (left is None) == (not weights) and (into is not None or left is w)
        if weights and into is not None:
            assert torch.equal(w.view(torch.int32), self.w.cuda().view(torch.int32))
        cache = self.kv if dst is None else dst
        kept = [min(n, keep) for n in self.lens]
        assert cache.get_lengths(batch) == kept and self.kv.get_lengths(batch) == (kept if dst is None else self.lens)
        slots = slots.cpu().numpy()
        left = None if left is None else left.cpu().numpy()
        for layer in range(self.layers):
            for b, n in enumerate(self.lens):
                k, v = (x.numpy() for x in cache.read(layer, b, 0, size))
                old_k, old_v = self.k[layer, b].numpy(), self.v[layer, b].numpy()
                for h in range(self.hkv):
                    row = self.w[layer, b, h].numpy()
                    want = wr.chosen(n, keep, sinks, recent, row if weights else None)
                    assert slots[layer, b, h].tolist() == want + [-1] * (size - len(want)), (layer, b, h)
                    if weights:
                        assert np.array_equal(left[layer, b, h, :len(want)].view(np.int32), row[want].view(np.int32)) and not left[layer, b, h, len(want):].any()
                    m = len(want)
                    assert np.array_equal(v[:m, h], old_v[want, h])
                    if not rotate:
                        assert np.array_equal(k[:m, h], old_k[want, h])
                    else:
                        moved = np.asarray(want) - np.arange(m)
                        turned = wr.turned_back(old_k[want, h][:, None], moved, THETA)[:, 0]
                        # the rotation's three roundings and the tables' one, on a pair's two products, then the one to the cache's type
                        pair = np.abs(old_k[want, h]) + np.abs(np.roll(old_k[want, h], self.d // 2, axis=1))
                        bound = 4 * tr.UNIT["f32"] * pair + (tr.UNIT[self.dtype] if self.dtype != "f32" else 0.0) * (np.abs(turned) + 4 * tr.UNIT["f32"] * pair) + 2.0 ** -25
                        assert np.all(np.abs(k[:m, h] - turned) <= bound)
                        assert np.array_equal(k[:m, h][moved == 0], old_k[want, h][moved == 0])
                    # what lies behind them is as it was
                    rest_k, rest_v = (old_k[m:, h], old_v[m:, h]) if dst is None else (5.0, 6.0)
                    assert np.all(k[m:, h] == rest_k) and np.all(v[m:, h] == rest_v)
        if dst is not None and dst.max_batch > batch:
            k, v = dst.read(0, batch, 0, size)
            assert (k == 5).all() and (v == 6).all()
        return cache


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("keep,sinks,recent", [(40, 4, 8), (1, 0, 0), (1, 1, 0), (1, 0, 1), (64, 0, 0), (33, 33, 0), (50, 0, 50), (50, 20, 30), (97, 1, 31), (200, 3, 4)])
@pytest.mark.parametrize("into", [None, 200])
def test_kept_slots(dtype, keep, sinks, recent, into):
    c = Case(dtype, 2, 4, 2, 64, [150, 40, 7, 0, 97], 200, seed=keep)
    c.check(keep, sinks, recent, into=into)


@pytest.mark.parametrize("kind", ["ties", "equal", "close", "wild"])
@pytest.mark.parametrize("lens,max_seq,keep,sinks,recent", [([900, 333], 900, 200, 5, 20), ([5000, 2047], 5001, 2048, 0, 0), ([2049, 4096], 4096, 100, 1, 1000 - 950)])
def test_weights_that_are_hard_to_order(kind, lens, max_seq, keep, sinks, recent):
    Case("f32", 1, 2, 1, 64, lens, max_seq, seed=1, kind=kind).check(keep, sinks, recent, into=keep)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("into", [None, 131])
@pytest.mark.parametrize("weights", [True, False])
def test_rotated_keys(dtype, d, into, weights):
    c = Case(dtype, 2, 4, 2, d, [300, 131, 160, 20], 320, seed=3)
    c.check(130, 4, 30, weights=weights, rotate=True, into=into)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_first_and_newest_without_weights(dtype):
    c = Case(dtype, 1, 8, 1, 128, [260, 64, 65], 260, seed=5)
    c.check(64, 4, 10, weights=False)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d,rotate", [(64, True), (128, False), (128, True)])
def test_many_rows_in_place(dtype, d, rotate):
    """Rows that one block moves in several steps, some of which move nothing."""
    c = Case(dtype, 1, 4, 2, d, [900, 611, 450], 900, seed=13)
    c.check(610, 200, 100, rotate=rotate)


def test_twice_in_place():
    """What an eviction leaves is a context like any other: it can be evicted from again."""
    c = Case("bf16", 1, 2, 2, 64, [220, 90], 256, seed=7)
    w = c.w.cuda()
    first, _ = c.kv.evict(100, sinks=2, recent=10, weights=w)
    second, _ = c.kv.evict(37, sinks=2, recent=10, weights=w)
    assert c.kv.get_lengths(2) == [37, 37]
    k, v = c.kv.read(0, 0, 0, 37)
    for h in range(2):
        at = first[0, 0, h].long()[second[0, 0, h, :37].long()].cpu()
        assert torch.equal(k[:, h], c.k[0, 0, at, h]) and torch.equal(v[:, h], c.v[0, 0, at, h])
        assert torch.equal(w[0, 0, h, :37].cpu(), c.w[0, 0, h, at]) and not w[0, 0, h, 37:].any()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rotate", [False, True])
def test_attention_reads_what_is_left(dtype, rotate):
    """Gather weights over a context, evict by them, attend: the device's lengths and the moved rows are the next call's context."""
    layers, lens, max_seq, keep = 2, [180, 64, 300], 330, 64
    c = Case(dtype, layers, 8, 2, 64, lens, max_seq, seed=9)
    small = c.stage.kv_cache_create(3, keep + 2)
    g = torch.Generator().manual_seed(1)
    td = tr.TORCH[dtype]
    weights = torch.zeros(layers, 3, 2, max_seq, device="cuda")
    new = [[torch.randn(6, x, 64, generator=g).to(td).cuda() for x in (8, 2, 2)] for _ in range(layers)]
    for layer in range(layers):
        c.kv.window_attention(layer, *new[layer], counts=[2, 1, 3], window=90, sinks=3, weights=weights[layer])
    c.kv.commit([2, 1, 3], 3)
    slots, left = c.kv.evict(keep, sinks=3, recent=8, weights=weights, rotate=rotate, into=small)
    assert torch.equal(left.sort(-1).values[..., -keep:].sum(-1) > 0, torch.ones(layers, 3, 2, dtype=torch.bool, device="cuda"))
    assert small.get_lengths(3) == [64, 64, 64]
    for layer in range(layers):
        q, k, v = [torch.randn(3, x, 64, generator=g).to(td) for x in (8, 2, 2)]
        out = small.window_attention(layer, q.cuda(), k.cuda(), v.cuda())
        for b in range(3):
            ctx = [x.double().numpy() for x in small.read(layer, b, 0, keep)]
            o, a, s, _, _ = wr.attention(*(x[b:b + 1].double().numpy() if i == 0 else x for i, x in enumerate((q, *ctx))), k[b:b + 1].double().numpy(), v[b:b + 1].double().numpy(), None, 0)
            assert np.all(np.abs(out[b:b + 1].double().cpu().numpy() - o) <= tr.attention_bound(o, a, s, dtype, 64, keep + 1))
            at = slots[layer, b, 0, :keep].long().cpu()
            want = torch.cat((c.v[layer, b, :lens[b]], new[layer][2][{0: slice(0, 2), 1: slice(2, 3), 2: slice(3, 6)}[b]].float().cpu()))[at, 0]
            assert torch.equal(small.read(layer, b, 0, keep)[1][:, 0], want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_drafted_trees_over_what_is_left(dtype):
    """The other attention over the cache takes the lengths and rows of an eviction as well: a tree of one node is a row."""
    c = Case(dtype, 1, 8, 2, 64, [180, 64, 300], 330, seed=15)
    c.kv.evict(70, sinks=3, recent=8, weights=c.w.cuda())
    g = torch.Generator().manual_seed(2)
    td = tr.TORCH[dtype]
    q, k, v = [torch.randn(3, x, 64, generator=g).to(td) for x in (8, 2, 2)]
    tree = hx.Tree(3, 3)
    tree.set([1, 1, 1], [-1, -1, -1])
    outs = [c.kv.tree_attention(0, tree, q.cuda(), k.cuda(), v.cuda()), c.kv.window_attention(0, q.cuda(), k.cuda(), v.cuda())]
    for b, n in enumerate((70, 64, 70)):
        ctx = [x.double().numpy() for x in c.kv.read(0, b, 0, n)]
        o, a, s, _, _ = wr.attention(q[b:b + 1].double().numpy(), *ctx, k[b:b + 1].double().numpy(), v[b:b + 1].double().numpy(), None, 0)
        for out in outs:
            assert np.all(np.abs(out[b:b + 1].double().cpu().numpy() - o) <= tr.attention_bound(o, a, s, dtype, 64, n + 1))


def test_more_layers_and_heads_than_a_grid_dimension():
    """66 layers x 63 sequences x 16 heads: 66528 units."""
    stage = hx.Stage(16 * 64, 16, 16, 256, 66, 1, 0, "bf16")
    kv = stage.kv_cache_create(63, 32)
    kv.set_lengths([7] * 63)
    w = torch.arange(32, device="cuda").float().expand(66, 63, 16, 32).contiguous()
    slots, left = kv.evict(3, sinks=1, weights=w)
    assert kv.get_lengths(63) == [3] * 63
    assert torch.equal(slots[..., :4], torch.tensor([0, 5, 6, -1], dtype=torch.int32, device="cuda").expand(66, 63, 16, 4)) and (slots[..., 4:] == -1).all()
    assert torch.equal(left[..., :4], torch.tensor([0., 5., 6., 0.], device="cuda").expand(66, 63, 16, 4))


def test_another_stream():
    c = Case("bf16", 1, 8, 1, 128, [500], 512, seed=2)
    small = c.stage.kv_cache_create(1, 128)
    w = c.w.cuda()
    want, left = c.kv.evict(100, sinks=2, recent=20, weights=w, into=small)
    k, v = small.read(0, 0, 0, 100)
    small.reset()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    slots, more = c.kv.evict(100, sinks=2, recent=20, weights=w, into=small, stream=stream)
    stream.synchronize()
    assert torch.equal(slots, want) and torch.equal(more, left)
    assert all(torch.equal(a, b) for a, b in zip(small.read(0, 0, 0, 100), (k, v)))


def test_refusals():
    c = Case("f32", 1, 4, 2, 64, [30, 9], 40)
    other = hx.Stage(256, 4, 2, 256, 1, 1, 0, "f32").kv_cache_create(2, 40)
    tight, few, small = c.stage.kv_cache_create(2, 19), c.stage.kv_cache_create(1, 40), c.stage.kv_cache_create(2, 20)
    w = c.w.cuda()
    for kw, status in ((dict(keep=0), 1), (dict(keep=-3), 1), (dict(keep=20, sinks=-1), 1), (dict(keep=20, recent=-1), 1), (dict(keep=20, sinks=10, recent=11), 1),
                       (dict(keep=20, into=other), 1), (dict(keep=20, into=tight), 4), (dict(keep=20, into=few), 4), (dict(keep=41, into=small), 4)):
        with pytest.raises(hx.HexgenError) as e:
            c.kv.evict(**kw)
        assert e.value.status == status
    for bad in (w[:, :1].contiguous(), w.double(), w.cpu(), w.transpose(2, 3)):
        with pytest.raises(ValueError, match="weights"):
            c.kv.evict(20, weights=bad)
    for name in ("keep", "sinks", "recent"):
        with pytest.raises(ValueError, match=name):
            c.kv.evict(**{"keep": 20, name: 1 << 32})
    empty = c.stage.kv_cache_create(2, 40)
    with pytest.raises(hx.HexgenError) as e:
        empty.evict(20)
    assert e.value.status == 3
    graph = torch.cuda.CUDAGraph()
    stream = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        with pytest.raises(hx.HexgenError) as e:
            c.kv.evict(20, weights=w, into=small, stream=stream)
        assert e.value.status == 6
    out = torch.zeros(1, 2, 2, 40, dtype=torch.int32, device="cuda")
    call = hx.lib.hexgen_kv_cache_evict
    assert call(c.kv.handle, small.handle, 20, 0, 0, w.data_ptr(), None, 0, out.data_ptr(), None) == 1
    assert call(c.kv.handle, small.handle, 20, 0, 0, None, w.data_ptr(), 0, out.data_ptr(), None) == 1
    assert call(c.kv.handle, small.handle, 20, 0, 0, w.data_ptr(), w.data_ptr(), 0, out.data_ptr(), None) == 1
    assert call(c.kv.handle, small.handle, 20, 0, 0, None, None, 0, out.data_ptr() + 2, None) == 1
    assert c.kv.get_lengths(2) == [30, 9] and torch.equal(w, c.w.cuda())
    # keys rotated under another theta than the stage has now
    c.stage2 = hx.Stage(256, 4, 2, 256, 1, 1, 0, "f32")
    kv = c.stage2.kv_cache_create(1, 40)
    kv.set_lengths([30])
    hx.lib.hexgen_stage_set_params(c.stage2.handle, 1e-5, 500.0)
    with pytest.raises(hx.HexgenError) as e:
        kv.evict(20, rotate=True)
    assert e.value.status == 3
    kv.evict(20)
    assert kv.get_lengths(1) == [20]
