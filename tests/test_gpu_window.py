"""Windowed rows on the GPU against 64 bits: attention with sinks over the cache and the sums of its weights, one row to whole prompts."""
import numpy as np
import pytest
import torch

import paper_2311_11514_amd as hx
from tests import tree_reference as tr
from tests import window_reference as wr

pytestmark = pytest.mark.gpu


class Case:
    """A cache with contexts, and new rows for them; values as they are stored."""

    def __init__(self, dtype, hq, hkv, d, lens, counts, window, sinks, max_seq=None, layers=1, seed=0, fill=True):
        self.dtype, self.hq, self.hkv, self.d, self.lens, self.counts, self.window, self.sinks = dtype, hq, hkv, d, lens, counts, window, sinks
        self.stage = hx.Stage(hq * d, hq, hkv, 256, layers, 1, 0, dtype)
        self.kv = self.stage.kv_cache_create(len(lens), max_seq or max(n + c for n, c in zip(lens, counts)))
        g = torch.Generator().manual_seed(seed)
        td = tr.TORCH[dtype]
        self.ctx = [[[torch.randn(n, hkv, d, generator=g).to(td) for _ in range(2)] for n in lens] for _ in range(layers)]
        if fill:
            for layer in range(layers):
                for b, n in enumerate(lens):
                    if n:
                        self.kv.fill(layer, b, *self.ctx[layer][b])
        self.kv.set_lengths(lens)
        self.rows = sum(counts)
        self.q = torch.randn(self.rows, hq, d, generator=g).to(td)
        self.k, self.v = (torch.randn(self.rows, hkv, d, generator=g).to(td) for _ in range(2))
        self.before = torch.rand(len(lens), hkv, self.kv.max_seq, generator=g)

    def attend(self, layer=0, **kw):
        out = self.kv.window_attention(layer, self.q.cuda(), self.k.cuda(), self.v.cuda(), self.counts, window=self.window, sinks=self.sinks, **kw)
        torch.cuda.synchronize()
        return out

    def attend_both(self, **kw):
        weights = self.before.cuda()
        return self.attend(weights=weights, **kw), weights

    def reference(self, layer=0):
        """(o, bound of o, weights, bound of the weights)."""
        row, found = 0, []
        weights, bound = self.before.double().numpy().copy(), np.zeros(self.before.shape)
        for b, n in enumerate(self.counts):
            part = [x[row:row + n].double().numpy() for x in (self.q, self.k, self.v)]
            ctx = [x.double().numpy() for x in self.ctx[layer][b]]
            o, a, s, sums, scaled = wr.attention(part[0], ctx[0], ctx[1], part[1], part[2], self.window, self.sinks)
            m = self.lens[b] + n
            found.append((o, tr.attention_bound(o, a, s, self.dtype, self.d, m)))
            bound[b, :, :m] = wr.weights_bound(sums, scaled, weights[b, :, :m], self.d, m, n * self.hq // self.hkv)
            weights[b, :, :m] += sums
            row += n
        return np.concatenate([x[0] for x in found]), np.concatenate([x[1] for x in found]), weights, bound

    def check(self, out, weights=None):
        o, bound, w, w_bound = self.reference()
        off = np.abs(out.double().cpu().numpy() - o) / bound
        print(f"{self.dtype} {self.lens} {self.counts} {self.window} {self.sinks}: {off.max():.3f} of the bound", flush=True)
        assert off.max() <= 1, np.unravel_index(off.argmax(), off.shape)
        if weights is not None:
            far = np.abs(weights.double().cpu().numpy() - w)
            print(f"  weights: {(far[w_bound > 0] / w_bound[w_bound > 0]).max():.3f} of the bound", flush=True)
            assert np.all(far <= w_bound), np.argwhere(far > w_bound)[:4]


FEW = [
    (2, 2, 64, [0], [1], 1, 0),                            # one row, itself alone
    (8, 2, 64, [40], [1], 24, 4),
    (2, 1, 64, [31, 32, 33, 0], [1, 1, 1, 2], 5, 1),       # around the end of a tile
    (8, 1, 128, [63, 64, 1], [3, 0, 4], 32, 0),            # a sequence without a row
    (8, 1, 128, [500, 321], [4, 2], 33, 32),               # the first positions are a tile of their own, and then some
    (4, 4, 128, [100, 7], [8, 33], 16, 40),                # one head a group; more first positions than a context has
    (6, 2, 64, [129], [17], None, 0),                      # groups of three; no window
    (16, 1, 128, [50, 300], [7, 2], 64, 33),               # the widest group
    (8, 1, 128, [300, 31, 5], [16, 9, 40], 100, 3),
    (8, 8, 64, [95], [64], 31, 2),
    (4, 1, 64, [20, 3], [100, 256], 50, 70),
    (2, 1, 64, [700, 650], [1, 1], 1, 1),                  # the first and itself
    (1, 1, 128, [64, 95, 96], [1, 31, 33], 64, 64),
    (1, 1, 128, [64, 95, 100], [1, 1, 1], 40, 2),          # an odd number of rows and heads
    (10, 5, 64, [200, 10], [2, 3], (1 << 31) - 1, (1 << 31) - 1),      # a window and sinks beyond everything
]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,lens,counts,window,sinks", FEW)
def test_attention_and_weights_match_64_bits(dtype, hq, hkv, d, lens, counts, window, sinks):
    c = Case(dtype, hq, hkv, d, lens, counts, window, sinks)
    alone = c.attend()
    out, weights = c.attend_both()
    c.check(out, weights)
    assert torch.equal(out, alone)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,lens,counts,window,sinks", [
    (2, 1, 128, [2900], [2], None, 0),                     # cut into runs
    (2, 1, 128, [3900], [1], 2500, 100),
    (4, 1, 64, [2100, 5, 1000], [13, 16, 2], 1800, 5),     # a context that is shorter than one run
    (8, 1, 128, [2500, 0, 700], [26, 20, 30], 2000, 33),   # rows of several blocks, cut
])
def test_long_contexts_in_runs_match_64_bits(dtype, hq, hkv, d, lens, counts, window, sinks):
    c = Case(dtype, hq, hkv, d, lens, counts, window, sinks, seed=3)
    out, weights = c.attend_both()
    c.check(out, weights)
    again, more = c.attend_both()                          # the same bits, whoever joined the runs, and with the rows in the cache by now
    assert torch.equal(again, out) and torch.equal(more, weights)


WIDE = [                                                   # enough rows that blocks share tiles
    (64, 8, 128, [0, 31, 300, 503], [64, 65, 70, 130], 100, 33),
    (64, 8, 64, [0, 31, 300, 203], [96, 65, 120, 130], None, 0),
    (64, 8, 64, [64, 1, 0, 0], [96, 65, 33, 200], 1, 0),
    (16, 16, 64, [0, 77], [900, 600], 128, 5),
    (24, 8, 128, [5, 260, 0], [701, 0, 600], 32, 64),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hkv,d,lens,counts,window,sinks", WIDE)
def test_blocks_that_share_tiles_match_64_bits(dtype, hq, hkv, d, lens, counts, window, sinks):
    c = Case(dtype, hq, hkv, d, lens, counts, window, sinks, seed=8)
    out, weights = c.attend_both()
    c.check(out, weights)
    assert torch.equal(c.attend(), out)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,lens,counts,window,sinks", [
    (8, 1, 128, [300, 31, 70], [4, 1, 2], 40, 3),
    (4, 2, 64, [190, 64, 0], [20, 33, 70], 33, 32),
    (64, 8, 64, [130, 77, 0, 300], [64, 65, 70, 100], 45, 7),      # 16 bits: shared tiles
])
def test_what_a_row_does_not_attend_has_no_influence(dtype, hq, hkv, d, lens, counts, window, sinks):
    """NaN and infinities in the slots between the first ones and every window, behind the rows, and in the rows that the others' windows end before."""
    c = Case(dtype, hq, hkv, d, lens, counts, window, sinks, max_seq=max(n + m for n, m in zip(lens, counts)) + 70, seed=5, fill=False)
    for b, n in enumerate(lens):
        k, v = (torch.full((c.kv.max_seq, hkv, d), float("nan")) for _ in range(2))
        v[::3] = float("inf")
        k[1::2] = -float("inf")
        first = n - window + 1                             # of what the first row's window reaches
        seen = [j for j in range(n) if j < sinks or j >= first]
        k[seen], v[seen] = c.ctx[0][b][0][seen].float(), c.ctx[0][b][1][seen].float()
        c.kv.fill(0, b, k, v)
    c.kv.set_lengths(lens)
    out, weights = c.attend_both()
    c.check(out, weights)
    # a row that nobody behind its window may notice
    row = 0
    touched = torch.ones(c.rows, dtype=torch.bool)
    q, k, v = c.q.cuda(), c.k.clone(), c.v.clone()
    for b, m in enumerate(counts):
        if m > 0:
            at = m // 3
            if lens[b] + at >= sinks:
                k[row + at], v[row + at] = float("nan"), float("inf")
                touched[row + at:row + min(m, at + window)] = False
        row += m
    got = c.kv.window_attention(0, q, k.cuda(), v.cuda(), counts, window=window, sinks=sinks)
    # Tiles with a value that is not finite are multiplied out element by element: the same terms in another order, which the bound against 64 bits
    # covers in either (it counts a rounding for every position that is added up), but not the same bits.
    o, bound, _, _ = c.reference()
    assert np.all((np.abs(got.double().cpu().numpy() - o) <= bound)[touched.numpy()])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,lens,counts,window,sinks", [(4, 1, 64, [100], [3], 10, 2), (8, 1, 128, [70, 3], [20, 9], 33, 1), (64, 8, 64, [130, 0], [200, 70], 45, 7)])
def test_a_row_of_nan_spoils_the_weights_of_what_it_attends_alone(dtype, hq, hkv, d, lens, counts, window, sinks):
    c = Case(dtype, hq, hkv, d, lens, counts, window, sinks, seed=6)
    out, weights = c.attend_both()
    at = counts[0] - 2
    c.q[at, 0] = float("nan")                              # the first query head of one row of the first sequence
    got, spoiled = c.attend_both()
    seen = wr.visible(lens[0] + at, window, sinks)
    rest = torch.ones_like(weights, dtype=torch.bool)
    rest[0, 0, seen] = False
    assert torch.isnan(spoiled[0, 0, seen]).all() and torch.equal(spoiled[rest], weights[rest])
    same = torch.ones_like(out, dtype=torch.bool)
    same[at, 0] = False
    assert torch.equal(got[same], out[same]) and torch.isnan(got[at, 0]).all()


@pytest.mark.parametrize("dtype,power", [(t, p) for t, most in (("bf16", 14), ("f16", 11), ("f32", 14)) for p in (5, 10, most)])
@pytest.mark.parametrize("hq,hkv,lens,counts", [(8, 1, [90], [2]), (64, 8, [70, 0], [200, 70])])
def test_scores_far_from_zero(dtype, hq, hkv, lens, counts, power):
    """Scores of 2^10 and more, the largest of a row far in front of its others: the row is that position's value.  The position's key is the row's query times 2^power in every
    group's first head; whatever comes after it in the tiles, and the bases that the largest scores need, change nothing."""
    c = Case(dtype, hq, hkv, 64, lens, counts, 64, 3, seed=12)
    group = hq // hkv
    unit = torch.sign(c.q[:, ::group].float())
    c.q[:, :] = (unit * 2.0 ** power).repeat_interleave(group, 1).to(c.q.dtype)
    c.k[:, :] = (unit * 2.0 ** 4).to(c.k.dtype)              # a row's own key is the one that fits: score 2^(power + 4) 64 / 8; any other's is smaller by 2^(power + 5) / 8 a sign
    for b in range(len(lens)):
        c.ctx[0][b][0] = torch.zeros_like(c.ctx[0][b][0])
        if lens[b]:
            c.kv.fill(0, b, *c.ctx[0][b])
    c.kv.set_lengths(lens)
    out, weights = c.attend_both()
    assert torch.equal(out.cpu(), c.v.repeat_interleave(group, 1))
    row = 0
    for b, (n, m) in enumerate(zip(lens, counts)):
        gathered = (weights[b].cpu() - c.before[b])[:, :n + m]
        assert torch.allclose(gathered[:, n:], torch.full((hkv, m), float(group)), rtol=0, atol=1e-4) and torch.allclose(gathered[:, :n], torch.zeros(hkv, n), rtol=0, atol=1e-6)
        row += m


def test_infinite_values_that_are_attended_stay():
    c = Case("f32", 4, 2, 64, [40], [3], 16, 0)
    c.v[1, 0, 5] = float("inf")
    out = c.attend()
    assert torch.isinf(out[1:, :2, 5]).all() and torch.isfinite(out[0]).all() and torch.isfinite(out[:, 2:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,lens,counts", [(8, 1, 128, [33, 0, 62], [4, 3, 2]), (8, 2, 64, [3, 40, 95], [40, 0, 33]), (64, 8, 64, [7, 64], [200, 65]),
                                                  (2, 2, 128, [31, 32], [1, 1])])
def test_rows_join_the_cache_and_nothing_else_changes(dtype, hq, hkv, d, lens, counts):
    c = Case(dtype, hq, hkv, d, lens, counts, 20, 3, max_seq=300, layers=2, seed=2)
    before = [[c.kv.read(layer, b, 0, 300) for b in range(len(lens))] for layer in range(2)]
    c.attend(layer=1)
    row = 0
    for b, (n, m) in enumerate(zip(lens, counts)):
        for got, old, new in zip(c.kv.read(1, b, 0, 300), before[1][b], (c.k, c.v)):
            assert torch.equal(got[:n], old[:n]) and torch.equal(got[n:n + m], new[row:row + m].float()) and torch.equal(got[n + m:], old[n + m:])
        for got, old in zip(c.kv.read(0, b, 0, 300), before[0][b]):
            assert torch.equal(got, old)
        row += m
    assert c.kv.get_lengths(len(lens)) == lens             # not committed
    c.kv.commit(counts, len(lens))
    assert c.kv.get_lengths(len(lens)) == [n + m for n, m in zip(lens, counts)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_a_fused_projection(dtype):
    """q, k and v as parts of rows of one tensor, and rows far apart."""
    c = Case(dtype, 8, 2, 64, [50, 9], [3, 2], 17, 2)
    want = c.attend()
    fused = torch.cat([x.flatten(1) for x in (c.q, c.k, c.v)], 1).cuda()
    q, k, v = fused[:, :512], fused[:, 512:640], fused[:, 640:]
    assert torch.equal(c.kv.window_attention(0, q, k, v, c.counts, window=17, sinks=2), want)
    apart = torch.zeros(5, 3, 8, 64, dtype=q.dtype, device="cuda")
    apart[:, 1] = c.q.cuda()
    out = torch.zeros(5, 8, 64, dtype=q.dtype, device="cuda")
    assert c.kv.window_attention(0, apart[:, 1], k, v, c.counts, window=17, sinks=2, out=out) is out
    assert torch.equal(out, want)


def test_one_row_each_needs_no_counts():
    c = Case("bf16", 8, 1, 128, [100, 3, 40], [1, 1, 1], 32, 1)
    want, weights = c.attend_both()
    more = c.before.cuda()
    assert torch.equal(c.kv.window_attention(0, c.q.cuda(), c.k.cuda(), c.v.cuda(), window=32, sinks=1, weights=more), want)
    assert torch.equal(more, weights)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_sequences_than_a_launch_takes(dtype):
    lens = [(7 * i) % 90 for i in range(300)]
    counts = [1 + i % 3 if i % 11 else 0 for i in range(300)]
    c = Case(dtype, 2, 1, 64, lens, counts, 24, 2, seed=11)
    out, weights = c.attend_both()
    c.check(out, weights)


def test_a_launch_of_sequences_without_rows():
    counts = [0] * 256 + [2, 0, 1]
    c = Case("bf16", 2, 1, 64, [30] * 259, counts, 8, 1, seed=13)
    out, weights = c.attend_both()
    c.check(out, weights)
    assert torch.equal(weights[:256].cpu(), c.before[:256])


def test_another_stream_and_the_order_that_the_caller_makes():
    c = Case("bf16", 8, 1, 128, [1500], [1], 900, 4)
    want, weights = c.attend_both()
    stream = torch.cuda.Stream()
    q, k, v, more = c.q.cuda(), c.k.cuda(), c.v.cuda(), c.before.cuda()
    stream.wait_stream(torch.cuda.current_stream())
    got = c.kv.window_attention(0, q, k, v, window=900, sinks=4, weights=more, stream=stream)
    stream.synchronize()
    assert torch.equal(got, want) and torch.equal(more, weights)


@pytest.mark.parametrize("dtype,hq,hkv,lens,counts", [("bf16", 8, 1, [1000, 40], [1, 1]), ("f16", 64, 8, [40, 0], [164, 170]), ("f32", 8, 2, [300, 17], [2, 1])])
def test_recorded_and_replayed(dtype, hq, hkv, lens, counts):
    """A replay appends, attends and gathers at the lengths that hold then."""
    c = Case(dtype, hq, hkv, 64, lens, counts, 50, 4, max_seq=1200 + max(counts))
    q, k, v = c.q.cuda(), c.k.cuda(), c.v.cuda()
    weights, out = torch.zeros(2, hkv, c.kv.max_seq, device="cuda"), torch.zeros_like(q)
    call = lambda: c.kv.window_attention(0, q, k, v, counts, window=50, sinks=4, weights=weights, out=out)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for step in range(3):
        now = [n + 3 * step for n in lens]
        for b in range(2):
            c.ctx[0][b] = [torch.randn(now[b], hkv, 64, generator=torch.Generator().manual_seed(step)).to(q.dtype) for _ in range(2)]
            if now[b]:
                c.kv.fill(0, b, *c.ctx[0][b])
        c.kv.set_lengths(now)
        c.lens = now
        weights.copy_(c.before)
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        c.check(out, weights)
        eager, more = c.attend_both()
        assert torch.equal(eager, out) and torch.equal(more, weights)


def test_a_replay_leaves_out_what_would_pass_the_cache():
    """The committed lengths come to stand where the recorded rows do not fit any more: rows beyond are neither stored nor gathered."""
    c = Case("bf16", 4, 2, 64, [20, 5], [3, 3], 16, 1, max_seq=40)
    q, k, v = c.q.cuda(), c.k.cuda(), c.v.cuda()
    weights, out = torch.zeros(2, 2, 40, device="cuda"), torch.zeros_like(q)
    call = lambda: c.kv.window_attention(0, q, k, v, c.counts, window=16, sinks=1, weights=weights, out=out)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    full = [torch.randn(40, 2, 64).to(q.dtype) for _ in range(2)]
    c.kv.fill(0, 0, *full)
    c.kv.set_lengths([38, 5])
    weights.zero_()
    out.fill_(7)
    graph.replay()
    torch.cuda.synchronize()
    got = c.kv.read(0, 0, 0, 40)
    assert torch.equal(got[0][38:], c.k[:2].float()) and torch.equal(got[0][:38], full[0][:38].float())
    assert (out[2] == 7).all() and torch.isfinite(out).all()
    assert abs(float(weights[0].sum()) - 2 * 4) < 1e-4 and abs(float(weights[1].sum()) - 3 * 4) < 1e-4
    with pytest.raises(hx.HexgenError) as e:
        call()
    assert e.value.status == 4


def test_two_recordings_share_the_workspace():
    """Contexts in runs, recorded twice, with and without weights, replayed in turn with eager calls between."""
    c = Case("bf16", 8, 1, 128, [3500, 2000], [2, 1], None, 0, seed=4)
    q, k, v = c.q.cuda(), c.k.cuda(), c.v.cuda()
    want, gathered = c.attend_both()
    graphs, outs, weights = [], [], c.before.cuda()
    for w in (None, weights):
        out, graph = torch.zeros_like(q), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.kv.window_attention(0, q, k, v, c.counts, weights=w, out=out)
        graphs.append(graph)
        outs.append(out)
    for _ in range(3):
        weights.copy_(c.before)
        for g, o in zip(graphs, outs):
            o.zero_()
            g.replay()
        assert torch.equal(c.attend(), want)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want) and torch.equal(weights, gathered)


def test_refusals():
    c = Case("bf16", 4, 2, 64, [10, 20], [2, 1], 8, 1, max_seq=24)
    q, k, v = c.q.cuda(), c.k.cuda(), c.v.cuda()
    call = c.kv.window_attention
    for args, kw, status in (((0, q, k, v, [2, 1]), dict(window=0), 1), ((0, q, k, v, [2, 1]), dict(window=-5), 1), ((0, q, k, v, [2, 1]), dict(sinks=-1), 1),
                             ((1, q, k, v, [2, 1]), {}, 1), ((-1, q, k, v, [2, 1]), {}, 1), ((0, q, k, v, [4, -1]), {}, None), ((0, q, k, v, [3]), {}, 3),
                             ((0, q, k, v), {}, 3), ((0, q, k, v, [1, 1, 1]), {}, 3)):
        with pytest.raises((hx.HexgenError, ValueError)) as e:
            call(*args, **kw)
        assert status is None or e.value.status == status
    five = [torch.cat((x, x))[:5].contiguous() for x in (q, k, v)]
    with pytest.raises(hx.HexgenError) as e:
        call(0, *five, [0, 5])                               # 25 slots of 24
    assert e.value.status == 4
    with pytest.raises(hx.HexgenError) as e:
        call(0, q[:0], k[:0], v[:0], [0, 0])
    assert e.value.status in (1, 2)
    for bad in (torch.zeros(2, 2, 25, device="cuda"), torch.zeros(2, 2, 24, device="cuda", dtype=torch.float64), torch.zeros(2, 2, 24),
                torch.zeros(2, 2, 48, device="cuda")[..., ::2], torch.zeros(3, 2, 24, device="cuda")):
        with pytest.raises(ValueError, match="weights"):
            call(0, q, k, v, [2, 1], weights=bad)
    for name, t in (("q", (q.float(), k, v)), ("k", (q, k[:, :1], v)), ("v", (q, k, v.cpu()))):
        with pytest.raises(ValueError, match=name):
            call(0, *t, [2, 1])
    with pytest.raises(ValueError, match="window"):
        call(0, q, k, v, [2, 1], window=1 << 31)
    unaligned = torch.zeros(3 * 256 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(3, 4, 64)
    with pytest.raises(hx.HexgenError) as e:
        call(0, unaligned, k, v, [2, 1])
    assert e.value.status == 1
    far = torch.zeros((1 << 24) + 8 + 256, dtype=torch.bfloat16, device="cuda")
    for apart, ok in ((1 << 24, True), ((1 << 24) + 8, False)):  # of 2 rows, elements
        rows = far.as_strided((2, 4, 64), (apart, 64, 1))
        if ok:
            rows.copy_(q[:2])
            assert torch.equal(call(0, rows, k[:2], v[:2], [1, 1], window=8), call(0, q[:2], k[:2], v[:2], [1, 1], window=8))
            continue
        with pytest.raises(hx.HexgenError) as e:
            call(0, rows, k[:2], v[:2], [1, 1])
        assert e.value.status == 1
    assert c.kv.get_lengths(2) == [10, 20]
    fresh = c.stage.kv_cache_create(2, 24)
    with pytest.raises(hx.HexgenError) as e:
        fresh.window_attention(0, q, k, v, [2, 1])
    assert e.value.status == 3
    c.check(c.attend())                                      # none of it changed anything
