"""A stage's layers over windowed rows: against the 64-bit stage with the same window, against prefill and decode where there is none, and as a stream that
gathers weights, evicts by them and goes on."""
import numpy as np
import pytest
import torch

import paper_2311_11514_amd as hx
from tests import window_reference as wr
from tests.helpers import TOL, check, make_gpu_stage, to_dev
from workloads import StageConfig, generate

pytestmark = pytest.mark.gpu


def _stage(dtype, window, sinks, heads=16, kv=4, layers=2, tp=1, rank=0, hidden=1024, ffn=2816, batch=2):
    cfg = StageConfig("window", dtype, hidden, heads, kv, ffn, layers, tp, (rank,), batch=batch, seed=78)
    w = [generate.layer_weights(cfg, l) for l in range(layers)]
    return cfg, make_gpu_stage(cfg, rank, w), wr.window_oracle(cfg, w, window, sinks, rank)


def _extend(st, kv, cfg, x, counts, **kw):
    xin = to_dev(x, cfg)
    outp, outr = torch.empty_like(xin), torch.empty_like(xin)
    st.extend(kv, xin, outp, outr, counts=counts, **kw)
    torch.cuda.synchronize()
    return outp.float().cpu().numpy(), outr.float().cpu().numpy()


@pytest.mark.parametrize("dtype,chunks,tp,window,sinks", [
    ("f32", [[9, 4], [1, 1], [20, 3], [0, 40]], 1, 16, 2), ("f32", [[60, 45], [3, 0]], 2, 33, 0),
    ("bf16", [[7, 12], [1, 1], [2, 0], [1, 1]], 1, 8, 3), ("bf16", [[80, 40], [5, 9], [70, 33]], 2, 40, 4), ("bf16", [[30, 2], [40, 27]], 1, None, 0),
    ("f16", [[2, 0], [20, 12], [1, 1]], 1, 11, 1), ("f16", [[100, 57], [4, 5]], 2, 32, 32)])
def test_extend_matches_the_stage_in_64_bits(dtype, chunks, tp, window, sinks):
    """Chunk behind chunk from an empty cache; the decode kernels up to 32 rows, the prefill kernels beyond; the weights' sums of every layer."""
    cfg, st, ora = _stage(dtype, window, sinks, tp=tp, rank=tp - 1)
    kv = st.kv_cache_create(2, 200)
    kv.set_lengths([0, 0])
    cache = ora.new_cache(2)
    weights = torch.zeros(2, 2, st.hkv_l, 200, device="cuda")
    done = [0, 0]
    for i, counts in enumerate(chunks):
        x = generate.hidden_rows(cfg, sum(counts), stream_id=i)
        p, r = _extend(st, kv, cfg, x, counts, window=window, sinks=sinks, weights=weights)
        ref_p, ref_r = ora.forward(cache, x.numpy(), [s for s, n in enumerate(counts) for _ in range(n)])
        check(f"partial {i}", p, ref_p, TOL[dtype])
        check(f"residual {i}", r, ref_r, TOL[dtype])
        done = [a + b for a, b in zip(done, counts)]
        assert kv.get_lengths(2) == done
    for layer in range(2):
        for b in range(2):
            got, want = weights[layer, b].cpu().numpy(), ora.gathered[layer, b]
            assert not got[:, done[b]:].any()
            check(f"weights {layer} {b}", got[:, :done[b]], want, TOL[dtype])
            assert abs(got.sum() - done[b] * cfg.n_heads // tp) < 1e-3 * done[b] * cfg.n_heads        # every row's weights are one in all


def test_more_sequences_than_a_launch_takes():
    """Some of them without a row, some beyond the first launch: against the same sequences in a call of their own."""
    cfg, st, _ = _stage("bf16", 12, 1, heads=4, kv=2, hidden=256, ffn=512, batch=300)
    counts = [(i * 7) % 4 for i in range(300)]
    x = generate.hidden_rows(cfg, sum(counts))
    kv = st.kv_cache_create(300, 16)
    kv.set_lengths([i % 5 for i in range(300)])              # contexts of zeros
    p, r = _extend(st, kv, cfg, x, counts, window=12, sinks=1)
    assert kv.get_lengths(300) == [i % 5 + n for i, n in enumerate(counts)]
    few = [2, 130, 255, 256, 257, 298]
    at = np.concatenate([[0], np.cumsum(counts)])
    rows = np.concatenate([np.arange(at[i], at[i + 1]) for i in few])
    other = st.kv_cache_create(6, 16)
    other.set_lengths([i % 5 for i in few])
    q, s = _extend(st, other, cfg, x[torch.tensor(rows)], [counts[i] for i in few], window=12, sinks=1)
    check("partial", p[rows], q, TOL["bf16"])
    check("residual", r[rows], s, TOL["bf16"])
    for j, i in enumerate(few):
        n = i % 5 + counts[i]
        if n:
            for a, b in zip(kv.read(0, i, 0, n), other.read(0, j, 0, n)):
                assert torch.allclose(a, b, rtol=0, atol=0.05 * float(b.abs().max()))


@pytest.mark.parametrize("dtype,lens", [("bf16", [50, 33]), ("f16", [9, 14]), ("f32", [40, 21])])
def test_without_a_window_it_is_prefill_and_decode(dtype, lens):
    cfg, st, _ = _stage(dtype, None, 0)
    x, new = generate.hidden_rows(cfg, sum(lens)), [generate.hidden_rows(cfg, 2, stream_id=1 + i) for i in range(3)]
    kv, other = st.kv_cache_create(2, 80), st.kv_cache_create(2, 80)
    xin = to_dev(x, cfg)
    outp, outr = torch.empty_like(xin), torch.empty_like(xin)
    st.prefill(kv, xin, lens, outp, outr)
    other.set_lengths([0, 0])
    p, r = _extend(st, other, cfg, x, lens)
    check("partial", p, outp.float().cpu().numpy(), TOL[dtype])
    check("residual", r, outr.float().cpu().numpy(), TOL[dtype])
    for step, rows in enumerate(new):
        xin = to_dev(rows, cfg)
        outp, outr = torch.empty_like(xin), torch.empty_like(xin)
        st.decode(kv, step, xin, outp, outr)
        p, r = _extend(st, other, cfg, rows, None)
        check(f"partial {step}", p, outp.float().cpu().numpy(), TOL[dtype])
        check(f"residual {step}", r, outr.float().cpu().numpy(), TOL[dtype])
    assert kv.get_lengths(2) == other.get_lengths(2)
    xin = to_dev(new[0], cfg)                                # and decode goes on behind it, at its own count of steps
    outp = torch.empty_like(xin)
    st.decode(other, 0, xin, outp)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("by_weight", [True, False])
def test_a_stream_in_a_cache_of_bounded_size(dtype, by_weight):
    """Rows without end through 48 slots: extend, gather, evict to 24 (keys turned back to their new places), extend and decode again; the oracle's cache follows the
    slots that the library kept, which are held to the definition against the library's own weights."""
    cfg, st, ora = _stage(dtype, 20, 2, heads=8, kv=2)
    size, keep, sinks, recent = 48, 24, 2, 8
    kv = st.kv_cache_create(2, size)
    kv.set_lengths([0, 0])
    cache = ora.new_cache(2)
    weights = torch.zeros(2, 2, st.hkv_l, size, device="cuda") if by_weight else None
    lens, seen = [0, 0], 0
    for step in range(22):
        counts = [[3, 7], [9, 1], [1, 1], [5, 12]][step % 4]
        if any(n + c > size for n, c in zip(lens, counts)):
            seen += 1
            before = None if weights is None else weights.clone()
            slots, left = kv.evict(keep, sinks=sinks, recent=recent, weights=weights, rotate=True)
            assert left is weights
            for layer in range(2):
                for b in range(2):
                    rows_k, rows_v = [], []
                    for h in range(st.hkv_l):
                        want = wr.chosen(lens[b], keep, sinks, recent, None if before is None else before[layer, b, h].cpu().numpy())
                        assert slots[layer, b, h, :len(want)].tolist() == want
                        moved = np.asarray(want) - np.arange(len(want))
                        rows_k.append(wr.turned_back(cache.k[layer][b][want][:, [h]], moved, cfg.rope_theta))
                        rows_v.append(cache.v[layer][b][want][:, [h]])
                    cache.k[layer][b], cache.v[layer][b] = np.concatenate(rows_k, 1), np.concatenate(rows_v, 1)
            ora.gathered.clear()                             # its sums are those of slots that are others' now
            lens = [min(n, keep) for n in lens]
            assert kv.get_lengths(2) == lens
        x = generate.hidden_rows(cfg, sum(counts), stream_id=step)
        p, r = _extend(st, kv, cfg, x, counts, window=20, sinks=2, weights=weights)
        ref_p, ref_r = ora.forward(cache, x.numpy(), [s for s, n in enumerate(counts) for _ in range(n)])
        check(f"partial {step}", p, ref_p, TOL[dtype])
        check(f"residual {step}", r, ref_r, TOL[dtype])
        lens = [a + b for a, b in zip(lens, counts)]
    assert seen >= 3


@pytest.mark.parametrize("dtype,counts", [("bf16", None), ("bf16", [20, 30]), ("f32", [3, 2])])
def test_extend_recorded_and_replayed(dtype, counts):
    """Every replay goes on where the last one ended; what it appends and gathers is what eager calls do, to the bit."""
    cfg, st, _ = _stage(dtype, 16, 2)
    rows = 2 if counts is None else sum(counts)
    one, two = st.kv_cache_create(2, 250), st.kv_cache_create(2, 250)
    for kv in (one, two):
        kv.set_lengths([0, 0])
    wa, wb = (torch.zeros(2, 2, st.hkv_l, 250, device="cuda") for _ in range(2))
    xs = [to_dev(generate.hidden_rows(cfg, rows, stream_id=i), cfg) for i in range(4)]
    x, p, r = xs[0].clone(), torch.empty_like(xs[0]), torch.empty_like(xs[0])
    st.extend(one, x, p, r, counts=counts, window=16, sinks=2, weights=wa)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        st.extend(one, x, p, r, counts=counts, window=16, sinks=2, weights=wa)
    for i in range(4):
        q, s = torch.empty_like(x), torch.empty_like(x)
        if i:
            x.copy_(xs[i])
            graph.replay()
            torch.cuda.synchronize()
            got = p.clone(), r.clone()
        else:
            got = p.clone(), r.clone()
        st.extend(two, xs[i], q, s, counts=counts, window=16, sinks=2, weights=wb)
        torch.cuda.synchronize()
        assert torch.equal(got[0], q) and torch.equal(got[1], s) and torch.equal(wa, wb)
    n = [4 * c for c in (counts or [1, 1])]
    for layer in range(2):
        for b in range(2):
            for a, c in zip(one.read(layer, b, 0, n[b]), two.read(layer, b, 0, n[b])):
                assert torch.equal(a, c)


@pytest.mark.parametrize("dtype,counts", [("bf16", [3, 1]), ("f16", [40, 9]), ("f32", [2, 5])])
def test_extend_on_another_stream(dtype, counts):
    """Behind an event, and an eviction and another step behind it on the same stream."""
    cfg, st, _ = _stage(dtype, 16, 2)
    x = to_dev(generate.hidden_rows(cfg, sum(counts)), cfg)
    found = []
    for stream in (None, torch.cuda.Stream()):
        kv = st.kv_cache_create(2, 90)
        kv.set_lengths([20, 12])                             # contexts of zeros
        weights = torch.zeros(2, 2, st.hkv_l, 90, device="cuda")
        p, r, last = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        st.extend(kv, x, p, r, counts=counts, window=16, sinks=2, weights=weights, stream=stream)
        slots, left = kv.evict(11, sinks=1, recent=4, weights=weights, rotate=True, stream=stream)
        st.extend(kv, x, last, counts=counts, window=16, sinks=2, weights=weights, stream=stream)
        torch.cuda.synchronize()
        assert left is weights and kv.get_lengths(2) == [min(n + c, 11) + c for n, c in zip([20, 12], counts)]
        found.append((p, r, last, slots, weights))
    assert all(torch.equal(a, b) for a, b in zip(*found))


def test_extend_refusals():
    cfg, st, _ = _stage("bf16", None, 0)
    kv = st.kv_cache_create(2, 40)
    x = to_dev(generate.hidden_rows(cfg, 5), cfg)
    out = torch.empty_like(x)
    call = lambda *a, **kw: st.extend(kv, x, out, **dict(dict(counts=[2, 3]), **kw))  # noqa: E731
    with pytest.raises(hx.HexgenError) as e:
        call()
    assert e.value.status == 3                               # no batch yet
    kv.set_lengths([39, 37])
    for kw, status in ((dict(window=0), 1), (dict(sinks=-1), 1), (dict(), 4), (dict(counts=[5]), 3), (dict(counts=[1, 1, 3]), 3), (dict(counts=None), 3)):
        with pytest.raises(hx.HexgenError) as e:
            call(**kw)
        assert e.value.status == status, kw
    for kw in (dict(counts=[2, 2]), dict(counts=[6, -1]), dict(weights=torch.zeros(2, 2, 4, 39, device="cuda")), dict(out_resid=out[:4])):
        with pytest.raises(ValueError):
            call(**kw)
    assert kv.get_lengths(2) == [39, 37]
    empty = hx.Stage(1024, 16, 4, 2816, 2, 1, 0, "bf16")
    other = empty.kv_cache_create(2, 40)
    other.set_lengths([0, 0])
    with pytest.raises(hx.HexgenError) as e:
        empty.extend(other, x, out, counts=[2, 3])
    assert e.value.status == 3                               # weights not loaded
    with pytest.raises(hx.HexgenError) as e:
        st.extend(other, x, out, counts=[2, 3])
    assert e.value.status == 1                               # another stage's cache
