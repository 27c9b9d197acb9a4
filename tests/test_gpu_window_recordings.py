"""A recorded call that gathers attention weights stays valid whatever calls follow it: wider windows, longer caches, other rows."""
import pytest
import torch

from tests.helpers import to_dev
from tests.test_gpu_extend import _stage
from tests.test_gpu_window import Case
from workloads import generate

pytestmark = pytest.mark.gpu


def occupy():
    """Memory that was given back meanwhile belongs to somebody else now."""
    torch.cuda.synchronize()
    return [torch.full((n,), float("nan"), device="cuda") for n in (1 << 24, 1 << 20, 1 << 16, 1 << 10)]


def attend(c, kv, q, k, v, counts, window, weights, out):
    kv.window_attention(0, q, k, v, counts, window=window, sinks=3, weights=weights, out=out)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("recorded", [[1, 1], [40, 9]])      # with scores left for the sums, and with the statistics alone
def test_attention(dtype, recorded):
    c = Case(dtype, 8, 1, 64, [1000, 300], recorded, 50, 3, max_seq=1200, seed=31)
    q, k, v = c.q.cuda(), c.k.cuda(), c.v.cuda()
    want, gathered = c.attend_both()
    weights, out, graph = torch.zeros_like(gathered), torch.zeros_like(q), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        attend(c, c.kv, q, k, v, recorded, 50, weights, out)
    long = c.stage.kv_cache_create(2, 4000)
    long.set_lengths([3000, 2000])                           # contexts of zeros
    held = []
    for kv, window, counts in ((c.kv, None, recorded), (c.kv, 900, [1, 1]), (long, None, [1, 1]), (c.kv, None, [7, 4]), (long, 2000, [300, 200]), (long, None, [900, 700])):
        x = [torch.randn(sum(counts), h, 64, device="cuda").to(q.dtype) for h in (8, 1, 1)]
        other = torch.zeros(2, 1, kv.max_seq, device="cuda")
        attend(c, kv, *x, counts, window, other, torch.empty_like(x[0]))
        held.append(occupy())
        weights.copy_(c.before)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(weights, gathered), (window, counts)
        assert torch.isfinite(other).all() and all(torch.isnan(t).all() for t in held[-1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_stage(dtype):
    """Steps of one row each; between the replays the same number of rows without a window, and on a longer cache."""
    cfg, st, _ = _stage(dtype, 16, 2)
    one, two, long = st.kv_cache_create(2, 100), st.kv_cache_create(2, 100), st.kv_cache_create(2, 3000)
    x = to_dev(generate.hidden_rows(cfg, 2), cfg)
    p, q = torch.empty_like(x), torch.empty_like(x)
    wa, wb = (torch.zeros(2, 2, st.hkv_l, 100, device="cuda") for _ in range(2))
    for kv, w in ((one, wa), (two, wb)):
        kv.set_lengths([30, 5])
        st.extend(kv, x, p, window=16, sinks=2, weights=w)
    long.set_lengths([2500, 1000])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        st.extend(one, x, p, window=16, sinks=2, weights=wa)
    held = []
    for step in range(4):
        st.extend(long, x, q, weights=torch.zeros(2, 2, st.hkv_l, 3000, device="cuda"))
        held.append(occupy())
        graph.replay()
        st.extend(two, x, q, window=16, sinks=2, weights=wb)
        torch.cuda.synchronize()
        assert torch.equal(p, q) and torch.equal(wa, wb), step
