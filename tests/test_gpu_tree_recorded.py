"""When steps over drafted trees can be recorded."""
import pytest
import torch

import paper_2311_11514_amd as hx
from tests.helpers import make_gpu_stage, to_dev
from tests.test_gpu_tree import _trees
from workloads import StageConfig, generate

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_recorded_behind_a_larger_prefill(dtype):
    """A step outside a graph, then a prefill that the workspace grows for, then a recording of the step's size."""
    cfg = StageConfig("rec", dtype, 512, 8, 2, 512, 2, 1, (0,), batch=2, seed=6)
    st = make_gpu_stage(cfg, 0, [generate.layer_weights(cfg, l) for l in range(2)])
    kv, tree = st.kv_cache_create(2, 400), hx.Tree(2, 32)
    counts = [6, 9]
    tree.set(counts, [p for t in _trees(counts) for p in t])
    x = to_dev(generate.hidden_rows(cfg, 15, stream_id=1), cfg)
    p, r = torch.empty_like(x), torch.empty_like(x)

    def prefill(lens):
        rows = to_dev(generate.hidden_rows(cfg, sum(lens)), cfg)
        st.prefill(kv, rows, lens, torch.empty_like(rows))

    prefill([10, 5])
    st.decode_tree(kv, tree, x, p, r)
    prefill([300, 250])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st.decode_tree(kv, tree, x, p, r)
    want = torch.empty_like(x), torch.empty_like(x)
    for k in range(3):
        x.copy_(to_dev(generate.hidden_rows(cfg, 15, stream_id=2 + k), cfg))
        graph.replay()
        torch.cuda.synchronize()
        got = p.clone(), r.clone()
        st.decode_tree(kv, tree, x, *want)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_path_that_passes_the_cache_is_not_counted(dtype):
    """Replays of a recorded decode step take the device's length from 11 to 29 of 32, of which the host knows 12: keeping five rows does nothing, and
    the next tree's rows follow the 29th position."""
    cfg = StageConfig("rec", dtype, 512, 8, 2, 512, 1, 1, (0,), batch=1, seed=6)
    st = make_gpu_stage(cfg, 0, [generate.layer_weights(cfg, 0)])
    kv, tree = st.kv_cache_create(1, 32), hx.Tree(1, 8)
    kv.set_lengths([10])
    x = to_dev(generate.hidden_rows(cfg, 1), cfg)
    p, r = torch.empty_like(x), torch.empty_like(x)
    st.decode(kv, 0, x, p, r)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st.decode(kv, 1, x, p, r)
    for _ in range(18):
        graph.replay()
    tree.set([5], [-1, 0, 1, 2, 3])
    rows = to_dev(generate.hidden_rows(cfg, 5, stream_id=1), cfg)
    st.decode_tree(kv, tree, rows, torch.empty_like(rows))
    kv.keep(tree, [5], [0, 1, 2, 3, 4])
    tree.set([1], [-1])
    q, k, v = (torch.full((1, heads, 64), 0.5 + heads, dtype=x.dtype, device="cuda") for heads in (8, 2, 2))
    kv.tree_attention(0, tree, q, k, v)
    torch.cuda.synchronize()
    for got, want in zip(kv.read(0, 0, 29, 1), (k, v)):
        assert torch.equal(got, want.float().cpu())
