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
