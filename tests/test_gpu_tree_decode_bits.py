"""A stage's step over drafted trees computes as its decode steps do: up to 32 rows every activation is carried in two parts, rotated queries and
softmax weights among them, so that both round the same numbers and say the same tokens."""
import pytest
import torch

import paper_2311_11514_amd as hx
from tests import tree_reference as tr
from tests.helpers import make_gpu_stage, to_dev
from workloads import StageConfig, generate

pytestmark = pytest.mark.gpu

# Share of the results that may round the other way.  Both calls carry q (a rounding of a rounding's remainder, u^2), the weights (2 u^2: cut off) and
# the attention's result (u^2) in two parts and sum in 32 bits in orders of their own (a chain of 8192 products, 2^-24 sqrt(8192)): together less than
# 2^-14 of a result in bf16 and 2^-16 in fp16.  A result is a multiple of a step of 2^-7 .. 2^-8 (fp16 2^-10 .. 2^-11) of itself and rounds the
# other way for that part of it: 2 %, 4 %.
MOST = {"bf16": 0.02, "f16": 0.04}


def differ(a, b):
    return (a != b).double().mean().item()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hidden,heads,kv,lens,nodes", [
    (1024, 8, 2, [200, 77], 1), (1024, 16, 4, [40, 0, 31, 300, 2000], 1), (2048, 16, 1, [500, 90], 1), (1024, 8, 8, [33], 1),
    (1024, 16, 2, [63, 250], 5),
    (8192, 128, 8, [4100] * 8, 4),                   # blocks that share tiles
    (8192, 64, 32, [4100] * 6, 5),
])
def test_chains_of_nodes_say_what_decode_steps_say(dtype, hidden, heads, kv, lens, nodes):
    """One layer, hidden rows so small that the residual stream behind the attention is the attention's."""
    batch = len(lens)
    cfg = StageConfig("bits", dtype, hidden, heads, kv, 256, 1, 1, (0,), batch=batch, seed=5)
    st = make_gpu_stage(cfg, 0, [generate.layer_weights(cfg, 0)])
    td, g = tr.TORCH[dtype], torch.Generator(device="cuda").manual_seed(3)
    ctx = [[torch.randn(n, kv, hidden // heads, generator=g, device="cuda").to(td) for _ in range(2)] for n in lens]
    kvs = [st.kv_cache_create(batch, max(lens) + nodes) for _ in range(2)]
    for cache in kvs:
        for b, (k, v) in enumerate(ctx):
            if lens[b]:
                cache.fill(0, b, k, v)
        cache.set_lengths(lens)
    x = (to_dev(generate.hidden_rows(cfg, batch * nodes), cfg) * 2.0 ** -7).view(batch, nodes, hidden)
    want = torch.empty_like(x)
    for step in range(nodes):
        now = x[:, step].contiguous()
        p, r = torch.empty_like(now), torch.empty_like(now)
        st.decode(kvs[0], step, now, p, r)
        want[:, step] = r
    tree = hx.Tree(batch, batch * nodes)
    tree.set([nodes] * batch, list(range(-1, nodes - 1)) * batch)
    rows = x.flatten(0, 1).contiguous()
    p, r = torch.empty_like(rows), torch.empty_like(rows)
    st.decode_tree(kvs[1], tree, rows, p, r)
    off = differ(r, want.flatten(0, 1))
    print(f"{dtype} hidden {hidden} heads {heads}/{kv} {lens[:3]} {nodes}: {100 * off:.2f} % of the results", flush=True)
    assert off <= MOST[dtype]
