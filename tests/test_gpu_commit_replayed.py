"""Committing rows behind replayed steps: the lengths on the device go on from where the replays have taken them."""
import pytest
import torch

from tests.helpers import to_dev
from tests.test_gpu_extend import _stage
from workloads import generate

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("replays", [0, 1, 9])
def test_lengths(dtype, replays):
    cfg, st, _ = _stage(dtype, 16, 2)
    kv = st.kv_cache_create(2, 40)
    x = to_dev(generate.hidden_rows(cfg, 2), cfg)
    p = torch.empty_like(x)
    kv.set_lengths([9, 1])                                   # contexts of zeros
    st.extend(kv, x, p, window=16, sinks=2)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        st.extend(kv, x, p, window=16, sinks=2)
    for _ in range(replays):
        graph.replay()
    lens = [10 + replays, 2 + replays]
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn(5, h, cfg.hidden // cfg.n_heads, generator=g, device="cuda").to(x.dtype) for h in (st.hq_l, st.hkv_l, st.hkv_l))
    for layer in range(2):
        kv.window_attention(layer, q, k, v, [2, 3], window=16, sinks=2)
    kv.commit([2, 3], 2)
    assert kv.get_lengths(2) == [lens[0] + 2, lens[1] + 3]
    for layer in range(2):
        for b, rows in enumerate((slice(0, 2), slice(2, 5))):
            got = kv.read(layer, b, lens[b], rows.stop - rows.start)
            assert all(torch.equal(a, t[rows].float().cpu()) for a, t in zip(got, (k, v)))
    graph.replay()                                           # goes on behind the rows that have been committed
    slots, _ = kv.evict(40)
    assert kv.get_lengths(2) == [lens[0] + 3, lens[1] + 4] and (slots[0, :, 0] >= 0).sum(-1).tolist() == kv.get_lengths(2)
    for layer in range(2):
        for b, rows in enumerate((slice(0, 2), slice(2, 5))):
            got = kv.read(layer, b, lens[b], rows.stop - rows.start)
            assert all(torch.equal(a, t[rows].float().cpu()) for a, t in zip(got, (k, v)))
