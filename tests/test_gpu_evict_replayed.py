"""Eviction behind replayed steps, which have taken the lengths on the device beyond what the host counted: the host's lengths are the device's again."""
import pytest
import torch

from tests.helpers import TOL, check, to_dev
from tests.test_gpu_extend import _stage
from workloads import generate

pytestmark = pytest.mark.gpu


def step(st, kv, call, n, x, p):
    if call == "extend":
        st.extend(kv, x, p, window=16, sinks=2)
    else:
        getattr(st, call)(kv, n, x, p)


@pytest.mark.parametrize("dtype,call", [("bf16", "extend"), ("f32", "extend"), ("bf16", "decode"), ("f32", "decode"), ("f16", "decode_static")])
@pytest.mark.parametrize("replays", [0, 1, 30])
@pytest.mark.parametrize("into", [False, True])
def test_lengths(dtype, call, replays, into):
    """Recorded once (not run), replayed or not; the twin cache takes the same steps eagerly.  Contexts come to stand below and beyond what is kept."""
    cfg, st, _ = _stage(dtype, 16, 2)
    size, keep = 80, 32
    one, two = (st.kv_cache_create(2, size) for _ in range(2))
    others = [st.kv_cache_create(2, 48) for _ in range(2)]
    x = to_dev(generate.hidden_rows(cfg, 2), cfg)
    p, q = torch.empty_like(x), torch.empty_like(x)
    for kv in (one, two):
        kv.set_lengths([9, 1])                               # contexts of zeros
        step(st, kv, call, 0, x, p)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(st, one, call, 1, x, p)
    for i in range(replays):
        graph.replay()
        step(st, two, call, 1 + i, x, q)
    lens = [10 + replays, 2 + replays]
    found = []
    for kv, other in zip((one, two), others):
        dst = other if into else kv
        slots, _ = kv.evict(keep, sinks=2, recent=3, rotate=True, into=dst if into else None)
        assert dst.get_lengths(2) == [min(n, keep) for n in lens]
        assert kv.get_lengths(2) == (lens if into else [min(n, keep) for n in lens])
        # rows up to the end of the cache fit, as one call, and one more does not
        room = [dst.max_seq - min(n, keep) for n in lens]
        y = to_dev(generate.hidden_rows(cfg, sum(room), stream_id=1), cfg)
        out = torch.empty_like(y)
        st.extend(dst, y, out, counts=room, window=16, sinks=2)
        assert dst.get_lengths(2) == [dst.max_seq] * 2
        torch.cuda.synchronize()
        found.append((slots, out))
    assert torch.equal(found[0][0], found[1][0])
    if call == "extend":
        assert torch.equal(found[0][1], found[1][1])
    else:                                                    # a recorded decode step may take other kernels, by the cache's size instead of its contexts
        check("out", found[0][1].float().cpu().numpy(), found[1][1].float().cpu().numpy(), TOL[dtype])
