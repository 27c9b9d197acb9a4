"""The largest launches of windowed rows and of evictions, and caches beyond 2^31 elements."""
import pytest
import torch

import paper_2311_11514_amd as hx
from tests.tree_reference import TORCH

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_blocks_than_a_launch_takes_are_refused(dtype):
    """256 sequences, 64 kv heads of 16 heads each: 1024 rows of one beside single ones pass 2^32 threads, 1000 do not and are right."""
    batch, hq, hkv, d = 256, 1024, 64, 64
    st = hx.Stage(hq * d, hq, hkv, 256, 1, 1, 0, dtype)
    kv = st.kv_cache_create(batch, 1024)
    kv.set_lengths([0] * batch)
    g = torch.Generator(device="cuda").manual_seed(1)

    def attend(rows):
        counts = [rows] + [1] * (batch - 1)
        q, k, v = (torch.randn(rows + batch - 1, h, d, generator=g, device="cuda").to(TORCH[dtype]) for h in (hq, hkv, hkv))
        return kv.window_attention(0, q, k, v, counts, window=1), v

    with pytest.raises(hx.HexgenError) as e:
        attend(1024)
    assert e.value.status == 4
    out, v = attend(1000)                                    # a window of one: every row is its value
    assert torch.equal(out, v.repeat_interleave(hq // hkv, 1))


def test_evictions_of_more_blocks_than_a_launch_takes_are_refused():
    """512 layers x 64 sequences x 128 heads: 2^22 units."""
    st = hx.Stage(128 * 64, 128, 128, 256, 512, 1, 0, "bf16")
    kv = st.kv_cache_create(64, 1)
    kv.set_lengths([1] * 64)
    out = torch.zeros(4, dtype=torch.int32, device="cuda")
    assert hx.lib.hexgen_kv_cache_evict(kv.handle, kv.handle, 1, 0, 0, None, None, 0, out.data_ptr(), None) == 4


@pytest.mark.parametrize("n", [40000])
def test_positions_and_offsets_of_a_long_cache(n):
    """A cache of 2^32 elements a tensor: the last sequence's rows, its weights and its eviction are at offsets that 32 bits do not hold."""
    batch, hkv, d, size = 8, 64, 128, 1 << 16
    st = hx.Stage(hkv * d, hkv, hkv, 256, 1, 1, 0, "bf16")
    kv = st.kv_cache_create(batch, size)
    kv.set_lengths([0] * (batch - 1) + [n])
    small = st.kv_cache_create(batch, 64)
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (torch.randn(2, hkv, d, generator=g, device="cuda").bfloat16() for _ in range(3))
    weights = torch.zeros(batch, hkv, size, device="cuda")
    out = kv.window_attention(0, q, k, v, [0] * (batch - 1) + [2], window=2, sinks=1, weights=weights)
    # the context's keys and values are zero: scores 0 of the first slot and, for the first row, of the one before it
    own = (q.double() * k.double()).sum(-1) / d ** 0.5
    cross = (q[1].double() * k[0].double()).sum(-1) / d ** 0.5
    first = torch.softmax(torch.stack([own[0], torch.zeros_like(cross), torch.zeros_like(cross)]), 0)
    second = torch.softmax(torch.stack([own[1], cross, torch.zeros_like(cross)]), 0)
    want = torch.stack([first[0, :, None] * v[0].double(), second[0, :, None] * v[1].double() + second[1, :, None] * v[0].double()])
    assert torch.allclose(out.double(), want, rtol=2.0 ** -7, atol=2.0 ** -9)
    assert torch.allclose(weights[-1, :, n:n + 2].double(), torch.stack([first[0] + second[1], second[0]], 1), rtol=1e-5, atol=1e-6)
    assert torch.allclose(weights[-1, :, 0].double(), first[1] + second[2], rtol=1e-5, atol=1e-6) and not weights[:-1].any() and not weights[-1, :, 1:n - 1].any()
    kv.commit([0] * (batch - 1) + [2], batch)
    slots, left = kv.evict(4, sinks=1, weights=weights[None], into=small)
    assert slots[0, -1, :, :4].tolist() == [[0, n - 1, n, n + 1]] * hkv and (slots[0, :-1] == -1).all()
    got_k, got_v = small.read(0, batch - 1, 0, 4)
    assert torch.equal(got_k[2:], k.float().cpu()) and torch.equal(got_v[2:], v.float().cpu()) and not got_k[:2].any()
    assert torch.equal(left[0, -1, :, :4], weights[-1][:, [0, n - 1, n, n + 1]])
    kv.evict(4, sinks=1, weights=weights[None])              # the same in place
    assert all(torch.equal(a, b) for a, b in zip(kv.read(0, batch - 1, 0, 4), (got_k, got_v))) and kv.get_lengths(batch) == [0] * (batch - 1) + [4]
