"""The largest launches of the drafted trees' attention."""
import pytest
import torch

import paper_2311_11514_amd as hx
from tests.tree_reference import TORCH

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_blocks_than_a_launch_takes_are_refused(dtype):
    """32768 sequences, two kv heads of 16 heads each: one tree of 256 nodes among single ones passes 2^32 threads, one of 254 does not and is right."""
    batch, hq, hkv, d = 1 << 15, 32, 2, 64
    st = hx.Stage(hq * d, hq, hkv, 256, 1, 1, 0, dtype)
    kv = st.kv_cache_create(batch, 256)
    kv.set_lengths([0] * batch)
    tree = hx.Tree(batch, batch + 256)
    g = torch.Generator(device="cuda").manual_seed(1)

    def attend(nodes):
        tree.set([nodes] + [1] * (batch - 1), [-1] + [0] * (nodes - 1) + [-1] * (batch - 1))
        q, k, v = (torch.randn(tree.rows, h, d, generator=g, device="cuda").to(TORCH[dtype]) for h in (hq, hkv, hkv))
        return kv.tree_attention(0, tree, q, k, v), v

    with pytest.raises(hx.HexgenError) as e:
        attend(256)
    assert e.value.status == 4
    if dtype == "bf16":
        out, v = attend(254)
        torch.cuda.synchronize()
        want = v.repeat_interleave(hq // hkv, 1)
        assert torch.equal(out[254:], want[254:]) and torch.equal(out[0], want[0])      # a root attends itself alone
        assert torch.isfinite(out.float()).all()
