"""Many positions of little weight beside a heavy one whose value is zero: the result is their sum, and as exact as their weights are."""
import numpy as np
import pytest
import torch

import paper_2311_11514_amd as hx
from tests import tree_reference as tr
from tests.test_gpu_window import Case

pytestmark = pytest.mark.gpu

SCORE = 15.5                                                 # of the heavy position; every other's is 0, its weight 2^-22.4 of the heavy one's


def tolerance(dtype):
    """Relative: the result's rounding; the second part of a weight has eight bits behind the first's eight (bf16), or is a multiple of 2^-37 of the largest weight and at
    least that (fp16: 2^-14.6 of a weight of 2^-22.4); the exponential's argument of 22.4, two roundings of 2^-24, the exponential's own and the sums."""
    return tr.UNIT[dtype] + 2.0 ** -14.5 + 2.0 ** -17


def expected(positions):
    """Row with that many light positions."""
    w = np.asarray(positions) * np.exp(-SCORE)
    return w / (1 + w)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hkv,d,n,rows", [(8, 1, 64, 3000, 1), (4, 4, 64, 1200, 20), (16, 16, 64, 3000, 1500)])       # few rows, in runs and whole; shared tiles
def test_windowed_rows(dtype, hq, hkv, d, n, rows):
    c = Case(dtype, hq, hkv, d, [n], [rows], None, 0, fill=False)
    k, v = torch.zeros(n, hkv, d), torch.ones(n, hkv, d)
    k[37], v[37] = SCORE / 8, 0.0                            # 64 products of 1 and a score's eighth, over the root of 64
    c.kv.fill(0, 0, k, v)
    c.kv.set_lengths([n])
    c.q[:], c.k[:], c.v[:] = 1.0, 0.0, 1.0
    c.before.zero_()
    out, weights = c.attend_both()
    light = n + np.arange(rows)
    want = expected(light)[:, None, None]
    off = np.abs(out.double().cpu().numpy() / want - 1).max()
    print(f"{dtype} {n} {rows}: {off:.3e} of {tolerance(dtype):.3e}", flush=True)
    assert off <= tolerance(dtype)
    sums = weights[0].double().cpu().numpy()
    heavy = (1 - expected(light)).sum() * hq / hkv
    assert np.allclose(sums[:, 37], heavy, rtol=1e-5, atol=0) and np.allclose(sums[:, 5], heavy * np.exp(-SCORE), rtol=1e-5, atol=0)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hkv,n,batch,nodes", [(8, 1, 3000, 1, 1), (4, 4, 1200, 1, 20), (16, 8, 2000, 32, 64)])
def test_drafted_trees(dtype, hq, hkv, n, batch, nodes):
    st = hx.Stage(hq * 64, hq, hkv, 256, 1, 1, 0, dtype)
    kv = st.kv_cache_create(batch, n + nodes)
    k, v = torch.zeros(n, hkv, 64), torch.ones(n, hkv, 64)
    k[37], v[37] = SCORE / 8, 0.0
    for b in range(batch):
        kv.fill(0, b, k, v)
    kv.set_lengths([n] * batch)
    tree = hx.Tree(batch, batch * nodes)
    tree.set([nodes] * batch, list(range(-1, nodes - 1)) * batch)
    td = tr.TORCH[dtype]
    q, k, v = (torch.full((batch * nodes, h, 64), x, dtype=td, device="cuda") for h, x in ((hq, 1.0), (hkv, 0.0), (hkv, 1.0)))
    out = kv.tree_attention(0, tree, q, k, v).double().cpu().numpy()
    want = np.tile(expected(n + np.arange(nodes)), batch)[:, None, None]
    off = np.abs(out / want - 1).max()
    print(f"{dtype} {n} {nodes}: {off:.3e} of {tolerance(dtype):.3e}", flush=True)
    assert off <= tolerance(dtype)
