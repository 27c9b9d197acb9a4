"""The criterion of exactness.py turns down inputs that were rounded to 16 bits, and takes 32-bit arithmetic, at every shape it is used at."""
import numpy as np
import pytest
import torch

from tests import exactness as ex
from tests import tree_reference as tr

ROUND = {"f16": torch.float16, "bf16": torch.bfloat16}


def rounded(x, to):
    return torch.tensor(x, dtype=torch.float32).to(ROUND[to]).double().numpy()


@pytest.mark.parametrize("n_in,n_out,group,counts", ex.PRODUCTS + [(h, v, g, (n,)) for h, v, g, n in ex.HEADS])
def test_products(n_in, n_out, group, counts):
    from tests.test_gpu_q4 import matrix

    _, w, _ = matrix("f32", n_in, min(n_out, 4104), group, True, seed=25)
    for n in counts:
        x = torch.tensor(np.random.default_rng(n).standard_normal((n, n_in)), dtype=torch.float32).double().numpy()
        y = x @ w
        limit = ex.product_limit(n_in) * ex.rms(y)
        assert ex.rms((x.astype(np.float32) @ w.astype(np.float32)).astype(np.float64) - y) <= limit
        for to in ROUND:
            assert ex.rms(rounded(x, to) @ w - y) > 2 * limit


@pytest.mark.parametrize("hq,hkv,d,lens,counts", ex.ATTENTION)
def test_attention(hq, hkv, d, lens, counts):
    trees = [tr.random_tree(n, 7 + i) for i, n in enumerate(counts)]
    rng = np.random.default_rng(3)

    def draw(*shape):
        return torch.tensor(rng.standard_normal(shape), dtype=torch.float32).double().numpy()

    seqs = [(draw(len(t), hq, d), draw(n, hkv, d), draw(n, hkv, d), draw(len(t), hkv, d), draw(len(t), hkv, d)) for n, t in zip(lens, trees)]
    o, s = ex.attention_rows(seqs, lens, trees)
    limit = ex.attention_limit(d, s, max(n + len(t) for n, t in zip(lens, trees))) * ex.rms(o)
    for to in ROUND:
        for which in ((0,), (1, 3), (2, 4)):                  # q, keys, values
            off = ex.attention_rows([tuple(rounded(x, to) if i in which else x for i, x in enumerate(q)) for q in seqs], lens, trees)[0] - o
            assert ex.rms(off) > 2 * limit, (to, which)
