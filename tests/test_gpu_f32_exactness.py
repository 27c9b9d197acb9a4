"""fp32 calls compute in 32 bits at every width: products with 4-bit weights, the 4-bit head, the drafted trees' attention."""
import numpy as np
import pytest
import torch

import paper_2311_11514_amd as hx
from tests import exactness as ex
from tests.test_gpu_q4 import matrix, rows
from tests.test_gpu_tree import Case, _trees

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_in,n_out,group,counts", ex.PRODUCTS)
def test_products(n_in, n_out, group, counts):
    arrays, w, _ = matrix("f32", n_in, n_out, group, True, seed=25)
    m = hx.Q4Matrix(n_in, n_out, group, "f32")
    m.load(*arrays)
    for n in counts:
        x, x64 = rows("f32", n, n_in, seed=n)
        y = x64 @ w
        off = ex.rms(m.project(x.cuda()).double().cpu().numpy() - y) / ex.rms(y) / ex.product_limit(n_in)
        print(f"{n} x {n_in} x {n_out}, groups of {group}: {off:.3f} of the limit", flush=True)
        assert off <= 1


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("hidden,vocab,group,n", ex.HEADS)
def test_head_logits(dtype, hidden, vocab, group, n):
    """The head computes in 32 bits for every type of rows."""
    arrays, w, _ = matrix(dtype, hidden, vocab, group, True, seed=26)
    a, a64 = rows(dtype, n, hidden, seed=2)
    b, b64 = rows(dtype, n, hidden, seed=3)
    gain = (1 + 0.02 * torch.tensor(np.random.default_rng(4).standard_normal(hidden))).to(a.dtype)
    hd = hx.Head(hidden, vocab, 1, 0, dtype)
    hd.load_q4(gain, *arrays, group=group)
    x = a64 + b64
    y = x / np.sqrt((x ** 2).mean(1, keepdims=True) + 1e-5) * gain.double().numpy() @ w
    token, logit = hd.greedy(a.cuda(), b.cuda())
    off = ex.rms(logit.double().cpu().numpy() - y.max(1)) / ex.rms(y) / ex.product_limit(hidden)
    print(f"{dtype} {n} x {hidden} x {vocab}: {off:.3f} of the limit", flush=True)
    assert off <= 1


@pytest.mark.parametrize("hq,hkv,d,lens,counts", ex.ATTENTION)
def test_attention(hq, hkv, d, lens, counts):
    c = Case("f32", hq, hkv, d, lens, _trees(counts, seed=7), seed=3)
    row, seqs = 0, []
    for b, t in enumerate(c.trees):
        q, k, v = (x[row:row + len(t)].double().numpy() for x in (c.q, c.k, c.v))
        seqs.append((q, *(x.double().numpy() for x in c.ctx[0][b]), k, v))
        row += len(t)
    o, s = ex.attention_rows(seqs, lens, c.trees)
    off = ex.rms(c.attend().double().cpu().numpy() - o) / ex.rms(o) / ex.attention_limit(d, s, max(n + len(t) for n, t in zip(lens, c.trees)))
    print(f"{hq}/{hkv} d {d} {lens} {counts}: {off:.3f} of the limit", flush=True)
    assert off <= 1
