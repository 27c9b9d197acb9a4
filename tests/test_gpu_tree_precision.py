"""How exactly the drafted trees' attention computes: 16-bit results are the 64-bit ones with their one rounding, since the softmax weights go
into the second product as two parts, of which neither turns an infinite value into a NaN."""
import numpy as np
import pytest
import torch

from tests import tree_reference as tr
from tests.test_gpu_tree import WIDE, Case, _trees

pytestmark = pytest.mark.gpu


def rms(x):
    return float(np.sqrt(np.mean(np.square(x))))


def rounded(o, dtype):
    return torch.tensor(o).to(tr.TORCH[dtype]).double().numpy()


def allowed(c):
    """RMS of the error that results with one rounding have, computed from the 64-bit results; plus what the second parts of the weights leave
    (a rounding of a rounding's remainder) and 32 roundings to 32 bits (scores: sqrt(128) in a chain of a head's products, times a score of a
    few units; one for each exponential and each sum), on the weighted magnitudes of the values."""
    row, o, a = 0, [], []
    for b, t in enumerate(c.trees):
        part = [x[row:row + len(t)].double().numpy() for x in (c.q, c.k, c.v)]
        ctx = [x.double().numpy() for x in c.ctx[0][b]]
        found = tr.attention(part[0], ctx[0], ctx[1], part[1], part[2], t)
        o.append(found[0])
        a.append(found[1])
        row += len(t)
    o, a = np.concatenate(o), np.concatenate(a)
    u = tr.UNIT[c.dtype]
    return o, rms(rounded(o, c.dtype) - o) + (u * u + 2.0 ** -19) * rms(a)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hkv,d,lens,counts", [
    (8, 2, 64, [40], [5]), (6, 2, 64, [129], [17]), (8, 1, 128, [300, 31, 5], [16, 9, 40]), (8, 8, 64, [95], [64]), (4, 1, 64, [20, 3], [100, 256]),
    (8, 1, 128, [1500, 0, 700], [26, 20, 30]), *WIDE])
def test_results_have_one_rounding(dtype, hq, hkv, d, lens, counts):
    c = Case(dtype, hq, hkv, d, lens, _trees(counts, seed=12), seed=13)
    o, most = allowed(c)
    for _ in range(2):                                    # the second time with rows that are in the cache already
        off = rms(c.attend().double().cpu().numpy() - o)
        print(f"{dtype} {hq}/{hkv} d {d} {lens[:4]} {counts[:4]}: RMS error {off:.3e} of {most:.3e}", flush=True)
        assert off <= most


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hkv,d,lens,counts", [(8, 2, 64, [140], [5]), (8, 1, 128, [300, 31], [16, 9]), WIDE[0], WIDE[3]])
def test_an_infinite_value_of_the_context_comes_out_infinite(dtype, hq, hkv, d, lens, counts):
    """Whole tiles of the context, weights between an eighth and one: the values' column of that element, for every head that reads it, and no other."""
    c = Case(dtype, hq, hkv, d, lens, _trees(counts, seed=2), seed=3, fill=False)
    c.q = c.q * 0.125                                     # scores of a fraction of a unit: no weight below the type's normal numbers
    for b, n in enumerate(lens):
        c.ctx[0][b][1][n // 2 if n < 64 else 17, hkv - 1, 5] = -float("inf")
        c.kv.fill(0, b, *c.ctx[0][b])
    c.kv.set_lengths(lens)
    out = c.attend().double().cpu().numpy()
    group = hq // hkv
    there = np.repeat([n > 0 for n in lens], counts)
    assert (out[there, hq - group:, 5] == -np.inf).all()
    out[:, hq - group:, 5] = 0.0
    assert np.isfinite(out).all()
