"""How exactly windowed rows are computed.  Blocks of few rows: 16-bit results are the 64-bit ones with their one rounding, since the softmax weights go into the second
product in two parts.  Blocks that share tiles round every weight once, as the prefill attention does.  fp32 computes in 32 bits; the weights' sums do for
every type."""
import numpy as np
import pytest
import torch

from tests import exactness as ex
from tests import tree_reference as tr
from tests import window_reference as wr
from tests.test_gpu_window import Case

pytestmark = pytest.mark.gpu


def found(c):
    """(o, a, s, weights, what the call adds to them) of all rows, in 64 bits."""
    row, o, a, s = 0, [], [], 0.0
    weights, added = c.before.double().numpy().copy(), np.zeros(c.before.shape)
    for b, n in enumerate(c.counts):
        part = [x[row:row + n].double().numpy() for x in (c.q, c.k, c.v)]
        ctx = [x.double().numpy() for x in c.ctx[0][b]]
        x = wr.attention(part[0], ctx[0], ctx[1], part[1], part[2], c.window, c.sinks)
        o.append(x[0])
        a.append(x[1])
        s = max(s, x[2].max() if n else 0.0)
        added[b, :, :c.lens[b] + n] += x[3]
        row += n
    return np.concatenate(o), np.concatenate(a), s, weights + added, added


def rounded(o, dtype):
    return torch.tensor(o).to(tr.TORCH[dtype]).double().numpy()


FEW = [(8, 2, 64, [40], [1], 24, 4), (6, 2, 64, [129], [5], None, 0), (8, 1, 128, [300, 31, 5], [3, 2, 4], 100, 3), (4, 1, 64, [20, 3], [100, 256], 50, 70),
       (2, 1, 128, [2900], [2], None, 0), (8, 1, 128, [2500, 0, 700], [26, 20, 30], 2000, 33)]
SHARED = [(64, 8, 128, [0, 31, 300, 503], [64, 65, 70, 130], 100, 33), (64, 8, 64, [0, 31, 300, 203], [96, 65, 120, 130], None, 0), (16, 16, 64, [0, 77], [900, 600], 128, 5)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", FEW + SHARED)
def test_results_of_16_bits(dtype, case):
    """One rounding's own error, computed from the 64-bit results; for few rows what the second parts of the weights leave, for shared tiles a rounding of every weight (half a
    step at most, uniform: over sqrt(3), and as if all of a row's went the same way); 32 roundings to 32 bits."""
    c = Case(dtype, *case, seed=3)
    o, a, _, _, _ = found(c)
    u = tr.UNIT[dtype]
    own = ex.rms(rounded(o, dtype) - o)
    allowed = own + (u * u + 2.0 ** -19) * ex.rms(a) if case in FEW else float(np.hypot(own, u / np.sqrt(3) * ex.rms(a))) + 2.0 ** -19 * ex.rms(a)
    off = ex.rms(c.attend().double().cpu().numpy() - o)
    print(f"{dtype} {case}: {off:.3e}, one rounding {own:.3e}, allowed {allowed:.3e}", flush=True)
    assert off <= allowed


@pytest.mark.parametrize("case", FEW + SHARED)
def test_results_of_32_bits(case):
    c = Case("f32", *case, seed=3)
    o, _, s, _, _ = found(c)
    off = ex.rms(c.attend().double().cpu().numpy() - o) / ex.rms(o) / ex.attention_limit(c.d, s, max(n + m for n, m in zip(c.lens, c.counts)))
    print(f"{case}: {off:.3f} of the limit", flush=True)
    assert off <= 1


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("case", FEW + SHARED)
def test_sums_of_the_weights(dtype, case):
    """The scores' error as for the results, a chain of as many additions as there are rows and heads."""
    c = Case(dtype, *case, seed=3)
    c.before.zero_()
    _, _, s, weights, added = found(c)
    off = ex.rms(c.attend_both()[1].double().cpu().numpy() - weights) / ex.rms(added)
    limit = ex.attention_limit(c.d, s, max(n + m for n, m in zip(c.lens, c.counts)) + max(c.counts) * c.hq // c.hkv)
    print(f"{dtype} {case}: {off / limit:.3f} of the limit", flush=True)
    assert off <= limit
