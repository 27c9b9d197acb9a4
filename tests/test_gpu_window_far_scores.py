"""Windowed rows whose scores are far from zero, in blocks that share tiles: rows that see nothing in a wave's first tiles while others of that wave have large
scores already, without first positions, scores of either sign.  Results are known: a row that attends itself alone is its value, one whose scores are all the same
the mean of its values."""
import numpy as np
import pytest
import torch

from tests import tree_reference as tr
from tests.test_gpu_window import Case

pytestmark = pytest.mark.gpu

SCORES = [2.0 ** 23, -2.0 ** 15, 0.0, -2.0 ** 23, 2.0 ** 10, -2.0 ** 12]      # from about 2^22.5 on (d 64) a score's base is the score itself


def set_rows(c, score):
    """Row x has the score score[x] (d 128: times sqrt(2)) with every key of the cache and of the rows: products of powers of two, exact in every order of summation."""
    k = 2.0 ** 6
    c.q[:] = (torch.tensor(score, dtype=torch.float64) / (8 * k))[:, None, None].to(c.q.dtype)
    c.k[:] = k
    for b, n in enumerate(c.lens):
        c.ctx[0][b][0] = torch.full_like(c.ctx[0][b][0], k)
        if n:
            c.kv.fill(0, b, *c.ctx[0][b])
    c.kv.set_lengths(c.lens)


def check(c, window):
    """The mean of the values that a row attends; every one of them has the same weight."""
    out, weights = c.attend_both()
    out, weights = out.double().cpu().numpy(), weights.double().cpu().numpy()
    group, row = c.hq // c.hkv, 0
    want = c.before.double().numpy().copy()
    for b, (n, m) in enumerate(zip(c.lens, c.counts)):
        values = torch.cat((c.ctx[0][b][1], c.v[row:row + m])).double().numpy()
        for x in range(m):
            at = slice(max(0, n + x - window + 1), n + x + 1)
            o, a = (y.repeat(group, 0) for y in (values[at].mean(0), np.abs(values[at]).mean(0)))
            # the scores are exact: what is left are the roundings of results and weights, of the exponential and of the sums
            assert np.all(np.abs(out[row + x] - o) <= tr.attention_bound(o, a, 0.0, c.dtype, 0, window)), (b, x, out[row + x, 0, :4], o[0, :4])
            want[b, :, at] += group / (at.stop - at.start)
        row += m
    # as many additions as rows attend a slot, one for each of the heads, and the weights' own roundings
    assert np.all(np.abs(weights - want) <= tr.UNIT["f32"] * (2 * window * group + 2 * window + 64) * want)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hkv,d", [(16, 16, 64), (16, 16, 128), (32, 16, 64)])
def test_rows_that_attend_themselves_alone(dtype, hq, hkv, d):
    """A wave's first rows are far from zero, its others see their first tile later."""
    c = Case(dtype, hq, hkv, d, [16, 80], [900, 600], 1, 0, seed=21)
    pick = np.random.default_rng(4).integers(0, len(SCORES), c.rows)
    pick[:16], pick[16:32] = 0, 1
    set_rows(c, [SCORES[i] for i in pick])
    check(c, 1)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("window", [7, 64])
@pytest.mark.parametrize("score", [-2.0 ** 23, -2.0 ** 15, 2.0 ** 23, None])
def test_rows_whose_scores_are_all_the_same(dtype, window, score):
    c = Case(dtype, 16, 16, 64, [0, 77], [900, 600], window, 0, seed=22)
    pick = np.random.default_rng(5).integers(0, len(SCORES), c.rows)
    set_rows(c, [SCORES[i] if score is None else score for i in pick])
    check(c, window)
