"""How exactly and how far products with 4-bit weights compute, against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2311_11514_amd as hx
from tests.test_gpu_q4 import bound, matrix, rows
from tests.tree_reference import UNIT

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_in,n_out,group", [(384, 64, 64), (1000, 1410, 32), (8192, 96, 128), (512, 8200, 256)])
def test_rows_up_to_the_end_of_the_range(dtype, n_in, n_out, group):
    """Values whose sums leave fp32's range before the group's scale is applied; the results are finite."""
    arrays, w, big = matrix(dtype, n_in, n_out, group, True, seed=21)
    m = hx.Q4Matrix(n_in, n_out, group, dtype)
    m.load(*arrays)
    for n in (1, 5, 24):
        x, _ = rows(dtype, n, n_in, seed=n)
        for i, top in zip(range(n), (2e35, 1e36, 1e37, 2e35, 9e34)):
            x[i] *= top
        if n > 1:
            x[1], x[3] = x[1].abs(), 2e35                      # equal signs, equal values
        x64 = x.double().numpy()
        y = x64 @ w
        assert np.abs(y).max() < 3e38
        got = m.project(x.cuda()).double().cpu().numpy()
        off = np.abs(got - y) / bound(y, x64, big, dtype, group)
        print(f"{dtype} {n} x {n_in} x {n_out}, groups of {group}: {off.max():.3f} of the bound", flush=True)
        assert off.max() <= 1                                  # a NaN fails as well



def exact_bound(y, x, w, dtype, group):
    """In relation to the products' own magnitudes |q - z| s |x|: the result's rounding; in 32 bits one rounding for every feature of a group (at most 128
    at a time), one a group, wave, split and part, and two of 2^-24 for what two fp16 parts leave of an fp32 value; and of the row's largest value what the
    operand's smallest step is off by (2^-39 for two parts, 2^-40 for bf16 rows, nothing for fp16 ones), on every weight."""
    least = {"f32": 2.0 ** -39, "bf16": 2.0 ** -40, "f16": 0.0}[dtype] * np.abs(x).max(1, keepdims=True) * np.abs(w).sum(0)
    return (UNIT[dtype] * np.abs(y) + UNIT["f32"] * (min(group, 128) + x.shape[1] / min(group, 128) + 66) * (np.abs(x) @ np.abs(w)) + least) * (1 + UNIT[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n_in,n_out,group,zeros", [(512, 256, 128, True), (512, 130, 64, False), (1000, 94, 32, True), (4096, 1024, 128, True), (8192, 96, 128, False),
                                                    (300, 8200, 64, True), (2304, 208, 256, True)])
def test_a_large_value_whose_weight_is_its_zero_point(dtype, n_in, n_out, group, zeros):
    """A row's values 2^20 times the others, at features that have no weight: they leave nothing in the results."""
    arrays, w, _ = matrix(dtype, n_in, n_out, group, zeros, seed=23)
    large = [5, n_in // 2 + 3, n_in - 1]
    for k in large:
        arrays[0][k] = arrays[2][k // group] if zeros else 0x88
        w[k] = 0
    m = hx.Q4Matrix(n_in, n_out, group, dtype)
    m.load(*arrays)
    for n in (1, 7, 20, 50):
        x, _ = rows(dtype, n, n_in, seed=n)
        x *= 2.0 ** -5
        x[:, large] = torch.tensor([2.0 ** 15, -2.0 ** 15, 1.75 * 2.0 ** 14], dtype=x.dtype)
        x64 = x.double().numpy()
        y = x64 @ w
        off = np.abs(m.project(x.cuda()).double().cpu().numpy() - y) / exact_bound(y, x64, w, dtype, group)
        print(f"{dtype} {n} x {n_in} x {n_out}, groups of {group}: {off.max():.3f} of the bound", flush=True)
        assert off.max() <= 1


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_largest_value_beside_the_smallest(dtype):
    """A value near the end of the range, again without a weight: the others of its row count as they are down to 2^-29 (2^-15 with all their bits in fp32)
    of it, and are off by 2^-40 (2^-39) of it at most below."""
    n_in, n_out, group = 256, 64, 64
    arrays, w, _ = matrix(dtype, n_in, n_out, group, True, seed=22)
    arrays[0][77] = arrays[2][77 // group]
    w[77] = 0
    m = hx.Q4Matrix(n_in, n_out, group, dtype)
    m.load(*arrays)
    for n in (4, 20):
        x, _ = rows(dtype, n, n_in, seed=30)
        for i, e in zip(range(4), (0, 80, 90, 110)):
            x[i] *= 2.0 ** e
        x[:, 77] = 2.0 ** 116
        x64 = x.double().numpy()
        y = x64 @ w
        assert (np.abs(m.project(x.cuda()).double().cpu().numpy() - y) <= exact_bound(y, x64, w, dtype, group)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [512, 1 << 20, 2 ** 31 - 128])
def test_groups_longer_than_the_matrix(dtype, group):
    """One group for all features, up to the largest group there is."""
    arrays, w, big = matrix(dtype, 384, 64, group, True, seed=24)
    m = hx.Q4Matrix(384, 64, group, dtype)
    m.load(*arrays)
    head = hx.Head(384, 64, 1, 0, dtype)
    head.load_q4(torch.ones(384), *arrays, group=group)
    x, x64 = rows(dtype, 3, 384)
    y = x64 @ w
    assert (np.abs(m.project(x.cuda()).double().cpu().numpy() - y) <= exact_bound(y, x64, w, dtype, group)).all()
    token, logit = head.greedy(x.cuda())
    assert (logit > 0).all() and (y[np.arange(3), token.cpu().numpy()] >= 0.99 * y.max(1)).all()
