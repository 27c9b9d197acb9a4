"""How exactly and how far products with 4-bit weights compute, against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2311_11514_amd as hx
from tests.test_gpu_q4 import bound, matrix, rows

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

