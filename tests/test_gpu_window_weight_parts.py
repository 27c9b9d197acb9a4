"""The softmax weights of windowed rows go into the second product in two parts, whatever blocks a call's rows are in: results of 16 bits have their one rounding."""
import numpy as np
import pytest
import torch

from tests import exactness as ex
from tests import tree_reference as tr
from tests.test_gpu_window import WIDE, Case
from tests.test_gpu_window_precision import SHARED, found, rounded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", SHARED + [x for x in WIDE if x not in SHARED])
def test_many_rows(dtype, case):
    """One rounding's own error, computed from the 64-bit results; what the second parts leave of the weights (u^2 of each) and 32 roundings to 32 bits."""
    c = Case(dtype, *case, seed=3)
    o, a, _, _, _ = found(c)
    u = tr.UNIT[dtype]
    allowed = ex.rms(rounded(o, dtype) - o) + (u * u + 2.0 ** -19) * ex.rms(a)
    off = ex.rms(c.attend().double().cpu().numpy() - o)
    print(f"{dtype} {case}: {off:.3e}, allowed {allowed:.3e}", flush=True)
    assert off <= allowed


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_a_row_beside_a_prompt(dtype):
    """One row of a sequence next to a prompt that is worth blocks of many rows: as exact as in a call of its own."""
    c = Case(dtype, 16, 4, 64, [400, 0], [1, 1100], 200, 2, seed=9)
    o, a, _, _, _ = found(c)
    u = tr.UNIT[dtype]
    got = c.attend().double().cpu().numpy()
    for rows in (slice(0, 1), slice(1, None)):
        allowed = ex.rms(rounded(o[rows], dtype) - o[rows]) + (u * u + 2.0 ** -19) * ex.rms(a[rows])
        assert ex.rms(got[rows] - o[rows]) <= allowed
