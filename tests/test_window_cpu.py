"""Windowed rows and eviction without a GPU: what the entry points refuse, and that the 64-bit reference says what its definition says."""
import numpy as np
import pytest
import torch

import paper_2311_11514_amd as hx
from oracle import stage_oracle as so
from tests import window_reference as wr


def test_null_handles_and_pointers():
    lib = hx.lib
    assert lib.hexgen_kv_window_attention(None, 0, None, 1, 16, 8, 16, 8, 16, 8, 1, 0, None, 16, None) == 1
    assert lib.hexgen_stage_extend(None, None, 16, None, 1, 1, 0, None, 16, 16, None) == 1
    assert lib.hexgen_kv_cache_evict(None, None, 1, 0, 0, None, None, 0, 16, None) == 1
    assert lib.hexgen_kv_cache_batch(None) == -1


def test_integers_that_32_bits_do_not_hold():
    span = hx.binding._span
    for kw in (dict(counts=[1, 1 << 32], given=1, window=4), dict(counts=None, given=1, window=1 << 31), dict(counts=None, given=1, window=-(1 << 31) - 1)):
        with pytest.raises(ValueError, match="32-bit"):
            span(**kw)
    assert span(None, 7, None) == (None, 7, 7, (1 << 31) - 1)
    counts, batch, rows, window = span([3, 0, 2], 5, 9)
    assert list(counts)[:3] == [3, 0, 2] and (batch, rows, window) == (3, 5, 9)
    assert span([], 0, 1)[1:] == (0, 0, 1)
    with pytest.raises(ValueError, match="sinks"):
        hx.binding._int32(1 << 31, "sinks")


def test_visible_slots():
    assert wr.visible(5, None, 0) == [0, 1, 2, 3, 4, 5] and wr.visible(5, 1, 0) == [5]
    assert wr.visible(5, 2, 2) == [0, 1, 4, 5] and wr.visible(1, 2, 9) == [0, 1] and wr.visible(0, 1, 3) == [0]


@pytest.mark.parametrize("window,sinks", [(None, 0), (3, 0), (2, 2), (1, 9)])
def test_reference_attention_is_masked_attention(window, sinks):
    rng = np.random.default_rng(6)
    q, k, v = rng.standard_normal((5, 4, 8)), rng.standard_normal((5, 2, 8)), rng.standard_normal((5, 2, 8))
    kc, vc = rng.standard_normal((4, 2, 8)), rng.standard_normal((4, 2, 8))
    o, a, _, sums, scaled = wr.attention(q, kc, vc, k, v, window, sinks)
    keys, values = (torch.tensor(np.concatenate(x)).repeat_interleave(2, 1).transpose(0, 1) for x in ((kc, k), (vc, v)))
    p, j = torch.arange(4, 9)[:, None], torch.arange(9)[None]
    mask = (j <= p) & ((p - j < (window or 99)) | (j < sinks))
    query = torch.tensor(q).transpose(0, 1)
    ref = torch.nn.functional.scaled_dot_product_attention(query, keys, values, attn_mask=mask)
    weight = torch.softmax((query @ keys.transpose(1, 2) / 8 ** 0.5).masked_fill(~mask, -float("inf")), -1)
    assert np.allclose(o, ref.transpose(0, 1).numpy(), rtol=0, atol=1e-13) and np.all(a >= np.abs(o) - 1e-15)
    assert np.allclose(sums, weight.sum(1).view(2, 2, 9).sum(1).numpy(), rtol=0, atol=1e-13) and np.all(scaled >= 0)


def test_reference_choice():
    w = [9, 1, 5, 5, 0, 5, 2, 7]
    assert wr.chosen(8, 8, 0, 0, w) == list(range(8)) and wr.chosen(3, 8, 1, 1, w) == [0, 1, 2]
    assert wr.chosen(8, 4, 0, 0, w) == [0, 2, 3, 7]
    assert wr.chosen(8, 4, 1, 1, w) == [0, 2, 3, 7] and wr.chosen(8, 4, 2, 2, w) == [0, 1, 6, 7]
    assert wr.chosen(8, 5, 2, 1) == [0, 1, 5, 6, 7] and wr.chosen(8, 2, 0, 2, w) == [6, 7]
    assert wr.chosen(4, 2, 0, 0, [float("nan"), -float("inf"), float("nan"), 0.0]) == [1, 3]
    assert wr.chosen(3, 2, 0, 0, [-0.0, 0.0, 0.0]) == [0, 1]


def test_a_key_turned_back_is_the_key_of_the_nearer_position():
    k = np.random.default_rng(1).standard_normal((3, 2, 64))
    at, to = np.array([9, 40, 1000]), np.array([9, 3, 0])
    turned = wr.turned_back(so.rope(k, at, 10000.0), at - to, 10000.0)
    assert np.allclose(turned, so.rope(k, to, 10000.0), rtol=0, atol=1e-12)


def test_window_oracle_without_a_window_is_the_stage():
    from tests.helpers import make_oracle
    from workloads import StageConfig, generate
    cfg = StageConfig("w", "f32", 256, 4, 2, 512, 2, 1, (0,), batch=2, seed=3)
    w = [generate.layer_weights(cfg, l) for l in range(2)]
    x = generate.hidden_rows(cfg, 7).numpy()
    plain, windowed = make_oracle(cfg, 0, w), wr.window_oracle(cfg, w, None, 0)
    for a, b in zip(plain.prefill(plain.new_cache(2), x, [4, 3]), windowed.prefill(windowed.new_cache(2), x, [4, 3])):
        assert np.allclose(a, b, rtol=0, atol=1e-12)
    assert all(np.allclose(windowed.gathered[layer, s].sum(), 4 * n) for layer in range(2) for s, n in ((0, 4), (1, 3)))
