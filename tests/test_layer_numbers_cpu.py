"""Layers, sequences and slots that 32 bits do not hold are refused, not cut off to another layer's number."""
import types

import pytest
import torch

import paper_2311_11514_amd as hx


def cache():
    """A cache without a device behind it: what is refused never gets there."""
    kv = object.__new__(hx.KVCache)
    kv.handle, kv.max_batch, kv.max_seq = None, 1, 8
    kv.stage = types.SimpleNamespace(dtype=1, hq_l=2, hkv_l=2, head_dim=64, n_layers=1)
    return kv


@pytest.mark.parametrize("far", [1 << 32, -(1 << 32), 1 << 31])
def test_layers_and_sequences(far):
    kv, rows = cache(), torch.zeros(1, 2, 64, dtype=torch.bfloat16)
    tree = types.SimpleNamespace(rows=1, handle=None)
    for call in (lambda: kv.window_attention(far, rows, rows, rows), lambda: kv.tree_attention(far, tree, rows, rows, rows), lambda: kv.fill(far, 0, rows, rows),
                 lambda: kv.fill(0, far, rows, rows), lambda: kv.read(far, 0, 0, 1), lambda: kv.read(0, far, 0, 1), lambda: kv.read(0, 0, far, 1)):
        with pytest.raises(ValueError, match="32-bit"):
            call()


def test_layers_of_a_stage():
    st = object.__new__(hx.Stage)
    st.handle, st.dtype, st._taps = None, 1, {}
    t = torch.zeros(1)
    for call in (lambda: st.load_layer(1 << 32, *[t] * 9), lambda: st.run_sublayer(cache(), 1 << 32, 0, t, None, 1, t, stream=types.SimpleNamespace(cuda_stream=0)),
                 lambda: st.set_tap(1 << 32, t)):
        with pytest.raises(ValueError, match="32-bit"):
            call()
    assert st._taps == {}
