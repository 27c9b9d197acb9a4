"""Drafted trees without a GPU: what the entry points refuse, and that the 64-bit reference says what its definition says."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2311_11514_amd as hx
from tests import tree_reference as tr


def test_create_limits():
    h = C.c_void_p()
    for args, status in (((0, 4), 1), ((4, 0), 1), ((-1, 4), 1), (((1 << 15) + 1, 4), 4), ((4, (1 << 16) + 1), 4)):
        assert hx.lib.hexgen_tree_create(*args, C.byref(h)) == status
    assert hx.lib.hexgen_tree_create(1, 1, None) == 1
    hx.lib.hexgen_tree_destroy(None)


@pytest.mark.parametrize("counts,parents,status", [
    ([1, 1, 1], [-1, -1, -1], 4),             # more sequences than the handle takes
    ([-1, 2], [-1, 0], 1),                     # a negative count
    ([257, 0], [-1] + list(range(256)), 4),    # more nodes than a tree may have
    ([4, 5], [-1, 0, 0, 0, -1, 0, 0, 0, 0], 4),    # more nodes than the handle takes
    ([0, 0], [], 2),                           # no node at all
    ([2], [0, 0], 2),                          # node 0 has a parent
    ([2], [-1, -1], 2),                        # a second root
    ([2], [-1, 1], 2),                         # its own parent
    ([3], [-1, 2, 0], 2),                      # a parent behind its child
    ([2, 2], [-1, 0, -1, 2], 2),               # a parent in another sequence
    ([2], [-1, -2], 2),
])
def test_set_refuses(counts, parents, status):
    tree = hx.Tree(2, 8)
    with pytest.raises(hx.HexgenError) as e:
        tree.set(counts, parents)
    assert e.value.status == status
    assert tree.batch == tree.rows == 0
    assert hx.lib.hexgen_tree_accept(tree.handle, 1, 1, 1, 1, 1, None) == 3       # nothing set: refused before a pointer is used


def test_set_and_accept_null_pointers():
    tree = hx.Tree(2, 8)
    one = (C.c_int32 * 1)(1)
    assert hx.lib.hexgen_tree_set(None, one, one, 1, None) == 1
    assert hx.lib.hexgen_tree_set(tree.handle, None, one, 1, None) == 1
    assert hx.lib.hexgen_tree_set(tree.handle, one, None, 1, None) == 1
    assert hx.lib.hexgen_tree_set(tree.handle, one, one, 0, None) == 1
    assert hx.lib.hexgen_tree_accept(None, 1, 1, 1, 1, 1, None) == 1
    for k in range(5):
        args = [1] * 5
        args[k] = None
        assert hx.lib.hexgen_tree_accept(tree.handle, *args, None) == 1
    with pytest.raises(ValueError):
        tree.set([2], [-1])
    assert hx.lib.hexgen_stage_decode_tree(None, None, tree.handle, 1, 1, 1, None) == 1
    assert hx.lib.hexgen_kv_tree_attention(None, 0, tree.handle, 16, 8, 16, 8, 16, 8, 16, None) == 1
    assert hx.lib.hexgen_kv_cache_keep(None, tree.handle, one, one, None) == 1


def test_tensor_checks_name_the_tensor():
    tree = hx.Tree(1, 4)
    tree.batch, tree.rows = 1, 4
    with pytest.raises(ValueError, match="draft"):
        tree.accept(torch.zeros(4, dtype=torch.int64), torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError, match="draft"):
        tree.accept(torch.zeros(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32))
    check = hx.binding._rows_of_heads
    for t in (torch.zeros(4, 2, 64), torch.zeros(4, 3, 64, dtype=torch.bfloat16), torch.zeros(4, 2, 128, dtype=torch.bfloat16)[..., ::2],
              torch.zeros(4, 4, 64, dtype=torch.bfloat16)[:, ::2]):
        with pytest.raises(ValueError):
            check(t, "q", 4, 2, 64, torch.bfloat16)


def test_reference_attention_of_a_chain_is_causal_attention():
    rng = np.random.default_rng(5)
    q, k, v = rng.standard_normal((4, 4, 8)), rng.standard_normal((4, 2, 8)), rng.standard_normal((4, 2, 8))
    kc, vc = rng.standard_normal((3, 2, 8)), rng.standard_normal((3, 2, 8))
    o, a, _ = tr.attention(q, kc, vc, k, v, tr.random_tree(4, 0, width=1))
    keys, values = torch.tensor(np.concatenate([kc, k])).repeat_interleave(2, 1), torch.tensor(np.concatenate([vc, v])).repeat_interleave(2, 1)
    mask = torch.ones(4, 7, dtype=torch.bool).tril(3)
    ref = torch.nn.functional.scaled_dot_product_attention(torch.tensor(q).transpose(0, 1), keys.transpose(0, 1), values.transpose(0, 1), attn_mask=mask)
    assert np.allclose(o, ref.transpose(0, 1).numpy(), rtol=0, atol=1e-13)
    assert np.all(a >= np.abs(o))


def test_reference_acceptance():
    parents = [-1, 0, 0, 1, 1, 3]
    assert tr.accept(parents, [9, 5, 6, 7, 7, 8], [5, 7, 1, 8, 2, 3]) == ([0, 1, 3, 5], [5, 7, 8, 3])
    assert tr.accept(parents, [9, 5, 6, 7, 7, 8], [4, 7, 1, 8, 2, 3]) == ([0], [4])
    assert tr.accept([], [], []) == ([], [])
    assert tr.depth(parents, 5) == 3 and tr.ancestors(parents, 4) == [4, 1, 0]
