"""Integers that 32 bits do not hold are refused, not cut off."""
import pytest

import paper_2311_11514_amd as hx


@pytest.mark.parametrize("counts,parents", [([2], [-1, 1 << 32]), ([2], [(1 << 32) - 1, 0]), ([2], [-1 - (1 << 32), 0]), ([2, -(1 << 32)], [-1, 0])])
def test_trees(counts, parents):
    """Each of them is a valid tree once its upper bits are gone."""
    tree = hx.Tree(2, 8)
    with pytest.raises(ValueError, match="32-bit"):
        tree.set(counts, parents)
    assert tree.batch == tree.rows == 0


def test_list_conversion():
    convert = hx.binding._i32
    assert convert(None) is None and list(convert([])) == [] and list(convert((3, -(1 << 31), (1 << 31) - 1))) == [3, -(1 << 31), (1 << 31) - 1]
    for bad in ([1 << 31], [0, -(1 << 31) - 1]):
        with pytest.raises(ValueError):
            convert(bad)
