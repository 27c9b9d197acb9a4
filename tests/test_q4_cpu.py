"""4-bit matrices without a GPU: what the entry points refuse."""
import ctypes as C

import pytest
import torch

import paper_2311_11514_amd as hx


@pytest.mark.parametrize("args,status", [
    ((512, 1024, 128, 1), 0), ((1, 2, 32, 0), 0), ((1000, 1410, 64, 2), 0), ((512, 1024, 256, 1), 0),
    ((0, 1024, 128, 1), 1), ((512, 0, 128, 1), 1), ((512, 1024, 0, 1), 1), ((512, 1024, 128, 3), 1), ((512, 1024, 128, -1), 1),
    ((512, 1023, 128, 1), 2),                      # columns come in pairs
    ((512, 1024, 16, 1), 2), ((512, 1024, 96, 1), 2), ((512, 1024, 192, 1), 2), ((512, 1024, 33, 1), 2),
    ((1 << 25, 2, 128, 1), 2), ((2, 1 << 25, 128, 1), 2),
])
def test_create(args, status):
    h = C.c_void_p()
    assert hx.lib.hexgen_q4_create(*args, C.byref(h)) == status
    if status == 0:
        hx.lib.hexgen_q4_destroy(h)
    else:
        assert not h.value


def test_null_pointers_and_state():
    assert hx.lib.hexgen_q4_create(64, 64, 32, 1, None) == 1
    hx.lib.hexgen_q4_destroy(None)
    q = hx.Q4Matrix(256, 64, 128, "bf16")
    assert hx.lib.hexgen_q4_load(q.handle, None, 16, None) == hx.lib.hexgen_q4_load(q.handle, 16, None, None) == hx.lib.hexgen_q4_load(None, 16, 16, None) == 1
    project = hx.lib.hexgen_q4_project
    assert project(None, 16, 256, 1, 16, None) == project(q.handle, None, 256, 1, 16, None) == project(q.handle, 16, 256, 1, None, None) == 1
    assert project(q.handle, 16, 255, 1, 16, None) == project(q.handle, 16, 256, 0, 16, None) == 1
    assert project(q.handle, 17, 256, 1, 16, None) == project(q.handle, 16, 256, 1, 18, None) == 1       # an odd address, half a pair
    assert project(q.handle, 16, 256, 1, 16, None) == 3                                                    # nothing loaded
    hd = hx.lib.hexgen_head_load_q4
    assert hd(None, 16, 16, 16, None, 128) == 1


def test_shapes_are_checked_where_they_are_known():
    q = hx.Q4Matrix(200, 64, 64, "bf16")
    w, s, z = torch.zeros(200, 32, dtype=torch.uint8), torch.zeros(4, 64), torch.zeros(4, 32, dtype=torch.uint8)
    for bad in ((w[:-1], s, z), (w, s[:3], z), (w, s, z[:3]), (w.to(torch.int8), s, z), (w, s, z.float()), (w[:, :31], s, z)):
        with pytest.raises(ValueError):
            q.load(*bad)
    for x in (torch.zeros(2, 200), torch.zeros(2, 199, dtype=torch.bfloat16), torch.zeros(200, dtype=torch.bfloat16), torch.zeros(0, 200, dtype=torch.bfloat16),
              torch.zeros(2, 400, dtype=torch.bfloat16)[:, ::2], torch.zeros(2, 200, dtype=torch.bfloat16)):
        with pytest.raises(ValueError, match="^x"):
            q.project(x)
