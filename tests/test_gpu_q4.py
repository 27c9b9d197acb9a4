"""Products with 4-bit weights and the 4-bit head on the GPU against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2311_11514_amd as hx
from tests.tree_reference import TORCH, UNIT

pytestmark = pytest.mark.gpu


def matrix(dtype, n_in, n_out, group, zeros, seed=0):
    """(w4, scales, zeros or None) and, in float64, the weights and s * (32 + q + z), whose products with |x| bound the 32-bit sums."""
    r = np.random.default_rng(seed)
    groups = -(-n_in // group)
    w4 = torch.tensor(r.integers(0, 256, (n_in, n_out // 2), dtype=np.uint8))
    s = torch.tensor(r.uniform(0.5, 2.0, (groups, n_out)) * 0.01).to(TORCH[dtype])
    z4 = torch.tensor(r.integers(0, 256, (groups, n_out // 2), dtype=np.uint8)) if zeros else None

    def nibbles(t):
        return np.stack([t.numpy() & 15, t.numpy() >> 4], -1).reshape(t.shape[0], -1).astype(np.float64)

    at = np.arange(n_in) // group
    q, z, s64 = nibbles(w4), (nibbles(z4) if zeros else np.full((groups, n_out), 8.0))[at], s.double().numpy()[at]
    return (w4, s, z4), (q - z) * s64, s64 * (32 + q + z)


def bound(y, x, big, dtype, group):
    """The result's rounding; and in 32 bits, for every group the products and the sum over its (at most 128 at a time) features against
    16 + q and against 16 + z, then one rounding a group, wave, split and part, all in relation to s (32 + q + z) |x|."""
    return UNIT[dtype] * np.abs(y) + UNIT["f32"] * (2 * min(group, 128) + x.shape[1] / min(group, 128) + 64) * (np.abs(x) @ big) * (1 + UNIT[dtype])


def check(got, x, w, big, dtype, group, label):
    y = x @ w
    off = np.abs(got.double().cpu().numpy() - y) / bound(y, x, big, dtype, group)
    print(f"{label}: {off.max():.3f} of the bound", flush=True)
    assert off.max() <= 1, np.unravel_index(off.argmax(), off.shape)


def rows(dtype, n, k, seed=1):
    x = torch.tensor(np.random.default_rng(seed).standard_normal((n, k))).to(TORCH[dtype])
    return x, x.double().numpy()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n_in,n_out,group,zeros", [
    (128, 64, 128, False), (1, 2, 32, True), (7, 6, 32, False), (33, 30, 32, True), (256, 130, 64, True), (1000, 94, 64, True),
    (1408, 512, 32, False), (512, 1000, 256, True), (2048, 258, 128, True), (640, 96, 512, False), (130, 8256, 128, True),
])
def test_project_sizes(dtype, n_in, n_out, group, zeros):
    """Odd widths, groups that end early, more columns than one tile a block takes; one row, and rows for every form of the kernel."""
    arrays, w, big = matrix(dtype, n_in, n_out, group, zeros)
    m = hx.Q4Matrix(n_in, n_out, group, dtype)
    m.load(*arrays)
    for n in (1, 5, 6, 16, 17):
        x, x64 = rows(dtype, n, n_in, seed=n)
        check(m.project(x.cuda()), x64, w, big, dtype, group, f"{dtype} {n} x {n_in} x {n_out}, groups of {group}")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_project_rows(dtype, group):
    """Every number of operand tiles, several launches of rows, split contractions."""
    arrays, w, big = matrix(dtype, 2304, 208, group, True, seed=3)
    m = hx.Q4Matrix(2304, 208, group, dtype)
    m.load(*[a.cuda() for a in arrays])
    for n in (2, 11, 22, 32, 33, 48, 49, 64, 65, 100, 130):
        x, x64 = rows(dtype, n, 2304, seed=n)
        check(m.project(x.cuda()), x64, w, big, dtype, group, f"{dtype} {n} rows, groups of {group}")


@pytest.mark.parametrize("dtype,n_rows", [("bf16", 20), ("f16", 64), ("f32", 9), ("f32", 20)])
def test_project_wide_matrix(dtype, n_rows):
    """Columns enough for two tiles a wave."""
    arrays, w, big = matrix(dtype, 384, 66000, 128, True, seed=4)
    m = hx.Q4Matrix(384, 66000, 128, dtype)
    m.load(*arrays)
    x, x64 = rows(dtype, n_rows, 384)
    check(m.project(x.cuda()), x64, w, big, dtype, 128, f"{dtype} {n_rows} x 384 x 66000")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("n_in,n_out", [(8192, 96), (8400, 206), (300, 4104), (130, 8256), (2000, 8200)])
def test_project_long_and_wide_matrices(dtype, group, n_in, n_out):
    """Long contractions, in one block and split; matrices of a few hundred tiles in groups of operand columns; operands that LDS holds and not."""
    arrays, w, big = matrix(dtype, n_in, n_out, group, True, seed=5)
    m = hx.Q4Matrix(n_in, n_out, group, dtype)
    m.load(*arrays)
    for n in (1, 4, 8, 9, 17, 33, 40, 64):
        x, x64 = rows(dtype, n, n_in, seed=n)
        check(m.project(x.cuda()), x64, w, big, dtype, group, f"{dtype} {n} x {n_in} x {n_out}, groups of {group}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_alignment_and_the_callers_output(dtype):
    arrays, w, big = matrix(dtype, 512, 100, 128, True)
    m = hx.Q4Matrix(512, 100, 128, dtype)
    m.load(*arrays)
    for n in (3, 20):
        x, x64 = rows(dtype, n, 512)
        want = m.project(x.cuda())
        check(want, x64, w, big, dtype, 128, f"{dtype} {n} rows")
        for ld, first in ((512 + 8, 0), (512 + 3, 0), (520, 1), (1024, 512)):      # 16-byte pieces, odd strides, an odd start
            flat = torch.full((first + n * ld + 8,), float("nan"), dtype=x.dtype, device="cuda")
            part = flat[first:first + n * ld].view(n, ld)[:, :512]
            part.copy_(x)
            assert torch.equal(m.project(part), want)
        guard = torch.full((n + 2, 100), 7.0, dtype=x.dtype, device="cuda")
        assert torch.equal(m.project(x.cuda(), out=guard[1:-1]), want)
        assert (guard[0] == 7).all() and (guard[-1] == 7).all()
    with pytest.raises(hx.HexgenError) as e:
        m.project(x.cuda()[:1].expand(4, 512))
    assert e.value.status == 1
    with pytest.raises(ValueError, match="^out"):
        m.project(x.cuda(), out=torch.empty(20, 100, dtype=torch.float64, device="cuda"))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_large_small_and_odd_values_stay_in_their_row(dtype):
    """A row's values have no influence on another's; magnitudes from the type's smallest normal number on; what is not finite gives NaN."""
    arrays, w, big = matrix(dtype, 384, 64, 64, True)
    m = hx.Q4Matrix(384, 64, 64, dtype)
    m.load(*arrays)
    for n in (4, 18):
        x, _ = rows(dtype, n, 384)
        tiny, large = torch.finfo(TORCH[dtype]).tiny, {"f16": 200.0}.get(dtype, 1e30)
        x[0] *= tiny * 64
        x[1] *= large
        x[2, 100] = float("inf")
        x[3, 383] = float("nan")
        got = m.project(x.cuda())
        keep = [i for i in range(n) if i not in (2, 3)]
        assert torch.isnan(got[2]).all() and torch.isnan(got[3]).all()
        x64 = x[keep].double().numpy()
        y = x64 @ w
        # (results below the type's normal numbers are rounded to its smallest step)
        off = np.abs(got[keep].double().cpu().numpy() - y) - bound(y, x64, big, dtype, 64) - torch.finfo(TORCH[dtype]).smallest_normal * UNIT[dtype]
        assert (off <= 0).all(), off.max()


@pytest.mark.parametrize("dtype,n", [("bf16", 4), ("bf16", 40), ("f32", 3), ("f32", 12)])
def test_streams_graphs_and_the_same_bits(dtype, n):
    arrays, _, _ = matrix(dtype, 1000, 512, 64, True)
    m = hx.Q4Matrix(1000, 512, 64, dtype)
    m.load(*arrays)
    xs = [rows(dtype, n, 1000, seed=s)[0].cuda() for s in range(4)]
    want = [m.project(x) for x in xs]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = [m.project(x, stream=s) for x in xs]
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    x, y = torch.empty_like(xs[0]), torch.empty_like(want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.project(x, out=y)
    for _ in range(2):
        for a, b in zip(xs, want):
            x.copy_(a)
            graph.replay()
            assert torch.equal(m.project(a), b)
            torch.cuda.synchronize()
            assert torch.equal(y, b)


def test_a_second_load_replaces_the_first():
    m = hx.Q4Matrix(256, 64, 64, "bf16")
    x, x64 = rows("bf16", 3, 256)
    for seed, zeros in ((0, True), (1, False), (2, True)):
        arrays, w, big = matrix("bf16", 256, 64, 64, zeros, seed=seed)
        m.load(*arrays)
        check(m.project(x.cuda()), x64, w, big, "bf16", 64, f"load {seed}")


# ---- the head -----------------------------------------------------------------------------------------------------
def _head_reference(a, b, gain, w, big, eps, group):
    x = a.double().numpy() + (b.double().numpy() if b is not None else 0)
    x = x / np.sqrt((x ** 2).mean(1, keepdims=True) + eps) * gain.double().numpy()
    y = x @ w
    # the 32-bit row: its sum of squares (one rounding a term at most), root, quotient and two products, on every product with a weight
    return y, bound(y, x, big, "f32", group) + UNIT["f32"] * (x.shape[1] / 2 + 16) * (np.abs(x) @ np.abs(w))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("hidden,vocab,tp,group,zeros,n_rows", [(512, 1000, 1, 128, False, 1), (1024, 4104, 1, 64, True, 5), (512, 8400, 1, 32, True, 6),
                                                               (256, 1030, 2, 64, True, 40), (512, 9000, 3, 128, True, 70)])
def test_head_greedy(dtype, hidden, vocab, tp, group, zeros, n_rows):
    arrays, w, big = matrix(dtype, hidden, vocab, group, zeros, seed=9)
    a, _ = rows(dtype, n_rows, hidden, seed=2)
    b, _ = rows(dtype, n_rows, hidden, seed=3)
    gain = (1 + 0.02 * torch.tensor(np.random.default_rng(4).standard_normal(hidden))).to(TORCH[dtype])
    for second in (b, None):
        y, off = _head_reference(a, second, gain, w, big, 1e-5, group)
        decisive = 0
        for r in range(tp):
            hd = hx.Head(hidden, vocab, tp, r, dtype)
            hd.load_q4(gain, *arrays, group=group)
            tok, val = hd.greedy(a.cuda(), None if second is None else second.cuda())
            torch.cuda.synchronize()
            tok, val = tok.cpu().numpy(), val.cpu().double().numpy()
            part, slack = y[:, r * vocab // tp:(r + 1) * vocab // tp], off[:, r * vocab // tp:(r + 1) * vocab // tp].max(1)
            best = np.sort(part, 1)[:, -2:]
            clear = best[:, 1] - best[:, 0] > 2 * slack
            decisive += clear.sum()
            assert (np.abs(val - best[:, 1]) <= slack).all()
            assert (tok[clear] == part.argmax(1)[clear] + r * vocab // tp).all()
        assert decisive >= 0.8 * tp * n_rows, "too many near-ties"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hidden,vocab,n_rows", [(8448, 1000, 7), (256, 4200, 21), (8448, 1000, 1)])
def test_head_greedy_split_and_grouped(dtype, hidden, vocab, n_rows):
    """The arg-max behind a split contraction, and over groups of operand columns."""
    arrays, w, big = matrix(dtype, hidden, vocab, 64, True, seed=11)
    a, _ = rows(dtype, n_rows, hidden, seed=2)
    gain = torch.ones(hidden, dtype=TORCH[dtype])
    y, off = _head_reference(a, None, gain, w, big, 1e-5, 64)
    hd = hx.Head(hidden, vocab, 1, 0, dtype)
    hd.load_q4(gain, *arrays, group=64)
    for _ in range(2):
        tok, val = hd.greedy(a.cuda())
        torch.cuda.synchronize()
        tok, val, slack = tok.cpu().numpy(), val.cpu().double().numpy(), off.max(1)
        assert (np.abs(val - y.max(1)) <= slack).all()
        # the chosen column is one that the bound does not rule out
        assert (y[np.arange(n_rows), tok] >= y.max(1) - 2 * slack).all()


def test_head_ties_go_to_the_lowest_column_and_loads_replace_each_other():
    """Equal columns at both ends of tiles and blocks; a plain matrix behind a 4-bit one and the other way round."""
    hidden, vocab = 128, 2500
    w4 = torch.zeros(hidden, vocab // 2, dtype=torch.uint8)           # q = 0 everywhere: w = -8 s
    s = torch.full((1, vocab), 0.01)
    for same in ([2499, 1337, 700, 16], [2048, 2047], [31, 32]):
        scale = s.clone()
        scale[:, same] = -0.01                                         # the same positive logit
        hd = hx.Head(hidden, vocab, 1, 0, "bf16")
        hd.load_q4(torch.ones(hidden), w4, scale)
        for n in (1, 8, 33):
            tok, _ = hd.greedy(torch.ones(n, hidden, dtype=torch.bfloat16, device="cuda"))
            assert (tok == min(same)).all(), (same, tok)
    x = torch.ones(2, hidden, dtype=torch.bfloat16, device="cuda")
    plain = torch.zeros(hidden, vocab)
    plain[:, 77] = 1.0
    hd.load(torch.ones(hidden), plain)
    assert hd.splits(2) >= 0 and (hd.greedy(x)[0] == 77).all()
    hd.load_q4(torch.ones(hidden), w4, scale)
    assert hd.splits(2) == -1 and (hd.greedy(x)[0] == 31).all()
    hd.load(torch.ones(hidden), plain)
    assert (hd.greedy(x)[0] == 77).all()


def test_head_refusals():
    hd = hx.Head(128, 300, 1, 0, "bf16")
    w, s = torch.zeros(128, 150, dtype=torch.uint8), torch.zeros(1, 300)
    with pytest.raises(hx.HexgenError) as e:
        hd.load_q4(torch.ones(128), w, torch.zeros(3, 300), group=48)
    assert e.value.status == 2
    with pytest.raises(ValueError, match="w4"):
        hd.load_q4(torch.ones(128), w[:, :-1], s)
    with pytest.raises(ValueError, match="g_final"):
        hd.load_q4(torch.ones(127), w, s)
    with pytest.raises(hx.HexgenError) as e:
        hd.greedy(torch.ones(1, 128, dtype=torch.bfloat16, device="cuda"))
    assert e.value.status == 3
    raw = hx.lib.hexgen_head_load_q4
    g = torch.ones(128, dtype=torch.bfloat16)
    assert raw(hd.handle, None, w.data_ptr(), s.data_ptr(), None, 128) == raw(hd.handle, g.data_ptr(), None, s.data_ptr(), None, 128) == 1
    assert raw(hd.handle, g.data_ptr(), w.data_ptr(), s.data_ptr(), None, 0) == 1
    odd = hx.Head(128, 301, 1, 0, "bf16")
    assert raw(odd.handle, g.data_ptr(), w.data_ptr(), s.data_ptr(), None, 128) == 2
