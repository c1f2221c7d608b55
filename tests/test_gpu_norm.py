"""The norm of rows on the GPU against the formula in 64 bits.

h is exact: a sum of two numbers of the type, rounded once.  y is off by its rounding (2^-8 of itself in bf16, 2^-24 in fp32)
and by what fp32 loses on the way: the sum of squares adds at most 33 values a lane (of rows in registers), then 6 and 4 times
sums of two or sixteen, so it is off by less than 64 * 2^-24 and its root by half of that; division, root and the two products
add less than 2^-21: less than 2^-18 in all.  Rows of any length are summed by 1024 lanes, which adds one 2^-24 for each further
8192 columns.  The 8- and 4-bit forms are those of y as it came out: the same bytes.
"""
import numpy as np
import pytest
import torch

import fp4_reference as ref4
import fp8_reference as ref8
from paper_2503_05066_amd import capmoe

pytestmark = [pytest.mark.gpu, pytest.mark.usefixtures("built_library")]
BF16, F32 = torch.bfloat16, torch.float32
TYPES = {BF16: capmoe.DTYPE_BF16, F32: capmoe.DTYPE_F32}


@pytest.fixture(autouse=True, scope="module")
def _device():
    torch.cuda.set_device(0)


def values(seed, r, c, dtype):
    g = np.random.default_rng([seed, r, c])
    x = g.standard_normal((r, c)) * np.exp(2 * g.standard_normal((r, 1)))
    return torch.from_numpy(x).to(dtype).cuda()


def buffers(r, c, bits):
    if not bits:
        return None, None
    q, s = (capmoe.fp8_row_buffers if bits == 8 else capmoe.fp4_row_buffers)(r, c)
    return q.fill_(0x55), s.fill_(0x55)


def f64(t):
    return t.double().cpu().numpy()


def check(x, residual, weight, eps, h, y, q, s, bits, rows=None):
    """The first `rows` rows of the outputs; behind them what the buffers held."""
    dtype, (r, c) = y.dtype, y.shape
    n = r if rows is None else rows
    rounded = lambda v: f64(torch.from_numpy(v).to(dtype))
    want_h, want = ref4.norm(f64(x), None if residual is None else f64(residual), None if weight is None else f64(weight), eps, rounded)
    if h is not None:
        assert np.array_equal(f64(h)[:n], want_h[:n], equal_nan=True)
    got = f64(y)
    half = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    tiny = 2.0 ** -133 if dtype == BF16 else 2.0 ** -148
    with np.errstate(invalid="ignore"):
        fine = np.isfinite(want[:n])
        off = np.abs(got[:n] - want[:n])
        limit = (half + 2.0 ** -18 + c * 2.0 ** -37) * np.abs(want[:n]) + tiny
        assert np.all(off[fine] <= limit[fine]), np.max(off[fine] / limit[fine])
    assert np.array_equal(np.isnan(got[:n]), np.isnan(want[:n]))
    if bits:
        if bits == 4:
            want_q, want_s = ref4.quantize(got)
        else:
            want_q, want_s = ref8.quantize_rows(got)
        got_q, got_s = q.cpu().numpy(), s.cpu().numpy()
        nan = (want_q[:n] & 127) == 127 if bits == 8 else np.zeros(want_q[:n].shape, bool)
        assert np.array_equal(np.where(nan, 0, got_q[:n]), np.where(nan, 0, want_q[:n]))
        assert np.all(got_q[:n][nan] & 127 == 127) and np.array_equal(got_s[:n], want_s[:n])
        assert np.all(got_q[n:] == 0x55) and np.all(got_s[n:] == 0x55)


SIZES = [(1, 8), (5, 64), (3, 264), (130, 512), (9, 520), (37, 1024), (6, 1032), (64, 1416), (11, 2048), (3, 2056), (37, 4096), (5, 5640), (2, 8192),
         (3, 14336), (2, 16392), (1, 32768), (2, 32776), (1, 131072)]


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("bits,residual", [(0, True), (4, True), (8, False), (8, True), (4, False)])
def test_norm(rows, cols, dtype, bits, residual):
    x, w = values(1, rows, cols, dtype), values(2, 1, cols, dtype)[0]
    r = values(3, rows, cols, dtype) if residual else None
    h = torch.full_like(x, 7.0) if residual else None
    y = torch.full_like(x, 7.0)
    q, s = buffers(rows, cols, bits)
    norm = capmoe.make_norm(rows, cols, 1e-5, TYPES[dtype], bits)
    capmoe.moe_norm_rows(norm, x, r, w, None, h, y, q, s)
    check(x, r, w, norm.eps, h, y, q, s, bits)
    if bits:  # without y: the same bytes
        q2, s2 = buffers(rows, cols, bits)
        capmoe.moe_norm_rows(norm, x, r, None if w is None else w, None, None, None, q2, s2)
        assert torch.equal(q, q2) and torch.equal(s, s2)


def test_narrow_rows_of_fp32():
    x = values(4, 5, 4, F32)
    y = torch.zeros_like(x)
    q, s = buffers(5, 4, 8)
    norm = capmoe.make_norm(5, 4, 1e-6, capmoe.DTYPE_F32, 8)
    capmoe.moe_norm_rows(norm, x, None, None, None, None, y, q, s)
    check(x, None, None, norm.eps, None, y, q, s, 8)


@pytest.mark.parametrize("cols", [12, 36, 516, 1020, 4100, 33004])
@pytest.mark.parametrize("bits", [4, 8])
def test_fp32_rows_that_end_in_the_middle_of_eight(cols, bits):
    x, r, w = values(30, 6, cols, F32), values(31, 6, cols, F32), values(32, 1, cols, F32)[0]
    x[2, cols - 1] = float("nan")  # a row that is no number ends in zeros all the same
    h, y = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    q, s = buffers(6, cols, bits)
    norm = capmoe.make_norm(6, cols, 1e-6, capmoe.DTYPE_F32, bits)
    capmoe.moe_norm_rows(norm, x, r, w, None, h, y, q, s)
    check(x, r, w, norm.eps, h, y, q, s, bits)


def test_rows_beyond_32_bit_offsets():
    rows, cols = 600000, 4096  # 4.9 GB each
    x = torch.zeros((rows, cols), dtype=BF16, device="cuda")
    last = values(33, 5, cols, BF16)
    x[-5:], x[:5] = last, last
    y, (q, s) = torch.full_like(x, 7.0), buffers(rows, cols, 4)
    capmoe.moe_norm_rows(capmoe.make_norm(rows, cols, bits=4), x, None, None, None, None, y, q, s)
    norm = capmoe.make_norm(5, cols, 1e-6, bits=4)
    check(last, None, None, norm.eps, None, y[-5:], q[-5:], s[-5:], 4)
    assert torch.equal(y[:5], y[-5:]) and torch.equal(q[:5], q[-5:]) and not y[5:-5].any() and not q[5:-5].any()
    x[:] = 0
    capmoe.moe_dequantize_rows(4, q, s, x)
    assert np.array_equal(f64(x[-5:]), ref4.value(q[-5:].cpu().numpy(), s[-5:].cpu().numpy())) and torch.equal(x[:5], x[-5:])
    q2, s2 = buffers(rows, cols, 4)
    capmoe.moe_quantize_rows_fp4(y, None, None, q2, s2)
    assert torch.equal(q, q2) and torch.equal(s, s2)


@pytest.mark.parametrize("cols", [264, 1024, 4096, 40000])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_outputs_in_place_of_inputs(cols, dtype):
    x, r, w = values(5, 7, cols, dtype), values(6, 7, cols, dtype), values(7, 1, cols, dtype)[0]
    norm = capmoe.make_norm(7, cols, 1e-6, TYPES[dtype], 4)
    want = [torch.zeros_like(x), torch.zeros_like(x), *buffers(7, cols, 4)]
    capmoe.moe_norm_rows(norm, x, r, w, None, *want)
    for sum_at, y_at in (("x", "r"), ("r", "x"), ("r", None), (None, "x"), (None, "r")):
        a = {"x": x.clone(), "r": r.clone(), None: None}
        q, s = buffers(7, cols, 4)
        capmoe.moe_norm_rows(norm, a["x"], a["r"], w, None, a[sum_at], a[y_at], q, s)
        if sum_at:
            assert torch.equal(a[sum_at], want[0])
        if y_at:
            assert torch.equal(a[y_at], want[1])
        assert torch.equal(q, want[2]) and torch.equal(s, want[3])


@pytest.mark.parametrize("count", [-2, 0, 1, 6, 13, 100])
@pytest.mark.parametrize("cols", [200, 1000, 2048, 33000])
def test_rows_behind_the_count_stay(count, cols):
    x, r = values(8, 13, cols, BF16), values(9, 13, cols, BF16)
    y, h = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    q, s = buffers(13, cols, 4)
    norm = capmoe.make_norm(13, cols, bits=4)
    capmoe.moe_norm_rows(norm, x, r, None, torch.tensor([count], dtype=torch.int32, device="cuda"), h, y, q, s)
    n = min(max(count, 0), 13)
    check(x, r, None, norm.eps, h, y, q, s, 4, rows=n)
    assert torch.all(y[n:] == 7.0) and torch.all(h[n:] == 7.0)


@pytest.mark.parametrize("cols", [264, 1024, 4096, 40000])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("bits", [4, 8])
def test_awkward_rows(cols, dtype, bits):
    x = values(10, 9, cols, dtype)
    x[0] = 0
    x[1] *= 2.0 ** 100          # squares beyond fp32
    x[2] = 3.3e38 * torch.sign(x[2].float())
    x[3] *= 2.0 ** -100         # far below eps
    x[4, cols // 2] = float("nan")
    x[5, 3] = float("inf")
    x[6, 1:] = 0                # one value alone
    x[7] = 2.0 ** 64
    y = torch.zeros_like(x)
    w = values(11, 1, cols, dtype)[0]
    q, s = buffers(9, cols, bits)
    norm = capmoe.make_norm(9, cols, 1e-6, TYPES[dtype], bits)
    capmoe.moe_norm_rows(norm, x, None, w, None, None, y, q, s)
    check(x, None, w, norm.eps, None, y, q, s, bits)


def test_sums_round_to_even_and_may_overflow():
    x = torch.tensor([[256.0, 256.0, 258.0, 3.3e38] * 2], dtype=BF16, device="cuda")
    r = torch.tensor([[1.0, 3.0, 1.0, 3.3e38] * 2], dtype=BF16, device="cuda")
    h, y = torch.zeros_like(x), torch.zeros_like(x)
    capmoe.moe_norm_rows(capmoe.make_norm(1, 8), x, r, None, None, h, y, None, None)
    assert h[0, :4].tolist() == [256.0, 260.0, 260.0, float("inf")]
    assert y[0, :3].tolist() == [0.0] * 3 and bool(torch.isnan(y[0, 3]))


def test_captured_norm_replays_on_its_stream():
    x, r, w = values(12, 37, 4096, BF16), values(13, 37, 4096, BF16), values(14, 1, 4096, BF16)[0]
    h, y = torch.zeros_like(x), torch.zeros_like(x)
    q, s = buffers(37, 4096, 4)
    norm = capmoe.make_norm(37, 4096, bits=4)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    capmoe.moe_norm_rows(norm, x, r, w, None, h, y, q, s, stream=side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        capmoe.moe_norm_rows(norm, x, r, w, None, h, y, q, s)
    for i in range(3):
        x.copy_(values(20 + i, 37, 4096, BF16))
        graph.replay()
        torch.cuda.synchronize()
        check(x, r, w, norm.eps, h, y, q, s, 4)


def test_many_rows():
    x, w = values(15, 20000, 264, BF16), values(16, 1, 264, BF16)[0]
    y = torch.zeros_like(x)
    q, s = buffers(20000, 264, 8)
    norm = capmoe.make_norm(20000, 264, bits=8)
    capmoe.moe_norm_rows(norm, x, None, w, None, None, y, q, s)
    check(x, None, w, norm.eps, None, y, q, s, 8)
