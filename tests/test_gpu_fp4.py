"""The 4-bit experts on the GPU against the formulas in 64 bits.

Quantising is exact: the same bytes.  A product of 4-bit numbers whose scales are near one another is exact in fp32 (multiples of
2^-4 below 2^20 here), so it is the 64-bit sum rounded to bf16 once: the same bits.  With scales of many sizes the sum loses at
most 2^-23 of the magnitudes for each of the K / 128 matrix instructions and a few more inside one: 2^-16 of them for any K here.

In the FFN the hidden activation is off by at most 2^-14 of itself before it is rounded (sums 2^-16 of the magnitudes, the
exponential and the reciprocal 2^-22).  A border between two 4-bit numbers or bf16 numbers next to one lies within that of at most
one value in 2^12, which then moves by half of itself at most: 2^-6 * 2^-1 = 2^-7 of the 2-norm.  With the rounding of the output
(2^-8) less than 2^-6.  One row may have all of a row's moves: of h values at most 1 + h / 2^9, each of at most twice the root of
the mean square or half of itself.
"""
import numpy as np
import pytest
import torch

import fp4_reference as ref
import fp8_reference as ref8
from paper_2503_05066_amd import capmoe

pytestmark = [pytest.mark.gpu, pytest.mark.usefixtures("built_library")]

BF16, F32 = torch.bfloat16, torch.float32
FFN_TOLERANCE = 2.0 ** -6


@pytest.fixture(autouse=True, scope="module")
def _device():
    torch.cuda.set_device(0)


def rng(*key):
    return np.random.default_rng(list(key))


def on(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def plain(t):
    return t.double().cpu().numpy()


# ---------------------------------------------------------------------------------------------
# quantising
# ---------------------------------------------------------------------------------------------
def awkward(g, r, c):
    """Values of many sizes with rows of zeros, the type's ends, exact ties and numbers that are not finite."""
    x = g.standard_normal((r, c)) * np.exp(3 * g.standard_normal((r, 1)))
    x[0] = 0
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    for i, f in enumerate((lambda v: v * 2.0 ** -125, lambda v: v * 2.0 ** -132, lambda v: np.where(v > 0, 3.3e38, -3.0e38),
                           lambda v: np.sign(v) * ties[np.arange(c) % 8], lambda v: np.where(v > 1, 2.0, 1.5), lambda v: -0.0 * np.ones(c))):
        if r > 1 + i:
            x[1 + i] = f(g.standard_normal(c))
    if r > 8:
        x[7, :: max(1, c // 3)] = np.nan
        x[8, 0], x[8, c - 1] = np.inf, -np.inf
    return x


ROWS = [(1, 8), (1, 64), (3, 72), (37, 4096), (9, 128), (11, 136), (64, 1416), (5, 520), (130, 2048), (2, 14336), (9, 1000)]


@pytest.mark.parametrize("rows,cols", ROWS)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_have_the_bytes_of_the_definition(rows, cols, dtype):
    x = on(awkward(rng(rows, cols), rows, cols), dtype)
    q, s = capmoe.fp4_row_buffers(rows, cols)
    q.fill_(0x55), s.fill_(0x55)
    capmoe.moe_quantize_rows_fp4(x, None, None, q, s)
    want_q, want_s = ref.quantize(plain(x))
    assert np.array_equal(s.cpu().numpy(), want_s) and np.array_equal(q.cpu().numpy(), want_q)
    for back in (BF16, F32):
        y = torch.full((rows, cols), 7.0, dtype=back, device="cuda")
        capmoe.moe_dequantize_rows(4, q, s, y)
        want = torch.from_numpy(ref.value(want_q, want_s)[:, :cols]).to(back).double().numpy()
        assert np.array_equal(plain(y), want, equal_nan=True)


@pytest.mark.parametrize("rows,cols", ROWS)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_eight_bit_rows_back_to_values(rows, cols, dtype):
    x = on(awkward(rng(rows, cols), rows, cols), F32)
    q, s = capmoe.fp8_row_buffers(rows, cols)
    capmoe.moe_quantize_rows(x, None, None, q, s)
    s[rows // 2, 0] = 255  # no number
    y = torch.full((rows, cols), 7.0, dtype=dtype, device="cuda")
    capmoe.moe_dequantize_rows(8, q, s, y)
    want = ref8.rows_value(q.cpu().numpy(), s.cpu().numpy())[:, :cols]
    want[rows // 2, :128] = np.nan
    assert np.array_equal(plain(y), torch.from_numpy(want).to(dtype).double().numpy(), equal_nan=True)


@pytest.mark.parametrize("cols", [4, 12, 36, 516, 1020])
def test_rows_of_fp32_that_end_in_the_middle_of_eight(cols):
    x = on(rng(4, cols).standard_normal((5, cols)), F32)
    q, s = capmoe.fp4_row_buffers(5, cols)
    capmoe.moe_quantize_rows_fp4(x, None, None, q, s)
    want_q, want_s = ref.quantize(plain(x))
    assert np.array_equal(q.cpu().numpy(), want_q) and np.array_equal(s.cpu().numpy(), want_s)
    y = torch.full((5, cols), 7.0, device="cuda")
    capmoe.moe_dequantize_rows(4, q, s, y)
    assert np.array_equal(plain(y), ref.value(want_q, want_s)[:, :cols])
    q8, s8 = capmoe.fp8_row_buffers(5, cols)
    capmoe.moe_quantize_rows(x, None, None, q8, s8)
    y.fill_(7.0)
    capmoe.moe_dequantize_rows(8, q8, s8, y)
    assert np.array_equal(plain(y), ref8.rows_value(q8.cpu().numpy(), s8.cpu().numpy())[:, :cols])


def test_rows_that_a_plan_names_more_than_once_and_out_of_order():
    p = Product([5, 0, 70], 520, 264, src=9)
    p.token[:] = np.array([8, 8, 0, 3, 3] + [8 - i % 9 for i in range(70)], np.int32)
    p.check(p.run())


def test_product_of_rows_beyond_31_bit_offsets():
    # 3 GiB of rows, fetched through a plan and in their order
    k, n, src = 12288, 128, 1 << 19
    x, xs = random_rows(src, k, 3)
    w, ws = random_rows(n, k, 4)
    pitch, scale_pitch = capmoe.moe_fp4_query(k)
    token = np.array([0, src - 1, src // 2, 5, src - 2, (1 << 31) // pitch, (1 << 31) // pitch + 1] * 20, np.int32)
    wv = device_value(w, ws)
    for rows, room in ((7, 7), (140, 140), (140, 20000)):
        offset = on(np.array([0, rows], np.int32))
        numbers = on(np.concatenate([token[:rows], np.zeros(room - rows, np.int32)]))
        y = torch.full((room, n), 7.0, dtype=BF16, device="cuda")
        capmoe.moe_grouped_gemm_fp4(capmoe.make_gemm(room, k, n, 1, src_rows=src), x, xs, numbers, offset, w.view(1, n, pitch),
                                    ws.view(1, n, scale_pitch), y)
        at = on(token[:rows]).long()
        assert torch.equal(y[:rows].double(), on(ref.to_bf16(plain(device_value(x[at], xs[at]) @ wv.T))))
    offset = on(np.array([0, 10, src], np.int32))
    y = torch.full((src, n), 7.0, dtype=BF16, device="cuda")
    capmoe.moe_grouped_gemm_fp4(capmoe.make_gemm(src, k, n, 2), x, xs, None, offset, torch.stack([w, w]).view(2, n, pitch),
                                torch.stack([ws, ws]).view(2, n, scale_pitch), y)
    for part in (slice(0, 300), slice(src // 2, src // 2 + 300), slice(src - 300, src)):
        assert torch.equal(y[part].double(), on(ref.to_bf16(plain(device_value(x[part], xs[part]) @ wv.T))))


@pytest.mark.parametrize("count", [-3, 0, 1, 40, 64, 1000])
def test_rows_are_permuted_and_those_behind_the_count_untouched(count):
    g = rng(7)
    x = on(g.standard_normal((20, 264)), BF16)
    token = g.integers(0, 20, 64).astype(np.int32)
    token[:4] = 19, 19, 0, 0
    q, s = capmoe.fp4_row_buffers(64, 264)
    q.fill_(0x33), s.fill_(0x33)
    capmoe.moe_quantize_rows_fp4(x, on(token), on(np.array([count], np.int32)), q, s)
    want_q, want_s = ref.quantize(plain(x)[token])
    n = min(max(count, 0), 64)
    got_q, got_s = q.cpu().numpy(), s.cpu().numpy()
    assert np.array_equal(got_q[:n], want_q[:n]) and np.array_equal(got_s[:n], want_s[:n])
    assert np.all(got_q[n:] == 0x33) and np.all(got_s[n:] == 0x33)


@pytest.mark.parametrize("e,n,k", [(1, 1, 8), (3, 130, 136), (2, 1000, 1416), (1, 128, 128), (5, 24, 520), (2, 256, 2048)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_weights_have_the_bytes_of_the_definition(e, n, k, dtype):
    w = rng(e, n, k).standard_normal((e, n, k))
    if n > 100:
        w[0, 1, 3], w[0, 2, 4] = np.nan, np.inf
        w[-1, :128, :128] = 0
        w[-1, -2:] *= 1e30
    w = on(w, dtype)
    q, s = capmoe.fp4_weight_buffers(e, n, k)
    q.fill_(0x55), s.fill_(0x55)
    capmoe.moe_quantize_weights_fp4(w, q, s)
    want_q, want_s = ref.quantize_weights(plain(w))
    assert np.array_equal(q.cpu().numpy(), want_q) and np.array_equal(s.cpu().numpy(), want_s)


def test_more_rows_than_the_grid_has_waves():
    x = on(rng(3).standard_normal((70000, 64)), BF16)
    q, s = capmoe.fp4_row_buffers(70000, 64)
    capmoe.moe_quantize_rows_fp4(x, None, None, q, s)
    want_q, want_s = ref.quantize(plain(x))
    assert np.array_equal(q.cpu().numpy(), want_q) and np.array_equal(s.cpu().numpy(), want_s)
    y = torch.zeros_like(x)
    capmoe.moe_dequantize_rows(4, q, s, y)
    assert np.array_equal(plain(y), ref.value(want_q, want_s)[:, :64])


# ---------------------------------------------------------------------------------------------
# products
# ---------------------------------------------------------------------------------------------
def filled(g, shape, cols, low, high):
    """4-bit rows of random codes and scale bytes from [low, high), zero behind the columns."""
    code = g.integers(0, 16, shape + (ref.up(cols, 256),)).astype(np.uint8)
    code[..., cols:] = 0
    blocks = ref.up(cols, 32) // 32
    scale = np.zeros(shape + (ref.up(cols, 512) // 32,), np.uint8)
    scale[..., ref.scale_places(blocks)] = g.integers(low, high, shape + (blocks,))
    return code[..., 0::2] | code[..., 1::2] << 4, scale


class Product:
    """4-bit rows and weights of the given sizes, as bytes."""

    def __init__(self, counts, k, n, src=0, seed=0, low=126, high=129):
        g = rng(seed, len(counts), k, n)
        self.offset = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        self.rows, self.e, self.k, self.n = int(self.offset[-1]), len(counts), k, n
        self.exact = high - low <= 3
        r = src or max(self.rows, 1)
        self.xq, self.xs = filled(g, (r,), k, low, high)
        self.wq, self.ws = filled(g, (self.e, ref.up(n, 128)), k, low, high)
        self.wq[:, n:], self.ws[:, n:] = 0, 0
        self.token = g.integers(0, r, max(self.rows, 1)).astype(np.int32) if src else None
        self.src = src

    def run(self, extra=0):
        g = capmoe.make_gemm(self.rows + extra, self.k, self.n, self.e, src_rows=self.src)
        y = torch.full((self.rows + extra, self.n), 7.0, dtype=BF16, device="cuda")
        self.keep = [on(a) for a in (self.xq, self.xs, self.offset, self.wq, self.ws)]
        token = None if self.token is None else on(np.concatenate([self.token, np.zeros(extra, np.int32)]))
        x, xs, off, w, wsc = self.keep
        capmoe.moe_grouped_gemm_fp4(g, x, xs, token, off, w, wsc, y)
        torch.cuda.synchronize()
        return y

    def check(self, y):
        want, mag = ref.gemm(ref.value(self.xq, self.xs), ref.value(self.wq, self.ws), self.offset, self.token)
        want, mag = want[:, : self.n], mag[:, : self.n]
        got = plain(y)[: self.rows]
        if self.exact:
            wrong = got != ref.to_bf16(want)
            assert not wrong.any(), (np.argwhere(wrong)[:5], wrong.mean())
        else:
            off = np.abs(got - want)
            limit = 2.0 ** -8 * np.abs(want) + 2.0 ** -16 * mag
            assert np.all(off <= limit), np.max(off / np.maximum(limit, 1e-300))


COUNTS = {"one": [1], "none": [0, 0, 0], "holes": [0, 1, 0, 17, 0], "sixteens": [16, 15, 33, 32], "tiles": [64, 65, 256, 255],
          "high": [257, 300, 0, 513], "ragged": [129, 3, 0, 160, 95, 224, 31, 200]}


@pytest.mark.parametrize("counts", COUNTS)
@pytest.mark.parametrize("k,n", [(128, 128), (8, 8), (520, 264), (256, 1000), (1416, 128), (2048, 256), (800, 136)])
def test_product(counts, k, n):
    p = Product(COUNTS[counts], k, n)
    y = p.run(extra=5)
    assert torch.all(y[p.rows:] == 7.0)  # rows behind the last expert's
    p.check(y)


@pytest.mark.parametrize("counts,k,n", [([40, 0, 300, 7], 520, 264), ([1, 1, 1], 2048, 1024), ([600], 768, 512)])
def test_product_through_a_plan(counts, k, n):
    p = Product(counts, k, n, src=50)
    p.check(p.run())


# Room for more rows than there are makes the row tiles higher (a rule on max_rows), here with every height in steps of 32; n: the
# narrow and the wide shape; k: odd and even numbers of slabs, down to one
@pytest.mark.parametrize("k", [8, 256, 512, 768, 1024, 1280, 1792, 2064, 2304, 4096])
@pytest.mark.parametrize("n,room", [(120, 20000), (264, 13000), (128, 40000), (392, 40000), (256, 60000), (512, 60000)])
def test_product_on_high_tiles(k, n, room):
    p = Product([1, 33, 70, 100, 0, 130, 161, 200, 230, 261, 768, 250], k, n)
    y = p.run(extra=room)
    assert torch.all(y[p.rows:] == 7.0)
    p.check(y)


@pytest.mark.parametrize("counts,k,n", [([300, 0, 70], 8, 102400), ([520, 30, 260, 600], 264, 39432)])
def test_product_of_many_rounds(counts, k, n):
    p = Product(counts, k, n)
    y = p.run(extra=1)
    assert torch.all(y[p.rows:] == 7.0)
    p.check(y)


@pytest.mark.parametrize("e,k,n,most", [(40, 520, 512, 8), (70, 136, 512, 8), (30, 1416, 1000, 16), (90, 512, 392, 40), (33, 8, 1032, 3)])
def test_product_of_many_experts_of_few_rows(e, k, n, most):
    g = rng(e, most)
    counts = g.integers(0, most + 1, e)
    if most > 16:
        counts[counts < 33] = 0
    p = Product(list(counts), k, n)
    p.check(p.run(extra=3))


@pytest.mark.parametrize("e,k,n", [(256, 512, 264), (130, 136, 512), (65, 768, 1024)])
def test_product_of_many_experts(e, k, n):
    g = rng(e)
    p = Product(list(g.choice([0, 0, 1, 17, 33, 40, 64, 65, 100, 255, 256, 257, 300, 512, 700], e)), k, n)
    p.check(p.run())


@pytest.mark.parametrize("counts,k,n", [([700, 20], 1280, 256), ([9, 30], 1024, 136), ([1], 14336, 264), ([300, 0, 77], 4104, 392)])
def test_product_of_scales_of_many_sizes(counts, k, n):
    p = Product(counts, k, n, low=100, high=140)
    p.check(p.run())
    p = Product(counts, k, n, src=61, low=100, high=140)
    p.check(p.run())


@pytest.mark.parametrize("counts", [[300], [5, 12]])
def test_every_block_has_its_own_scale(counts):
    # ones everywhere, scales alone differ: a scale taken from another row or k block shows as a power of two
    p = Product(counts, 1416, 392, low=122, high=132)
    p.xq[p.xq != 0], p.wq[p.wq != 0] = 0x22, 0x22  # e2m1 of 1
    p.check(p.run())


@pytest.mark.parametrize("counts", [[40, 300], [5, 12]])
def test_blocks_that_are_no_numbers_stay_by_themselves(counts):
    p = Product(counts, 520, 264)
    p.xs[3, ref.scale_places(17)[7]] = 255
    p.xq[4] = 0
    p.ws[1, 130, ref.scale_places(17)[16]] = 255
    got = plain(p.run())
    nan = np.zeros(got.shape, bool)
    nan[3], nan[counts[0]:, 130] = True, True
    assert np.array_equal(np.isnan(got), nan) and np.all(got[4] == 0)


@pytest.mark.parametrize("counts", [[5, 12], [300, 12]])
def test_the_largest_and_smallest_scale_bytes(counts):
    # 2^127 and 2^-127 meet as 1
    p = Product(counts, 520, 264)
    at = ref.scale_places(17)
    p.xs[:, at], p.ws[:, :264, at] = np.where(np.arange(17) % 2, 0, 254), np.where(np.arange(17) % 2, 254, 0)
    p.check(p.run())


def test_the_same_call_gives_the_same_bits():
    p = Product([700, 40, 0, 300, 1], 2048, 1024, seed=5, low=100, high=140)
    first = p.run()
    for _ in range(3):
        assert torch.equal(first, p.run())


@pytest.mark.parametrize("counts,most", [([3, 0, 7, 2], 4096), ([300, 0, 200, 12], 4096), ([1, 0, 4, 2], 12)])
def test_captured_product_follows_its_offsets(counts, most):
    # the grid depends on max_rows alone: a replay does the plan that its arrays then hold
    k, n = 520, 392
    p = Product([most // 4] * 4, k, n)
    y = torch.zeros((most, n), dtype=BF16, device="cuda")
    x, xs, off, w, ws = (on(a) for a in (p.xq, p.xs, p.offset, p.wq, p.ws))
    gemm = capmoe.make_gemm(most, k, n, 4)
    capmoe.moe_grouped_gemm_fp4(gemm, x, xs, None, off, w, ws, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        capmoe.moe_grouped_gemm_fp4(gemm, x, xs, None, off, w, ws, y)
    for now in (counts, [most // 4] * 4, counts[::-1], [0, 0, 0, 0], [most, 0, 0, 0]):
        p.offset = np.concatenate([[0], np.cumsum(now)]).astype(np.int32)
        p.rows = int(p.offset[-1])
        off.copy_(torch.from_numpy(p.offset))
        y.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.all(y[p.rows:] == 7.0)
        p.check(y)


def test_two_streams():
    p, r = Product([300, 20, 0, 64], 512, 384, seed=1), Product([5, 9, 1, 0], 640, 264, seed=2)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    inputs = [(capmoe.make_gemm(q.rows, q.k, q.n, q.e), [on(a) for a in (q.xq, q.xs, q.offset, q.wq, q.ws)],
               torch.zeros((q.rows, q.n), dtype=BF16, device="cuda")) for q in (p, r)]
    torch.cuda.synchronize()
    for _ in range(10):
        for st, (g, (x, xs, off, w, ws), y) in zip(streams, inputs):
            capmoe.moe_grouped_gemm_fp4(g, x, xs, None, off, w, ws, y, stream=st)
    torch.cuda.synchronize()
    for q, (_, _, y) in zip((p, r), inputs):
        q.check(y)


# ---------------------------------------------------------------------------------------------
# the FFN and the layer
# ---------------------------------------------------------------------------------------------
def layer(tokens, d, e, k, h, seed=0, **more):
    g = rng(seed, tokens, d, e, h)
    desc = capmoe.make_desc(tokens, d, e, k, h, **more)
    x = on(g.standard_normal((tokens, d)), BF16)
    weights = [on(g.standard_normal(s) * s[2] ** -0.5, BF16) for s in ((e, h, d), (e, h, d), (e, d, h))]
    return desc, x, weights, on(g.standard_normal((e, d)) * d ** -0.5, F32), on(g.standard_normal(e), F32)


def plan_of(g, tokens, counts):
    offset = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    token = np.concatenate([np.sort(g.choice(tokens, c, replace=False)) for c in counts] + [np.zeros(0)]).astype(np.int32)
    return offset, token


def four(x):
    q, s = capmoe.fp4_row_buffers(*x.shape)
    capmoe.moe_quantize_rows_fp4(x, None, None, q, s)
    return q, s


def assert_close(got, want, h, rows_too=True):
    off = got - want
    norms = np.linalg.norm(want, axis=1)
    assert np.linalg.norm(off) <= FFN_TOLERANCE * np.linalg.norm(want), np.linalg.norm(off) / np.linalg.norm(want)
    if rows_too:
        # 1 + h / 2^9 values of a row, each moved by twice the root of the mean square (or half of a value of four times it)
        most = 2.0 ** -8 + 2 * np.sqrt(1 + h / 512) / np.sqrt(h) * 1.5
        assert np.all(np.linalg.norm(off, axis=1) <= most * norms), (np.linalg.norm(off, axis=1) / norms).max() / most


FFN = [(300, 136, 2, 2, 51200, [300, 40]), (1, 256, 8, 2, 128, [1, 0, 0, 0, 0, 0, 0, 1]), (16, 512, 4, 2, 384, [16, 0, 7, 9]), (37, 264, 6, 2, 200, [37, 1, 0, 20, 16, 0]),
       (300, 256, 4, 2, 384, [300, 2, 0, 290]), (520, 1032, 3, 2, 136, [520, 64, 300]), (700, 384, 5, 2, 1416, [257, 700, 100, 0, 33]),
       (5, 136, 2, 1, 8, [2, 3]), (64, 264, 64, 2, 384, [2, 0, 1, 5] * 16), (40, 392, 40, 2, 264, [1, 4, 0, 2, 0] * 8),
       (90, 256, 1, 1, 384, [90]), (30, 640, 1, 1, 128, [29]), (12, 256, 256, 6, 128, [0, 1, 0, 0] * 64), (1000, 512, 8, 4, 640, [1000, 700, 512, 256, 255, 96, 0, 130])]


@pytest.mark.parametrize("tokens,d,e,k,h,counts", FFN)
def test_ffn(tokens, d, e, k, h, counts):
    desc, x, weights, _, _ = layer(tokens, d, e, k, h, mode=capmoe.MODE_NONE)
    offset, token = plan_of(rng(1, tokens), tokens, counts)
    rows = len(token)
    experts = capmoe.Fp4Experts.quantized(*weights)
    max_rows = capmoe.moe_query(desc)[2]
    ws = torch.empty(capmoe.moe_query_fp4(desc), dtype=torch.uint8, device="cuda")
    ws.fill_(0xFF)  # scale bytes of 255 where nothing was written
    yp = torch.full((max_rows + 3, d), 7.0, dtype=BF16, device="cuda")
    padded = np.zeros(max_rows, np.int32)
    padded[:rows] = token
    capmoe.moe_dispatch_ffn_fp4(desc, x, None, on(offset), on(padded), experts, yp, ws)
    got = plain(yp)
    assert np.all(got[rows:] == 7.0)
    values = [ref.value(*ref.quantize_weights(plain(w))) for w in weights]
    want = ref.ffn(ref.value(*ref.quantize(plain(x))), *values, offset, h, token)[:, :d]
    assert_close(got[:rows], want, h)
    # rows that are permuted already, in bf16 and in 4 bits, and tokens in 4 bits: the same bits
    xp = torch.zeros((max_rows, d), dtype=BF16, device="cuda")
    capmoe.moe_dispatch(desc, x, on(offset), on(padded), xp)
    xq, xs = four(x)
    for call in (lambda y: capmoe.moe_grouped_ffn_fp4(desc, xp, None, on(offset), experts, y, ws),
                 lambda y: capmoe.moe_grouped_ffn_fp4(desc, *four(xp), on(offset), experts, y, ws),
                 lambda y: capmoe.moe_dispatch_ffn_fp4(desc, xq, xs, on(offset), on(padded), experts, y, ws)):
        yp2 = torch.full_like(yp, 7.0)
        ws.fill_(0x5A)
        call(yp2)
        assert torch.equal(yp, yp2)


@pytest.mark.parametrize("tokens,d,k,h", [(5000, 136, 4, 128), (14000, 256, 4, 128), (14000, 136, 4, 264), (6000, 1032, 4, 384), (10000, 640, 4, 512)])
def test_ffn_on_high_tiles(tokens, d, k, h):
    counts = [1, 33, 70, 100, 0, 130, 161, 200, 230, 261, 768, 250]
    desc, x, weights, _, _ = layer(tokens, d, len(counts), k, h, mode=capmoe.MODE_NONE)
    offset, token = plan_of(rng(2, tokens), tokens, counts)
    rows = len(token)
    experts = capmoe.Fp4Experts.quantized(*weights)
    ws = torch.empty(capmoe.moe_query_fp4(desc), dtype=torch.uint8, device="cuda")
    ws.fill_(0xFF)
    yp = torch.full((tokens * k, d), 7.0, dtype=BF16, device="cuda")
    padded = np.zeros(tokens * k, np.int32)
    padded[:rows] = token
    capmoe.moe_dispatch_ffn_fp4(desc, x, None, on(offset), on(padded), experts, yp, ws)
    assert torch.all(yp[rows:] == 7.0)
    values = [ref.value(*ref.quantize_weights(plain(w))) for w in weights]
    want = ref.ffn(ref.value(*ref.quantize(plain(x)))[token], *values, offset, h)[:, :d]
    assert_close(plain(yp[:rows]), want, h)


@pytest.mark.parametrize("tokens", [4, 300])
def test_gates_that_are_shut(tokens):
    # gate -2^71 and up 2^71: their product leaves the range of fp32, silu(gate) * up is a zero
    desc, x, weights, _, _ = layer(tokens, 128, 2, 1, 128, mode=capmoe.MODE_NONE)
    x.fill_(2.0 ** 64)
    weights[0].fill_(-1.0), weights[1].fill_(1.0), weights[2].fill_(1.0)
    experts = capmoe.Fp4Experts.quantized(*weights)
    ws = torch.empty(capmoe.moe_query_fp4(desc), dtype=torch.uint8, device="cuda")
    yp = torch.full((tokens, 128), 7.0, dtype=BF16, device="cuda")
    capmoe.moe_grouped_ffn_fp4(desc, x, None, on(np.array([0, tokens // 2, tokens], np.int32)), experts, yp, ws)
    assert torch.all(yp == 0)


@pytest.mark.parametrize("tokens,counts", [(400, [300, 12, 0, 88]), (40, [12, 16, 0, 12])])
def test_a_token_that_is_not_a_number_stays_by_itself(tokens, counts):
    desc, x, weights, _, _ = layer(tokens, 256, 4, 1, 384, mode=capmoe.MODE_NONE)
    last = tokens - 5
    x[7, 3], x[20, 255] = float("nan"), float("inf")
    offset = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    token = np.arange(tokens, dtype=np.int32)
    token[[7, last]] = last, 7  # one among the first expert's rows, one among the last one's
    experts = capmoe.Fp4Experts.quantized(*weights)
    ws = torch.empty(capmoe.moe_query_fp4(desc), dtype=torch.uint8, device="cuda")
    yp = torch.zeros((tokens, 256), dtype=BF16, device="cuda")
    capmoe.moe_dispatch_ffn_fp4(desc, x, None, on(offset), on(token), experts, yp, ws)
    bad = np.isnan(plain(yp)).any(axis=1)
    assert set(np.flatnonzero(bad)) == {20, last}


@pytest.mark.parametrize("tokens,counts", [(12, [12, 3, 0, 9]), (300, [300, 64, 0, 211])])
def test_tokens_of_zeros_and_of_extreme_sizes(tokens, counts):
    desc, x, weights, _, _ = layer(tokens, 264, 4, 3, 200, mode=capmoe.MODE_NONE)
    x[1], x[2] = 0, 0
    x[3] *= 2.0 ** -100
    x[4] *= 2.0 ** 60  # the hidden activation reaches 2^120
    x[5, :128] = 0     # blocks of zeros beside others
    x[6] = 1e-40       # below the type's normal numbers
    offset, token = plan_of(rng(5, tokens), tokens, counts)
    experts = capmoe.Fp4Experts.quantized(*weights)
    ws = torch.empty(capmoe.moe_query_fp4(desc), dtype=torch.uint8, device="cuda")
    yp = torch.zeros((capmoe.moe_query(desc)[2], 264), dtype=BF16, device="cuda")
    padded = np.zeros(yp.shape[0], np.int32)
    padded[:len(token)] = token
    capmoe.moe_dispatch_ffn_fp4(desc, x, None, on(offset), on(padded), experts, yp, ws)
    got = plain(yp)[:len(token)]
    values = [ref.value(*ref.quantize_weights(plain(w))) for w in weights]
    want = ref.ffn(ref.value(*ref.quantize(plain(x))), *values, offset, 200, token)[:, :264]
    assert np.all(got[np.isin(token, (1, 2))] == 0)
    assert np.all(np.abs(got[np.isin(token, (3, 6))]) <= 2.0 ** -90)
    rest = ~np.isin(token, (1, 2, 3, 6))
    assert_close(got[rest] / np.abs(want[rest]).max(axis=1, keepdims=True), want[rest] / np.abs(want[rest]).max(axis=1, keepdims=True), 200)


@pytest.mark.parametrize("tokens,counts", [(12, [12, 3, 0, 9]), (300, [300, 64, 0, 211])])
@pytest.mark.parametrize("h", [203, 259])
def test_hidden_widths_that_are_no_multiple_of_8(tokens, counts, h):
    # the down weights of such a width are quantised with columns of zeros behind it
    desc, x, (gate, up, down), _, _ = layer(tokens, 264, 4, 3, h, mode=capmoe.MODE_NONE)
    with pytest.raises(capmoe.CapMoeError):
        capmoe.Fp4Experts.quantized(gate, up, down)
    experts = capmoe.Fp4Experts.quantized(gate, up, torch.nn.functional.pad(down, (0, -h % 8)))
    offset, token = plan_of(rng(5, tokens), tokens, counts)
    ws = torch.empty(capmoe.moe_query_fp4(desc), dtype=torch.uint8, device="cuda")
    ws.fill_(0xFF)
    yp = torch.zeros((capmoe.moe_query(desc)[2], 264), dtype=BF16, device="cuda")
    padded = np.zeros(yp.shape[0], np.int32)
    padded[:len(token)] = token
    capmoe.moe_dispatch_ffn_fp4(desc, x, None, on(offset), on(padded), experts, yp, ws)
    values = [ref.value(*ref.quantize_weights(plain(w))) for w in (gate, up, down)]
    want = ref.ffn(ref.value(*ref.quantize(plain(x))), *values, offset, h, token)[:, :264]
    assert_close(plain(yp)[:len(token)], want, h)


# offsets from elsewhere, within P_max: capacities of 16 rows, 128 in all, and an expert with up to all of them
@pytest.mark.parametrize("counts", [[0, 0, 128, 0, 0, 0, 0, 0], [16, 17, 33, 0, 0, 1, 0, 50], [1, 0, 0, 100, 2, 17, 0, 1], [64, 0, 0, 0, 0, 0, 0, 64]])
def test_ffn_of_few_rows_with_long_experts(counts):
    desc, x, weights, _, _ = layer(128, 264, 8, 1, 392, mode=capmoe.MODE_TOKEN_DROP, capacity_scope=capmoe.SCOPE_GLOBAL, gamma=1.0)
    assert capmoe.moe_query(desc)[0] == 16 and capmoe.moe_query(desc)[2] == 128
    offset = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    rows, token = int(offset[-1]), rng(12).integers(0, 128, 128).astype(np.int32)
    experts = capmoe.Fp4Experts.quantized(*weights)
    ws = torch.empty(capmoe.moe_query_fp4(desc), dtype=torch.uint8, device="cuda")
    yp = torch.full((128, 264), 7.0, dtype=BF16, device="cuda")
    capmoe.moe_dispatch_ffn_fp4(desc, x, None, on(offset), on(token), experts, yp, ws)
    assert torch.all(yp[rows:] == 7.0)
    values = [ref.value(*ref.quantize_weights(plain(w))) for w in weights]
    want = ref.ffn(ref.value(*ref.quantize(plain(x))), *values, offset, 392, token[:rows])[:, :264]
    assert_close(plain(yp[:rows]), want, 392)


LAYERS = [dict(tokens=64, d=256, e=8, k=2, h=384, device_groups=4, mode=capmoe.MODE_EXPANDED_DROP),
          dict(tokens=512, d=512, e=16, k=4, h=640, mode=capmoe.MODE_TOKEN_DROP, gamma=1.5),
          dict(tokens=1, d=264, e=8, k=2, h=200, mode=capmoe.MODE_NONE),
          dict(tokens=300, d=256, e=4, k=1, h=128, mode=capmoe.MODE_TOKEN_DROP, gamma=0.0),
          dict(tokens=0, d=256, e=4, k=2, h=128, mode=capmoe.MODE_TOKEN_DROP),
          dict(tokens=2048, d=256, e=8, k=2, h=256, mode=capmoe.MODE_TOKEN_DROP, capacity_scope=capmoe.SCOPE_GLOBAL)]


def separate(desc, x, w_router, bias, experts):
    buf = capmoe.LayerBuffers(desc, fp4=True)
    capmoe.moe_route_topk(desc, x, w_router, bias, 0, buf.logits, buf.scores, buf.topk_idx, buf.topk_score, buf.workspace)
    capmoe.moe_capacity_drop(desc, buf.scores, buf.topk_idx, buf.expert_count, buf.seg_count, buf.expert_offset, buf.row_token,
                             buf.row_weight, buf.pair_row, buf.workspace)
    capmoe.moe_dispatch_ffn_fp4(desc, x, None, buf.expert_offset, buf.row_token, experts, buf.yp, buf.workspace)
    capmoe.moe_combine(desc, buf.yp, buf.row_weight, buf.pair_row, buf.y)
    return buf


@pytest.mark.parametrize("case", range(len(LAYERS)))
@pytest.mark.parametrize("small_rows", [False, True])
def test_layer_is_the_separate_calls(case, small_rows):
    desc, x, weights, w_router, bias = layer(**LAYERS[case])
    experts = capmoe.Fp4Experts.quantized(*weights)
    want = separate(desc, x, w_router, bias, experts)
    got = capmoe.LayerBuffers(desc, fp4=True)
    got.workspace.fill_(0xA5)
    xq, xs = four(x) if small_rows and desc.n_tokens else (None, None)
    capmoe.moe_layer_forward_fp4(desc, x, xq, xs, w_router, bias, experts, None, 0, got)
    rows = int(want.expert_offset[-1])
    assert torch.equal(got.expert_offset, want.expert_offset) and torch.equal(got.pair_row, want.pair_row)
    assert torch.equal(got.yp[:rows], want.yp[:rows]) and torch.equal(got.y, want.y)
    # and near the same layer in bf16: a value is off by a fourth of itself at most, 2^-3 in the mean square, in both operands of the
    # three products
    buf = capmoe.LayerBuffers(desc)
    if desc.d_model % 128 == 0 and desc.d_hidden % 128 == 0 and rows:
        y = capmoe.moe_layer_forward(desc, x, w_router, bias, *weights, None, 0, buf)
        assert float((y.float() - got.y.float()).norm() / y.float().norm()) < 0.5


def test_norm_and_layers_one_after_the_other():
    # h += previous output; norm; layer, as a stack of layers runs them, captured and replayed
    desc, x, weights, w_router, bias = layer(**LAYERS[1])
    experts = capmoe.Fp4Experts.quantized(*weights)
    n, d = x.shape
    weight = on(1 + 0.1 * rng(8).standard_normal(d), BF16)
    norm = capmoe.make_norm(n, d, 1e-6, bits=4)

    def buffers():
        return [torch.zeros_like(x), torch.zeros_like(x), *capmoe.fp4_row_buffers(n, d), capmoe.LayerBuffers(desc, fp4=True)]

    def run(b, start):
        h, y, q, s, buf = b
        h.copy_(start)
        buf.y.zero_()
        for _ in range(3):
            capmoe.moe_norm_rows(norm, buf.y, h, weight, None, h, y, q, s)
            capmoe.moe_layer_forward_fp4(desc, y, q, s, w_router, bias, experts, None, 0, buf)

    b = buffers()
    run(b, x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(b, x)
    for i in range(3):
        x.copy_(on(rng(60 + i).standard_normal((n, d)), BF16))
        graph.replay()
        # by the single calls
        h, out = x, torch.zeros_like(x)
        for _ in range(3):
            s, y = torch.zeros_like(x), torch.zeros_like(x)
            capmoe.moe_norm_rows(capmoe.make_norm(n, d, 1e-6), out, h, weight, None, s, y, None, None)
            h, out = s, separate(desc, y, w_router, bias, experts).y
        torch.cuda.synchronize()
        assert torch.equal(b[0], h) and torch.equal(b[1], y) and torch.equal(b[4].y, out), i


def test_calls_on_two_streams_at_once():
    cases = [layer(**LAYERS[i], seed=9) for i in (0, 1, 5)]
    experts = [capmoe.Fp4Experts.quantized(*c[2]) for c in cases]
    want = []
    for (desc, x, _, w_router, bias), e in zip(cases, experts):
        buf = capmoe.LayerBuffers(desc, fp4=True)
        capmoe.moe_layer_forward_fp4(desc, x, None, None, w_router, bias, e, None, 0, buf)
        want.append(buf)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [capmoe.LayerBuffers(c[0], fp4=True) for c in cases]
    torch.cuda.synchronize()
    for _ in range(5):
        for (desc, x, _, w_router, bias), e, buf, stream in zip(cases, experts, got, streams):
            capmoe.moe_layer_forward_fp4(desc, x, None, None, w_router, bias, e, None, 0, buf, stream=stream)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a.y, b.y) and torch.equal(a.expert_offset, b.expert_offset)


# ---------------------------------------------------------------------------------------------
# Cases by the form that the call takes (test_fp4_forms.py holds the forms against the rules): few rows with 4, 2 or 1 waves to a weight
# row, or column width x row tile.  (rows per expert, columns of x, columns of y, form)
# ---------------------------------------------------------------------------------------------
PRODUCT_FORMS = [
    ([128], 520, 4104, "128x64"), ([0, 60, 0, 4], 2568, 264, "few/4"), ([0, 120, 0, 8], 264, 392, "few/4"),
    ([1, 0] * 8 + [70, 0, 22], 136, 1032, "few/2"), ([3, 0, 1, 40] + [1] * 16 + [33], 1032, 1000, "few/2"),
    ([0, 1] * 20 + [65, 0, 23], 520, 1032, "few/1"), ([100] + [0, 1] * 14, 2056, 2056, "few/1"),
    ([600, 1, 700, 0, 333, 200, 9, 3, 64, 128, 12, 288], 520, 4352, "256x256"), ([300, 1, 400, 0, 33, 200, 9, 3, 64, 128, 12, 88], 1032, 4352, "256x128"),
    ([300, 1, 0, 20], 1032, 136, "128x64"), ([700, 1, 400], 264, 2048, "128x128"), ([900, 33, 0, 400], 776, 3712, "128x256"),
    ([40, 1, 0, 20, 33, 0, 9, 3, 2, 1, 12, 8], 392, 4352, "256x64")]


@pytest.mark.parametrize("counts,k,n,form", PRODUCT_FORMS)
def test_product_of_every_form(counts, k, n, form):
    p = Product(counts, k, n)
    p.check(p.run())
    p = Product(counts, k, n, src=31)
    p.check(p.run())


def random_rows(n, k, seed):
    """4-bit rows on the device: random codes, scale bytes 126 to 128."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, s = capmoe.fp4_row_buffers(n, k)
    assert k % 512 == 0 or k % 512 == 256
    q.random_(0, 256, generator=g)
    s.random_(126, 129, generator=g)
    if k % 512:
        s.view(n, -1, 4, 4)[:, -1, :, 2:] = 0
    return q, s


def device_value(q, s):
    """4-bit rows in 64 bits on the device."""
    levels = torch.tensor(ref.E2M1, device="cuda")
    code = torch.stack([q & 15, q >> 4], dim=2).flatten(1)
    byte = s.view(len(s), -1, 4, 4).transpose(2, 3).reshape(s.shape)[:, : code.shape[1] // 32]
    return levels[code.long()] * torch.exp2(byte.double() - 127).repeat_interleave(32, 1)


# every height in steps of 32 rows, and experts with two tiles (whose weights are kept)
HEIGHTS = [256, 225, 200, 161, 129, 100, 65, 40, 31, 300, 0, 1]
STREAMED_PRODUCTS = [(HEIGHTS, 14336, 6144, "256x256 stream"), (HEIGHTS, 14080, 6144, "256x256 stream"), (HEIGHTS, 14080, 4352, "256x128 stream"), (HEIGHTS, 15616, 3712, "128x256 stream"),
                     ([5, 0, 1, 16, 9, 0, 2, 30, 0, 1, 0, 0], 14336, 4096, "few/2 stream"), ([1, 0, 1, 0, 0, 2, 0, 0, 1, 0, 0, 0], 14080, 4096, "few/4 stream"),
                     ([3, 0, 1, 0, 33, 2, 0, 0, 1, 0, 0, 0], 3328, 20480, "few/1 stream"), ([3, 0, 1, 0, 33, 2, 0, 0, 1, 0, 0, 0], 7936, 8192, "few/2 stream")]


@pytest.mark.parametrize("counts,k,n,form", STREAMED_PRODUCTS)
def test_streamed_product_of_every_form(counts, k, n, form):
    # odd and even numbers of slabs: walks over k that begin in the middle wrap around
    e, rows = len(counts), sum(counts)
    pitch, scale_pitch = capmoe.moe_fp4_query(k)
    w, ws = random_rows(e * n, k, 1)
    x, xs = random_rows(rows, k, 2)
    offset = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    y = torch.full((rows, n), 7.0, dtype=BF16, device="cuda")
    capmoe.moe_grouped_gemm_fp4(capmoe.make_gemm(rows, k, n, e), x, xs, None, on(offset), w.view(e, n, pitch), ws.view(e, n, scale_pitch), y)
    xv = device_value(x, xs)
    for i in range(e):
        if counts[i]:
            want = xv[offset[i]:offset[i + 1]] @ device_value(w[i * n:(i + 1) * n], ws[i * n:(i + 1) * n]).T
            assert torch.equal(y[offset[i]:offset[i + 1]].double(), on(ref.to_bf16(plain(want)))), i


# tokens, top-k, rows per expert, d, h, forms of the two products
STREAMED_FFNS = [(600, 4, HEIGHTS, 4352, 4608, "128x256 256x256 stream"), (600, 4, HEIGHTS, 4224, 4480, "128x256 128x256 stream"),
                 (24, 2, [16, 3, 0, 1, 24, 0, 2, 0, 0, 1, 0, 0], 4352, 4480, "few/2 few/2 stream"), (2, 2, [0, 2, 0, 0, 0, 1, 0, 0, 0, 0, 1, 0], 4096, 4608, "few/2 few/4 stream"),
                 (1, 2, [0, 0, 0, 1, 0, 0, 0, 0, 0, 0, 0, 1], 5120, 4096, "few/4 few/4 stream"), (90, 1, [40, 0, 0, 33, 0, 0, 9, 0, 0, 0, 0, 8], 3328, 6144, "few/1 few/2 stream")]


@pytest.mark.parametrize("tokens,k,counts,d,h,forms", STREAMED_FFNS)
def test_streamed_ffn_of_every_form(tokens, k, counts, d, h, forms):
    e, rows = len(counts), sum(counts)
    desc = capmoe.make_desc(tokens, d, e, k, h, mode=capmoe.MODE_NONE)
    g = torch.Generator(device="cuda").manual_seed(tokens)
    parts = []
    for n, c in ((h, d), (h, d), (d, h)):
        q, s = capmoe.fp4_weight_buffers(e, n, c)
        for i in range(e):
            w = torch.randn((1, n, c // 128, 128), generator=g, device="cuda") * c ** -0.5
            w *= torch.exp2(torch.randint(-2, 3, (1, n, c // 128, 1), generator=g, device="cuda").float())
            capmoe.moe_quantize_weights_fp4(w.view(1, n, c), q[i:i + 1], s[i:i + 1])
        parts.append((q, s))
    experts = capmoe.Fp4Experts(*[t for p in parts for t in p])
    x = on(rng(31, tokens).standard_normal((tokens, d)), BF16)
    offset, token = plan_of(rng(32, tokens), tokens, counts)
    padded = np.zeros(max(tokens * k, rows), np.int32)
    padded[:rows] = token
    yp = torch.full((tokens * k, d), 7.0, dtype=BF16, device="cuda")
    ws = torch.empty(capmoe.moe_query_fp4(desc), dtype=torch.uint8, device="cuda")
    ws.fill_(0xFF)
    capmoe.moe_dispatch_ffn_fp4(desc, x, None, on(offset), on(padded), experts, yp, ws)
    assert torch.all(yp[rows:] == 7.0)
    xv = on(ref.value(*ref.quantize(plain(x)))[token])
    want = np.zeros((rows, d))
    for i in np.flatnonzero(counts):
        gate, up, down = (device_value(q[i], s[i]) for q, s in parts)
        a = xv[offset[i]:offset[i + 1]]
        gv, uv = plain(a @ gate.T), plain(a @ up.T)
        hidden = ref.value(*ref.quantize(ref.to_bf16(gv / (1 + np.exp(-gv)) * uv)[:, :h]))
        want[offset[i]:offset[i + 1]] = plain(on(hidden) @ down.T)[:, :d]
    assert_close(plain(yp[:rows]), want, h)
