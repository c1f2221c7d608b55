"""The 8-bit experts on the GPU against the formulas in 64 bits.

Quantising is exact: the same bytes.  A product's result differs from the 64-bit sum by its one rounding to bf16, at most
2^-8 of the value, and by what the matrix cores' fp32 sums lose: the 8-bit instructions add the products of a few k with
their bits aligned to the largest one, which costs up to 2^-12 of the sum of their magnitudes (2^-13.4 on bytes drawn
evenly from the whole type).  In the FFN a hidden value that lies that close to a border between two 8-bit values may fall
on the other side: 2^-13 against steps of 2^-3 is one value in 2^10, off by 2^-4 to 2^-3, which adds at most
2^-3 * 2^-5 = 2^-8 to the 2-norm; with the two roundings to bf16 less than 2^-7.
"""
import numpy as np
import pytest
import torch

import fp8_reference as ref
from paper_2503_05066_amd import capmoe

pytestmark = [pytest.mark.gpu, pytest.mark.usefixtures("built_library")]

BF16, F32 = torch.bfloat16, torch.float32


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


def awkward(g, r, c):
    """Values of many sizes with rows of zeros, the type's ends, exact ties and numbers that are not finite."""
    x = g.standard_normal((r, c)) * np.exp(3 * g.standard_normal((r, 1)))
    x[0] = 0
    for i, f in enumerate((lambda v: v * 2.0 ** -125, lambda v: v * 2.0 ** -132, lambda v: np.where(v > 0, 3.3e38, -3.0e38),
                           lambda v: 448.0 * np.sign(v), lambda v: np.where(v > 1, 2.0, 1.5), lambda v: -0.0 * np.ones(c))):
        if r > 1 + i:
            x[1 + i] = f(g.standard_normal(c))
    if r > 8:
        x[7, :: max(1, c // 3)] = np.nan
        x[8, 0], x[8, c - 1] = np.inf, -np.inf
    return x


ROWS = [(1, 8), (1, 64), (3, 72), (37, 4096), (9, 128), (11, 136), (64, 1416), (5, 520), (130, 2048), (2, 14336)]


@pytest.mark.parametrize("rows,cols", ROWS)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_have_the_bytes_of_the_definition(rows, cols, dtype):
    x = on(awkward(rng(rows, cols), rows, cols), dtype)
    q, s = capmoe.fp8_row_buffers(rows, cols)
    q.fill_(0x55), s.fill_(0x55)
    capmoe.moe_quantize_rows(x, None, None, q, s)
    want_q, want_s = ref.quantize_rows(plain(x))
    assert np.array_equal(s.cpu().numpy(), want_s)
    got = q.cpu().numpy()
    nan = (want_q & 127) == 127
    assert np.array_equal(np.where(nan, 0, got), np.where(nan, 0, want_q)) and np.all(got[nan] & 127 == 127)


def test_rows_narrower_than_a_block_of_fp32():
    x = on(rng(4).standard_normal((5, 4)), F32)
    q, s = capmoe.fp8_row_buffers(5, 4)
    capmoe.moe_quantize_rows(x, None, None, q, s)
    want_q, want_s = ref.quantize_rows(plain(x))
    assert np.array_equal(q.cpu().numpy(), want_q) and np.array_equal(s.cpu().numpy(), want_s)


@pytest.mark.parametrize("count", [-3, 0, 1, 40, 64, 1000])
def test_rows_are_permuted_and_those_behind_the_count_untouched(count):
    g = rng(7)
    x = on(g.standard_normal((20, 264)), BF16)
    token = g.integers(0, 20, 64).astype(np.int32)
    token[:4] = 19, 19, 0, 0
    q, s = capmoe.fp8_row_buffers(64, 264)
    q.fill_(0x33), s.fill_(0x33)
    capmoe.moe_quantize_rows(x, on(token), on(np.array([count], np.int32)), q, s)
    want_q, want_s = ref.quantize_rows(plain(x)[token])
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
    q, s = capmoe.fp8_weight_buffers(e, n, k)
    q.fill_(0x55), s.fill_(0x55)
    capmoe.moe_quantize_weights(w, q, s)
    want_q, want_s = ref.quantize_weights(plain(w))
    got = q.cpu().numpy()
    nan = (want_q & 127) == 127
    assert np.array_equal(s.cpu().numpy(), want_s)
    assert np.array_equal(np.where(nan, 0, got), np.where(nan, 0, want_q)) and np.all(got[nan] & 127 == 127)


class Product:
    """8-bit rows and weights of the given sizes, on the device and as 64-bit values."""

    def __init__(self, counts, k, n, src=0, seed=0, scale_spread=0.0):
        g = rng(seed, len(counts), k, n)
        self.offset = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        self.rows, self.e, self.k, self.n = int(self.offset[-1]), len(counts), k, n
        r = src or max(self.rows, 1)
        x = g.standard_normal((r, k)) * np.exp(scale_spread * g.standard_normal((r, k)))
        w = g.standard_normal((self.e, n, k)) * k ** -0.5 * np.exp(scale_spread * g.standard_normal((self.e, n, k)))
        self.xq, self.xs = ref.quantize_rows(x)
        self.wq, self.ws = ref.quantize_weights(w)
        self.token = g.integers(0, r, max(self.rows, 1)).astype(np.int32) if src else None
        self.src = src

    def run(self, extra=0, workspace=None):
        g = capmoe.make_gemm(self.rows + extra, self.k, self.n, self.e, src_rows=self.src)
        y = torch.full((self.rows + extra, self.n), 7.0, dtype=BF16, device="cuda")
        self.keep = [on(a) for a in (self.xq, self.xs, self.offset, self.wq, self.ws)]
        token = None if self.token is None else on(np.concatenate([self.token, np.zeros(extra, np.int32)]))
        ws = torch.empty(capmoe.moe_gemm_query(g), dtype=torch.uint8, device="cuda")
        ws.fill_(0xA5)
        x, xs, off, w, wsc = self.keep
        capmoe.moe_grouped_gemm_fp8(g, x, xs, token, off, w, wsc, y, ws)
        torch.cuda.synchronize()
        return y

    def check(self, y):
        want, mag = ref.gemm(ref.rows_value(self.xq, self.xs), ref.weights_value(self.wq, self.ws), self.offset, self.token)
        want, mag = want[:, : self.n], mag[:, : self.n]
        got = plain(y)[: self.rows]
        off = np.abs(got - want)
        assert np.all(off <= 2.0 ** -8 * np.abs(want) + 2.0 ** -12 * mag), np.max(off / (2.0 ** -8 * np.abs(want) + 2.0 ** -12 * mag))
        assert np.linalg.norm(off) <= 2.0 ** -8 * np.linalg.norm(want)


COUNTS = {"one": [1], "none": [0, 0, 0], "holes": [0, 1, 0, 17, 0], "sixteens": [16, 15, 33, 32], "tiles": [64, 65, 256, 255],
          "high": [257, 300, 0, 513], "ragged": [129, 3, 0, 160, 95, 224, 31, 200]}


@pytest.mark.parametrize("counts", COUNTS)
@pytest.mark.parametrize("k,n", [(128, 128), (8, 8), (520, 264), (256, 1000), (1416, 128), (2048, 256)])
def test_product(counts, k, n):
    p = Product(COUNTS[counts], k, n)
    y = p.run(extra=5)
    assert torch.all(y[p.rows:] == 7.0)  # rows behind the last expert's
    p.check(y)


@pytest.mark.parametrize("counts,k,n", [([40, 0, 300, 7], 520, 264), ([1, 1, 1], 2048, 1024), ([600], 384, 512)])
def test_product_through_a_plan(counts, k, n):
    p = Product(counts, k, n, src=50)
    p.check(p.run())


# Room for more rows than there are makes the row tiles higher (a rule on max_rows): 128 and 256 rows, here with every height in
# steps of 32; n: the narrow and the wide shape
@pytest.mark.parametrize("k", [8, 128, 256, 384, 512, 640, 896, 1032, 1152, 2048])
@pytest.mark.parametrize("n,room", [(120, 20000), (264, 13000), (128, 40000), (392, 40000), (256, 60000), (512, 60000)])
def test_product_on_high_tiles(k, n, room):
    p = Product([1, 33, 70, 100, 0, 130, 161, 200, 230, 261, 768, 250], k, n)
    y = p.run(extra=room)
    assert torch.all(y[p.rows:] == 7.0)
    p.check(y)


@pytest.mark.parametrize("counts,k,n", [([300, 0, 70], 8, 102400), ([520, 30, 260, 600], 136, 39432)])
def test_product_of_many_rounds(counts, k, n):
    # more than 4.5 items for every compute unit: another order of the work
    p = Product(counts, k, n)
    y = p.run(extra=1)
    assert torch.all(y[p.rows:] == 7.0)
    p.check(y)


@pytest.mark.parametrize("e,k,n,most", [(40, 520, 512, 8), (70, 136, 512, 8), (30, 1416, 1000, 16), (90, 256, 392, 40), (33, 8, 1032, 3)])
def test_product_of_many_experts_of_few_rows(e, k, n, most):
    # two and one of a block's waves share a weight row; more than one pass over an expert's weights
    g = rng(e, most)
    counts = g.integers(0, most + 1, e)
    if most > 16:
        counts[counts < 33] = 0
    p = Product(list(counts), k, n)
    p.check(p.run(extra=3))


@pytest.mark.parametrize("e,k,n", [(256, 256, 264), (130, 136, 512), (65, 384, 1024)])
def test_product_of_many_experts(e, k, n):
    g = rng(e)
    p = Product(list(g.choice([0, 0, 1, 17, 33, 40, 64, 65, 100, 255, 256, 257, 300, 512, 700], e)), k, n)
    p.check(p.run())


@pytest.mark.parametrize("counts", [[300, 256, 1, 0, 65, 40, 129, 16, 520, 200, 33, 225], [1, 2, 16, 0, 5, 9, 3, 16, 4, 8, 0, 12]])
def test_product_whose_weights_are_streamed(counts):
    # more weights than the memory-side cache holds: other fetch policies, walks over k that begin at different places
    e, k, n = len(counts), 14336, 2176
    g = torch.Generator(device="cuda").manual_seed(sum(counts))

    def values(*shape):
        q = torch.randint(0, 256, shape, generator=g, device="cuda", dtype=torch.uint8)
        return torch.where((q & 127) > 0x47, q & 0xBF, q)  # magnitudes below 4

    x, w = values(sum(counts), k), values(e, n, k)
    xs = torch.randint(122, 132, (sum(counts), 112), generator=g, device="cuda", dtype=torch.uint8)
    ws = torch.randint(122, 132, (e, n // 128, 112), generator=g, device="cuda", dtype=torch.uint8)
    offset = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    y = torch.full((sum(counts), n), 7.0, dtype=BF16, device="cuda")
    gemm = capmoe.make_gemm(sum(counts), k, n, e)
    capmoe.moe_grouped_gemm_fp8(gemm, x, xs, None, on(offset), w, ws, y, torch.empty(0, dtype=torch.uint8, device="cuda"))
    f8 = torch.float8_e4m3fn
    xv = x.view(f8).double() * torch.exp2(xs.double() - 127).repeat_interleave(128, 1)
    for i in range(e):
        if counts[i]:
            wv = w[i].view(f8).double() * torch.exp2(ws[i].double() - 127).repeat_interleave(128, 0).repeat_interleave(128, 1)
            a = xv[offset[i]:offset[i + 1]]
            want, mag = a @ wv.T, a.abs() @ wv.abs().T
            off = (y[offset[i]:offset[i + 1]].double() - want).abs()
            assert bool((off <= 2.0 ** -8 * want.abs() + 2.0 ** -12 * mag).all()), i


@pytest.mark.parametrize("counts,k,n", [([700, 20], 640, 256), ([9, 30], 1024, 136)])
def test_product_of_values_of_many_sizes(counts, k, n):
    p = Product(counts, k, n, scale_spread=2.0)
    p.check(p.run())


@pytest.mark.parametrize("counts", [[300], [5, 12]])
def test_every_block_has_its_own_scale(counts):
    # ones everywhere, scales alone differ: a scale taken from another row, column block or k block shows as a power of two
    p = Product(counts, 1416, 392)
    g = rng(3)
    kb = 12
    p.xq[:], p.wq[:] = 0x38, 0x38  # e4m3 of 1
    p.xs[:, :kb] = g.integers(120, 134, p.xs[:, :kb].shape)
    p.ws[:, :, :kb] = g.integers(120, 134, p.ws[:, :, :kb].shape)
    p.check(p.run())


def test_nan_and_zero_rows_stay_by_themselves():
    p = Product([40, 300], 512, 256)
    p.xq[3, 100] = 0x7F
    p.xq[50, 511] = 0xFF
    p.xq[51] = 0
    got = plain(p.run())
    assert np.all(np.isnan(got[[3, 50]])) and np.all(got[51] == 0)
    rest = np.delete(np.arange(340), [3, 50])
    assert np.all(np.isfinite(got[rest]))


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


FFN = [(300, 136, 2, 2, 51200, [300, 40]), (1, 256, 8, 2, 128, [1, 0, 0, 0, 0, 0, 0, 1]), (16, 512, 4, 2, 384, [16, 0, 7, 9]), (37, 264, 6, 2, 200, [37, 1, 0, 20, 16, 0]),
       (300, 256, 4, 2, 384, [300, 2, 0, 290]), (520, 1032, 3, 2, 136, [520, 64, 300]), (700, 384, 5, 2, 1416, [257, 700, 100, 0, 33]),
       (5, 136, 2, 1, 8, [2, 3]), (64, 264, 64, 2, 384, [2, 0, 1, 5] * 16), (40, 392, 40, 2, 264, [1, 4, 0, 2, 0] * 8),
       (90, 256, 1, 1, 384, [90]), (30, 640, 1, 1, 128, [29]), (12, 256, 256, 6, 128, [0, 1, 0, 0] * 64), (1000, 512, 8, 4, 640, [1000, 700, 512, 256, 255, 96, 0, 130])]


@pytest.mark.parametrize("tokens,d,e,k,h,counts", FFN)
def test_ffn(tokens, d, e, k, h, counts):
    desc, x, weights, _, _ = layer(tokens, d, e, k, h, mode=capmoe.MODE_NONE)
    offset, token = plan_of(rng(1, tokens), tokens, counts)
    rows = len(token)
    assert rows <= tokens * k or tokens < 10
    experts = capmoe.Fp8Experts.quantized(*weights)
    max_rows = capmoe.moe_query(desc)[2]
    ws = torch.empty(capmoe.moe_query_fp8(desc), dtype=torch.uint8, device="cuda")
    ws.fill_(0xA5)
    yp = torch.full((max_rows + 3, d), 7.0, dtype=BF16, device="cuda")
    padded = np.zeros(max_rows, np.int32)
    padded[:rows] = token
    capmoe.moe_dispatch_ffn_fp8(desc, x, on(offset), on(padded), experts, yp, ws)
    got = plain(yp)
    assert np.all(got[rows:] == 7.0)
    values = [ref.weights_value(*ref.quantize_weights(plain(w))) for w in weights]
    want = ref.ffn(plain(x), *values, offset, token)[:, :d]
    off = got[:rows] - want
    assert np.linalg.norm(off) <= 2.0 ** -7 * np.linalg.norm(want), np.linalg.norm(off) / np.linalg.norm(want)
    rms = np.sqrt(np.mean(want ** 2))
    assert np.abs(off).max() <= 0.5 * np.maximum(rms, np.abs(want).max() / 8)
    # the two calls on permuted rows: the same bits
    xp = torch.zeros((max_rows, d), dtype=BF16, device="cuda")
    capmoe.moe_dispatch(desc, x, on(offset), on(padded), xp)
    yp2 = torch.full_like(yp, 7.0)
    ws.fill_(0x5A)
    capmoe.moe_grouped_ffn_fp8(desc, xp, on(offset), experts, yp2, ws)
    assert torch.equal(yp, yp2)


@pytest.mark.parametrize("tokens,d,k,h", [(5000, 136, 4, 128), (14000, 256, 4, 128), (14000, 136, 4, 264), (6000, 1032, 4, 384), (10000, 640, 4, 512)])
def test_ffn_on_high_tiles(tokens, d, k, h):
    counts = [1, 33, 70, 100, 0, 130, 161, 200, 230, 261, 768, 250]
    desc, x, weights, _, _ = layer(tokens, d, len(counts), k, h, mode=capmoe.MODE_NONE)
    offset, token = plan_of(rng(2, tokens), tokens, counts)
    rows = len(token)
    experts = capmoe.Fp8Experts.quantized(*weights)
    ws = torch.empty(capmoe.moe_query_fp8(desc), dtype=torch.uint8, device="cuda")
    ws.fill_(0xA5)
    yp = torch.full((tokens * k, d), 7.0, dtype=BF16, device="cuda")
    padded = np.zeros(tokens * k, np.int32)
    padded[:rows] = token
    capmoe.moe_dispatch_ffn_fp8(desc, x, on(offset), on(padded), experts, yp, ws)
    assert torch.all(yp[rows:] == 7.0)
    values = [ref.weights_value(*ref.quantize_weights(plain(w))) for w in weights]
    want = ref.ffn(plain(x)[token], *values, offset)[:, :d]
    off = plain(yp[:rows]) - want
    assert np.linalg.norm(off) <= 2.0 ** -7 * np.linalg.norm(want), np.linalg.norm(off) / np.linalg.norm(want)
    rms = np.sqrt(np.mean(want ** 2))
    assert np.abs(off).max() <= 0.5 * np.maximum(rms, np.abs(want).max() / 8)


@pytest.mark.parametrize("tokens", [4, 300])
def test_gates_that_are_shut(tokens):
    # gate -2^71 and up 2^71: their product leaves the range of fp32, silu(gate) * up is a zero
    desc, x, weights, _, _ = layer(tokens, 128, 2, 1, 128, mode=capmoe.MODE_NONE)
    x.fill_(2.0 ** 64)
    weights[0].fill_(-1.0), weights[1].fill_(1.0), weights[2].fill_(1.0)
    experts = capmoe.Fp8Experts.quantized(*weights)
    ws = torch.empty(capmoe.moe_query_fp8(desc), dtype=torch.uint8, device="cuda")
    yp = torch.full((tokens, 128), 7.0, dtype=BF16, device="cuda")
    capmoe.moe_grouped_ffn_fp8(desc, x, on(np.array([0, tokens // 2, tokens], np.int32)), experts, yp, ws)
    assert torch.all(yp == 0)


def test_a_token_that_is_not_a_number_stays_by_itself():
    desc, x, weights, _, _ = layer(400, 256, 4, 1, 384, mode=capmoe.MODE_NONE)
    x[7, 3], x[200, 255] = float("nan"), float("inf")
    counts = [300, 12, 0, 88]
    offset = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    token = np.arange(400, dtype=np.int32)
    token[[7, 305]] = 305, 7  # one among the long expert's rows, one among the short one's
    experts = capmoe.Fp8Experts.quantized(*weights)
    ws = torch.empty(capmoe.moe_query_fp8(desc), dtype=torch.uint8, device="cuda")
    yp = torch.zeros((400, 256), dtype=BF16, device="cuda")
    capmoe.moe_dispatch_ffn_fp8(desc, x, on(offset), on(token), experts, yp, ws)
    bad = np.isnan(plain(yp)).any(axis=1)
    assert set(np.flatnonzero(bad)) == {200, 305}


@pytest.mark.parametrize("tokens,counts", [(12, [12, 3, 0, 9]), (300, [300, 64, 0, 211])])
def test_tokens_of_zeros_and_of_extreme_sizes(tokens, counts):
    desc, x, weights, _, _ = layer(tokens, 264, 4, 3, 200, mode=capmoe.MODE_NONE)
    x[1], x[2] = 0, 0
    x[3] *= 2.0 ** -100
    x[4] *= 2.0 ** 60  # the hidden activation reaches 2^120
    x[5, :128] = 0     # a block of zeros beside another
    x[6] = 1e-40       # below the type's normal numbers
    offset, token = plan_of(rng(5, tokens), tokens, counts)
    experts = capmoe.Fp8Experts.quantized(*weights)
    ws = torch.empty(capmoe.moe_query_fp8(desc), dtype=torch.uint8, device="cuda")
    yp = torch.zeros((capmoe.moe_query(desc)[2], 264), dtype=BF16, device="cuda")
    padded = np.zeros(yp.shape[0], np.int32)
    padded[:len(token)] = token
    capmoe.moe_dispatch_ffn_fp8(desc, x, on(offset), on(padded), experts, yp, ws)
    got = plain(yp)[:len(token)]
    values = [ref.weights_value(*ref.quantize_weights(plain(w))) for w in weights]
    want = ref.ffn(plain(x), *values, offset, token)[:, :264]
    assert np.all(got[np.isin(token, (1, 2))] == 0)
    assert np.all(np.abs(got[np.isin(token, (3, 6))]) <= 2.0 ** -90)
    rest = ~np.isin(token, (1, 2, 3, 6))
    err = np.linalg.norm(got[rest] - want[rest], axis=1) / np.linalg.norm(want[rest], axis=1)
    # a row's own error: one value in 2^10 of its 200 on the other side of a border is one at most, of 2^-3 * three times the mean
    # square of 200: 2^-5.2, and the two roundings
    assert np.all(err <= 2.0 ** -5), err.max()


LAYERS = [dict(tokens=64, d=256, e=8, k=2, h=384, device_groups=4, mode=capmoe.MODE_EXPANDED_DROP),
          dict(tokens=512, d=512, e=16, k=4, h=640, mode=capmoe.MODE_TOKEN_DROP, gamma=1.5),
          dict(tokens=1, d=264, e=8, k=2, h=200, mode=capmoe.MODE_NONE),
          dict(tokens=300, d=256, e=4, k=1, h=128, mode=capmoe.MODE_TOKEN_DROP, gamma=0.0),
          dict(tokens=0, d=256, e=4, k=2, h=128, mode=capmoe.MODE_TOKEN_DROP),
          dict(tokens=2048, d=256, e=8, k=2, h=256, mode=capmoe.MODE_TOKEN_DROP, capacity_scope=capmoe.SCOPE_GLOBAL)]


def separate(desc, x, w_router, bias, experts):
    buf = capmoe.LayerBuffers(desc, fp8=True)
    capmoe.moe_route_topk(desc, x, w_router, bias, 0, buf.logits, buf.scores, buf.topk_idx, buf.topk_score, buf.workspace)
    capmoe.moe_capacity_drop(desc, buf.scores, buf.topk_idx, buf.expert_count, buf.seg_count, buf.expert_offset, buf.row_token,
                             buf.row_weight, buf.pair_row, buf.workspace)
    capmoe.moe_dispatch_ffn_fp8(desc, x, buf.expert_offset, buf.row_token, experts, buf.yp, buf.workspace)
    capmoe.moe_combine(desc, buf.yp, buf.row_weight, buf.pair_row, buf.y)
    return buf


@pytest.mark.parametrize("case", range(len(LAYERS)))
def test_layer_is_the_separate_calls(case):
    desc, x, weights, w_router, bias = layer(**LAYERS[case])
    experts = capmoe.Fp8Experts.quantized(*weights)
    want = separate(desc, x, w_router, bias, experts)
    got = capmoe.LayerBuffers(desc, fp8=True)
    got.workspace.fill_(0xA5)
    capmoe.moe_layer_forward_fp8(desc, x, w_router, bias, experts, None, 0, got)
    rows = int(want.expert_offset[-1])
    assert torch.equal(got.expert_offset, want.expert_offset) and torch.equal(got.pair_row, want.pair_row)
    assert torch.equal(got.yp[:rows], want.yp[:rows]) and torch.equal(got.y, want.y)
    # and close to the same layer in bf16: the values are off by 2^-4 at most, 2^-5.6 in the mean square, in three products' operands
    buf = capmoe.LayerBuffers(desc)
    if desc.d_model % 128 == 0 and desc.d_hidden % 128 == 0 and rows:
        y = capmoe.moe_layer_forward(desc, x, w_router, bias, *weights, None, 0, buf)
        assert float((y.float() - got.y.float()).norm() / y.float().norm()) < 0.1


def test_captured_layer_replays():
    desc, x, weights, w_router, bias = layer(**LAYERS[1])
    experts = capmoe.Fp8Experts.quantized(*weights)
    buf = capmoe.LayerBuffers(desc, fp8=True)
    capmoe.moe_layer_forward_fp8(desc, x, w_router, bias, experts, None, 0, buf)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        capmoe.moe_layer_forward_fp8(desc, x, w_router, bias, experts, None, 0, buf)
    for i in range(4):
        x.copy_(on(rng(50 + i).standard_normal(tuple(x.shape)), BF16))
        graph.replay()
        got = buf.y.clone()
        want = capmoe.LayerBuffers(desc, fp8=True)
        capmoe.moe_layer_forward_fp8(desc, x, w_router, bias, experts, None, 0, want)
        torch.cuda.synchronize()
        assert torch.equal(got, want.y), i


def test_two_streams_with_workspaces_of_their_own():
    p, r = Product([300, 20, 0, 64], 512, 384, seed=1), Product([5, 9, 1, 0], 640, 264, seed=2)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    out = []
    inputs = []
    for q in (p, r):
        g = capmoe.make_gemm(q.rows, q.k, q.n, q.e)
        inputs.append((g, [on(a) for a in (q.xq, q.xs, q.offset, q.wq, q.ws)], torch.zeros((q.rows, q.n), dtype=BF16, device="cuda"),
                       torch.empty(capmoe.moe_gemm_query(g), dtype=torch.uint8, device="cuda")))
    torch.cuda.synchronize()
    for _ in range(10):
        for st, (g, (x, xs, off, w, ws), y, work) in zip(streams, inputs):
            capmoe.moe_grouped_gemm_fp8(g, x, xs, None, off, w, ws, y, work, stream=st)
    torch.cuda.synchronize()
    for q, (_, _, y, _) in zip((p, r), inputs):
        q.check(y)


def test_the_same_call_gives_the_same_bits():
    p = Product([700, 40, 0, 300, 1], 2048, 1024, seed=5)
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
    none = torch.empty(0, dtype=torch.uint8, device="cuda")
    capmoe.moe_grouped_gemm_fp8(gemm, x, xs, None, off, w, ws, y, none)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        capmoe.moe_grouped_gemm_fp8(gemm, x, xs, None, off, w, ws, y, none)
    for now in (counts, [most // 4] * 4, counts[::-1], [0, 0, 0, 0], [most, 0, 0, 0]):
        p.offset = np.concatenate([[0], np.cumsum(now)]).astype(np.int32)
        p.rows = int(p.offset[-1])
        off.copy_(torch.from_numpy(p.offset))
        y.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.all(y[p.rows:] == 7.0)
        p.check(y)


def test_calls_on_two_streams_at_once():
    cases = [layer(**LAYERS[i], seed=9) for i in (0, 1, 5)]
    experts = [capmoe.Fp8Experts.quantized(*c[2]) for c in cases]
    want = []
    for (desc, x, _, w_router, bias), e in zip(cases, experts):
        buf = capmoe.LayerBuffers(desc, fp8=True)
        capmoe.moe_layer_forward_fp8(desc, x, w_router, bias, e, None, 0, buf)
        want.append(buf)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [capmoe.LayerBuffers(c[0], fp8=True) for c in cases]
    torch.cuda.synchronize()
    for _ in range(5):
        for (desc, x, _, w_router, bias), e, buf, stream in zip(cases, experts, got, streams):
            capmoe.moe_layer_forward_fp8(desc, x, w_router, bias, e, None, 0, buf, stream=stream)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a.y, b.y) and torch.equal(a.expert_offset, b.expert_offset)


def test_experts_quantized_on_a_stream_have_memory_of_that_stream(monkeypatch):
    # memory of another stream may still be written by work on it when the quantising begins
    side, asked, buffers = torch.cuda.Stream(), [], capmoe.fp8_weight_buffers
    monkeypatch.setattr(capmoe, "fp8_weight_buffers", lambda *a, **k: (asked.append(torch.cuda.current_stream()), buffers(*a, **k))[1])
    _, _, weights, _, _ = layer(8, 136, 3, 2, 264)
    want = capmoe.Fp8Experts.quantized(*weights)
    assert all(s == torch.cuda.default_stream() for s in asked)
    torch.cuda.synchronize()
    asked.clear()
    got = capmoe.Fp8Experts.quantized(*weights, stream=side)
    assert len(asked) == 3 and all(s == side for s in asked)
    assert torch.cuda.current_stream() == torch.cuda.default_stream()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got.tensors, want.tensors))


# Cases by the form that the call takes (test_fp8_forms.py holds the forms against the rules): few rows with 4, 2 or 1 waves to a weight
# row, or column width x row tile.  (rows per expert, columns of x, columns of y, form)
PRODUCT_FORMS = [
    ([128], 520, 264, "128x64"), ([0, 60, 0, 4], 1416, 264, "few/4"), ([0, 120, 0, 8], 264, 392, "few/4"),
    ([1, 0] * 8 + [70, 0, 22], 136, 1032, "few/2"), ([3, 0, 1, 40] + [1] * 16 + [33], 640, 1000, "few/2"),
    ([0, 1] * 20 + [65, 0, 33], 520, 1032, "few/1"), ([100] + [0, 1] * 14, 1032, 2056, "few/1"),
    ([40, 1, 0, 20, 33, 0, 9, 3, 2, 1, 12, 8], 392, 4352, "256x64"), ([100, 1, 0, 130, 33, 200, 9, 3, 64, 128, 12, 88], 520, 4096, "256x128"),
    ([128, 1, 0, 256, 33, 127, 9, 3, 64, 128, 12, 7], 1152, 4096, "256x128"), ([300, 1, 0, 20], 1032, 136, "128x64"), ([700, 1, 400], 264, 2048, "128x128")]


@pytest.mark.parametrize("counts,k,n,form", PRODUCT_FORMS)
def test_product_of_every_form(counts, k, n, form):
    p = Product(counts, k, n)
    p.check(p.run())
    p = Product(counts, k, n, src=31)
    p.check(p.run())


# offsets from elsewhere, within P_max: capacities of 16 rows, 128 in all, and an expert with up to all of them
@pytest.mark.parametrize("counts", [[0, 0, 128, 0, 0, 0, 0, 0], [16, 17, 33, 0, 0, 1, 0, 50], [1, 0, 0, 100, 2, 17, 0, 1], [64, 0, 0, 0, 0, 0, 0, 64]])
def test_ffn_of_few_rows_with_long_experts(counts):
    desc, x, weights, _, _ = layer(128, 264, 8, 1, 392, mode=capmoe.MODE_TOKEN_DROP, capacity_scope=capmoe.SCOPE_GLOBAL, gamma=1.0)
    assert capmoe.moe_query(desc)[0] == 16 and capmoe.moe_query(desc)[2] == 128
    offset = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    rows, token = int(offset[-1]), rng(12).integers(0, 128, 128).astype(np.int32)
    experts = capmoe.Fp8Experts.quantized(*weights)
    ws = torch.empty(capmoe.moe_query_fp8(desc), dtype=torch.uint8, device="cuda")
    yp = torch.full((128, 264), 7.0, dtype=BF16, device="cuda")
    capmoe.moe_dispatch_ffn_fp8(desc, x, on(offset), on(token), experts, yp, ws)
    assert torch.all(yp[rows:] == 7.0)
    values = [ref.weights_value(*ref.quantize_weights(plain(w))) for w in weights]
    want = ref.ffn(plain(x), *values, offset, token[:rows])[:, :264]
    off = plain(yp[:rows]) - want
    assert np.linalg.norm(off) <= 2.0 ** -7 * np.linalg.norm(want)
    assert np.abs(off).max() <= 0.5 * np.maximum(np.sqrt(np.mean(want ** 2)), np.abs(want).max() / 8)


def device_value(q, s):
    """8-bit weights [n, k] of an expert with their scales, in 64 bits on the device."""
    return q.view(torch.float8_e4m3fn).double() * torch.exp2(s[:, : q.shape[1] // 128].double() - 127).repeat_interleave(128, 0).repeat_interleave(128, 1)


def streamed_weights(e, n, k, seed):
    """More 8-bit weights than the memory-side cache holds, normal values of sizes that differ from block to block."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, s = capmoe.fp8_weight_buffers(e, n, k)
    for i in range(e):
        w = torch.randn((n // 128, 128, k // 128, 128), generator=g, device="cuda") * k ** -0.5
        w *= torch.exp2(torch.randint(-2, 3, (n // 128, 1, k // 128, 1), generator=g, device="cuda").float())
        capmoe.moe_quantize_weights(w.view(1, n, k), q[i:i + 1], s[i:i + 1])
    return q, s


# every height in steps of 32 rows, and experts with two tiles (whose weights are kept)
HEIGHTS = [256, 225, 200, 161, 129, 100, 65, 40, 31, 300, 0, 1]
STREAMED_PRODUCTS = [(HEIGHTS, 8320, 4096, "256x256 stream"), (HEIGHTS, 7168, 4096, "256x256 stream"), (HEIGHTS, 8192, 3712, "128x256 stream"),
                     ([5, 0, 1, 16, 9, 0, 2, 30, 0, 1, 0, 0], 8320, 4096, "few/1 stream"), ([1, 0, 1, 0, 0, 2, 0, 0, 1, 0, 0, 0], 8320, 4096, "few/4 stream"),
                     ([1, 0, 1, 0, 0, 2, 0, 0, 1, 0, 0, 0], 7168, 4096, "few/2 stream")]


@pytest.mark.parametrize("counts,k,n,form", STREAMED_PRODUCTS)
def test_streamed_product_of_every_form(counts, k, n, form):
    # odd and even numbers of slabs: walks over k that begin in the middle wrap around at either half of a word of scales
    q, s = streamed_weights(len(counts), n, k, 1)
    rows = sum(counts)
    x = rng(21, rows, k).standard_normal((rows, k)) * np.exp2(rng(22).integers(-2, 3, (rows, k // 128))).repeat(128, 1)
    xq, xs = capmoe.fp8_row_buffers(rows, k)
    capmoe.moe_quantize_rows(on(x, BF16), None, None, xq, xs)
    offset = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    y = torch.full((rows, n), 7.0, dtype=BF16, device="cuda")
    capmoe.moe_grouped_gemm_fp8(capmoe.make_gemm(rows, k, n, len(counts)), xq, xs, None, on(offset), q, s, y, None)
    xv = on(ref.rows_value(xq.cpu().numpy(), xs.cpu().numpy()))
    for i in range(len(counts)):
        a, w = xv[offset[i]:offset[i + 1]], device_value(q[i], s[i])
        want, mag = a @ w.T, a.abs() @ w.abs().T
        off = (y[offset[i]:offset[i + 1]].double() - want).abs()
        assert bool((off <= 2.0 ** -8 * want.abs() + 2.0 ** -12 * mag).all()), i


# tokens, top-k, rows per expert, d, h, forms of the two products
STREAMED_FFNS = [(600, 4, HEIGHTS, 4096, 2304, "128x256 256x256 stream"), (600, 4, HEIGHTS, 4224, 2432, "128x256 128x256 stream"),
                 (600, 4, HEIGHTS, 4352, 2304, "128x256 256x256 stream"),
                 (16, 2, [16, 3, 0, 1, 9, 0, 2, 0, 0, 1, 0, 0], 4224, 2432, "few/1 few/1 stream"), (2, 2, [0, 2, 0, 0, 0, 1, 0, 0, 0, 0, 1, 0], 4096, 2304, "few/2 few/4 stream"),
                 (1, 2, [0, 0, 0, 1, 0, 0, 0, 0, 0, 0, 0, 1], 4224, 2432, "few/4 few/4 stream")]


@pytest.mark.parametrize("tokens,k,counts,d,h,forms", STREAMED_FFNS)
def test_streamed_ffn_of_every_form(tokens, k, counts, d, h, forms):
    e, rows = len(counts), sum(counts)
    desc = capmoe.make_desc(tokens, d, e, k, h, mode=capmoe.MODE_NONE)
    parts = [streamed_weights(e, n, c, seed) for seed, (n, c) in enumerate(((h, d), (h, d), (d, h)))]
    experts = capmoe.Fp8Experts(*[t for p in parts for t in p])
    x = on(rng(31, tokens).standard_normal((tokens, d)), BF16)
    offset, token = plan_of(rng(32, tokens), tokens, counts)
    padded = np.zeros(tokens * k, np.int32)
    padded[:rows] = token
    yp = torch.full((tokens * k, d), 7.0, dtype=BF16, device="cuda")
    ws = torch.empty(capmoe.moe_query_fp8(desc), dtype=torch.uint8, device="cuda")
    ws.fill_(0xA5)
    capmoe.moe_dispatch_ffn_fp8(desc, x, on(offset), on(padded), experts, yp, ws)
    assert torch.all(yp[rows:] == 7.0)
    xv = on(ref.rows_value(*ref.quantize_rows(plain(x)))[token])
    want = np.zeros((rows, d))
    for i in np.flatnonzero(counts):
        gate, up, down = (device_value(q[i], s[i]) for q, s in parts)
        a = xv[offset[i]:offset[i + 1]]
        g, u = plain(a @ gate.T), plain(a @ up.T)
        hidden = ref.rows_value(*ref.quantize_rows(ref.to_bf16(g / (1 + np.exp(-g)) * u)))
        want[offset[i]:offset[i + 1]] = plain(on(hidden) @ down.T)
    off = plain(yp[:rows]) - want
    assert np.linalg.norm(off) <= 2.0 ** -7 * np.linalg.norm(want), np.linalg.norm(off) / np.linalg.norm(want)
    # a row's own error: eight of its 2304 or more hidden values, or one of ten times their mean square, on the other side of a border
    # are 2^-3 * 10 / 48 = 2^-5.3, and the two roundings
    err = np.linalg.norm(off, axis=1) / np.linalg.norm(want, axis=1)
    assert np.all(err <= 2.0 ** -5), (np.argmax(err), err.max())


@pytest.mark.parametrize("counts", [[5, 12], [300, 12]])
def test_a_scale_byte_of_255_is_not_a_number(counts):
    # and those behind the last block stand for nothing
    p = Product(counts, 520, 264)
    p.xs[:, 5:], p.ws[:, :, 5:] = 255, 255
    p.check(p.run())
    p.xs[3, 1], p.ws[1, 1, 4] = 255, 255
    got = plain(p.run())
    nan = np.zeros(got.shape, bool)
    nan[3], nan[counts[0]:, 128:256] = True, True
    assert np.array_equal(np.isnan(got), nan)


@pytest.mark.parametrize("counts", [[5, 12], [300, 12]])
def test_the_largest_and_smallest_scale_bytes(counts):
    # 2^127 and 2^-127 meet as 1
    p = Product(counts, 520, 264)
    p.xs[:, :5], p.ws[:, :, :5] = [254, 0, 254, 0, 254], [0, 254, 0, 254, 0]
    p.check(p.run())


@pytest.mark.parametrize("tokens,counts", [(12, [12, 3, 0, 9]), (300, [300, 64, 0, 211])])
def test_hidden_widths_that_are_no_multiple_of_8(tokens, counts):
    # the down weights of such a width are quantised with columns of zeros behind it
    desc, x, (gate, up, down), _, _ = layer(tokens, 264, 4, 3, 203, mode=capmoe.MODE_NONE)
    with pytest.raises(capmoe.CapMoeError):
        capmoe.Fp8Experts.quantized(gate, up, down)
    experts = capmoe.Fp8Experts.quantized(gate, up, torch.nn.functional.pad(down, (0, 5)))
    offset, token = plan_of(rng(5, tokens), tokens, counts)
    ws = torch.empty(capmoe.moe_query_fp8(desc), dtype=torch.uint8, device="cuda")
    yp = torch.zeros((capmoe.moe_query(desc)[2], 264), dtype=BF16, device="cuda")
    padded = np.zeros(yp.shape[0], np.int32)
    padded[:len(token)] = token
    capmoe.moe_dispatch_ffn_fp8(desc, x, on(offset), on(padded), experts, yp, ws)
    values = [ref.weights_value(*ref.quantize_weights(plain(w))) for w in (gate, up, down)]
    want = ref.ffn(plain(x), *values, offset, token)[:, :264]
    off = plain(yp)[:len(token)] - want
    assert np.linalg.norm(off) <= 2.0 ** -7 * np.linalg.norm(want)
