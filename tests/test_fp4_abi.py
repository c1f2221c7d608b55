"""The norm and the 4-bit experts without a GPU: sizes, refusals before anything is launched, and the reference's own format."""
import ctypes

import numpy as np
import pytest
import torch

import fp4_reference as ref
from paper_2503_05066_amd import capmoe

pytestmark = pytest.mark.usefixtures("built_library")
OK, INVALID, UNSUPPORTED, SMALL = 0, 1, 2, 3
P = 1 << 20  # an aligned address that nothing reads


class Stream:
    """A stream of a device that none of the host tensors lies on."""

    cuda_stream, device_index = None, 0


def test_reference_codes():
    # every border between two values goes to the even code, and to either side of it next to it
    for lo in range(7):
        mid = (ref.MAGNITUDES[lo] + ref.MAGNITUDES[lo + 1]) / 2
        even = lo if lo % 2 == 0 else lo + 1
        v = np.array([mid, np.nextafter(mid, 0), np.nextafter(mid, 9), -mid, ref.MAGNITUDES[lo], -ref.MAGNITUDES[lo]])
        assert list(ref.encode(v)) == [even, lo, lo + 1, 8 + even, lo, 8 + lo]
    assert list(ref.encode(np.array([6.0, -6.0]))) == [7, 15]


@pytest.mark.parametrize("amax,byte", [(6.0, 127), (6.0001, 128), (3.0, 126), (3.00001, 127), (0.0, 0), (1e-45, 0), (3.4e38, 253),
                                       (6.0 * 2.0 ** -127, 0), (6.1 * 2.0 ** -127, 1), (np.inf, 255), (np.nan, 255)])
def test_reference_scales(amax, byte):
    assert ref.block_byte(np.array([amax]))[0] == byte


def test_reference_layout():
    x = np.zeros((1, 1024))
    x[0, 0], x[0, 1], x[0, 32], x[0, 128], x[0, 32 * 15], x[0, 32 * 17] = 6, -0.5, 12, 24, 48, 96
    q, s = ref.quantize(x)
    assert q.shape == (1, 512) and s.shape == (1, 32)
    assert q[0, 0] == 0x97 and q[0, 16] == 7 and q[0, 64] == 7
    assert s[0, 0] == 127 and s[0, 4] == 128 and s[0, 1] == 129 and s[0, 15] == 130 and s[0, 16 + 4] == 131 and np.count_nonzero(s) == 5
    assert np.array_equal(ref.value(q, s), x)


@pytest.mark.parametrize("cols,pitch,scale", [(1, 128, 16), (256, 128, 16), (257, 256, 16), (512, 256, 16), (520, 384, 32),
                                              (14336, 7168, 448), (1 << 21, 1 << 20, 1 << 16)])
def test_sizes(cols, pitch, scale):
    assert capmoe.moe_fp4_query(cols) == (pitch, scale)


def test_size_refusals():
    lib = capmoe.load()
    assert lib.moe_fp4_query(0, None, None) == INVALID
    assert lib.moe_fp4_query((1 << 21) + 1, None, None) == UNSUPPORTED


def test_quantize_rows_refusals():
    f = capmoe.load().moe_quantize_rows_fp4
    good = dict(dtype=1, x=P, n=4, cols=64, token=None, count=None, q=P, s=P)

    def call(**change):
        a = {**good, **change}
        return f(a["dtype"], a["x"], a["n"], a["cols"], a["token"], a["count"], a["q"], a["s"], None)

    assert call(dtype=2) == INVALID and call(dtype=-1) == INVALID
    assert call(n=-1) == INVALID and call(cols=0) == INVALID and call(cols=-8) == INVALID
    assert call(cols=12) == UNSUPPORTED and call(dtype=0, cols=6) == UNSUPPORTED
    assert call(cols=(1 << 21) + 8) == UNSUPPORTED
    assert call(n=1 << 31) == UNSUPPORTED and call(n=1 << 30, cols=1024) == UNSUPPORTED and call(n=1 << 62, cols=1 << 20) == UNSUPPORTED
    for a in ("x", "q", "s"):
        assert call(**{a: None}) == INVALID and call(**{a: P + 8}) == INVALID
    assert call(n=0, x=None, q=None, s=None) == OK


def test_quantize_weights_refusals():
    f = capmoe.load().moe_quantize_weights_fp4
    good = dict(dtype=1, w=P, e=2, n=16, k=64, q=P, s=P)

    def call(**change):
        a = {**good, **change}
        return f(a["dtype"], a["w"], a["e"], a["n"], a["k"], a["q"], a["s"], None)

    assert call(dtype=7) == INVALID and call(e=0) == INVALID and call(n=0) == INVALID and call(k=0) == INVALID
    assert call(k=12) == UNSUPPORTED and call(dtype=0, k=3) == UNSUPPORTED and call(n=(1 << 21) + 1) == UNSUPPORTED
    assert call(e=1 << 10, n=1 << 21, k=1 << 21) == UNSUPPORTED and call(e=(1 << 31) - 1, n=1 << 21) == UNSUPPORTED
    for a in ("w", "q", "s"):
        assert call(**{a: None}) == INVALID and call(**{a: P + 4}) == INVALID


def test_dequantize_refusals():
    f = capmoe.load().moe_dequantize_rows
    good = dict(bits=4, dtype=1, q=P, s=P, n=4, cols=64, y=P)

    def call(**change):
        a = {**good, **change}
        return f(a["bits"], a["dtype"], a["q"], a["s"], a["n"], a["cols"], a["y"], None)

    assert call(bits=0) == INVALID and call(bits=16) == INVALID and call(dtype=3) == INVALID and call(n=-1) == INVALID and call(cols=0) == INVALID
    assert call(cols=12) == UNSUPPORTED and call(n=1 << 31) == UNSUPPORTED and call(n=1 << 30, cols=1024) == UNSUPPORTED
    for a in ("q", "s", "y"):
        assert call(**{a: None}) == INVALID and call(**{a: P + 8 if a != "s" else P + 4}) == INVALID
    assert call(bits=8, s=P + 2) == INVALID
    assert call(n=0, q=None, s=None, y=None) == OK


def test_norm_refusals():
    f = capmoe.load().moe_norm_rows
    good = dict(n=4, cols=64, dtype=1, bits=0, eps=1e-6, x=P, r=None, w=None, count=None, sum=None, y=P, q=None, s=None)

    def call(**change):
        a = {**good, **change}
        norm = capmoe.MoeNorm(a["n"], a["cols"], a["dtype"], a["bits"], a["eps"])
        return f(ctypes.byref(norm), a["x"], a["r"], a["w"], a["count"], a["sum"], a["y"], a["q"], a["s"], None)

    assert f(None, P, None, None, None, None, P, None, None, None) == INVALID
    assert call(n=-1) == INVALID and call(cols=0) == INVALID and call(dtype=2) == INVALID and call(bits=2) == INVALID
    assert call(cols=12) == UNSUPPORTED and call(dtype=0, cols=6) == UNSUPPORTED and call(cols=(1 << 21) + 8) == UNSUPPORTED
    assert call(n=1 << 30, cols=1024) == UNSUPPORTED
    for eps in (0.0, -1.0, 1e-45, float("inf"), float("nan")):
        assert call(eps=eps) == INVALID
    assert call(x=None) == INVALID and call(y=None) == INVALID
    for bits in (4, 8):
        assert call(bits=bits, q=P) == INVALID and call(bits=bits, s=P) == INVALID and call(bits=bits, y=None) == INVALID
        assert call(bits=bits, q=P + 8, s=P) == INVALID and call(bits=bits, q=P, s=P + 2) == INVALID
    assert call(bits=4, q=P, s=P + 4) == INVALID
    for a in ("x", "r", "w", "sum", "y"):
        assert call(**{a: P + 8}) == INVALID
    assert call(sum=P) == INVALID  # both outputs in one place
    assert call(n=0, x=None, y=None) == OK


def test_gemm_refusals():
    lib = capmoe.load()
    good = dict(rows=8, src=0, e=4, k=256, n=64, x=P, xs=P, token=None, off=P, w=P, ws=P, y=P)

    def call(**change):
        a = {**good, **change}
        g = capmoe.MoeGemm(a["rows"], a["src"], a["e"], a["k"], a["n"])
        return lib.moe_grouped_gemm_fp4(ctypes.byref(g), a["x"], a["xs"], a["token"], a["off"], a["w"], a["ws"], a["y"], None)

    for bad in (dict(rows=-1), dict(src=-1), dict(e=0), dict(k=0), dict(n=0), dict(token=P, src=0)):
        assert call(**bad) == INVALID
    for bad in (dict(e=257), dict(n=12), dict(n=(1 << 21) + 8), dict(k=(1 << 21) + 1), dict(token=P, src=1 << 20, k=1 << 13)):
        assert call(**bad) == UNSUPPORTED
    for a in ("x", "xs", "off", "w", "ws", "y"):
        assert call(**{a: None}) == INVALID
    for a in ("x", "w", "y", "xs", "ws"):
        assert call(**{a: P + 8}) == INVALID
    assert call(rows=0) == OK
    assert call(rows=0, **{a: None for a in ("x", "xs", "off", "w", "ws", "y")}) == OK  # tensors of no rows have no address
    assert lib.moe_grouped_gemm_fp4(None, P, P, None, P, P, P, P, None) == INVALID


def _desc(**more):
    a = dict(n_tokens=16, d_model=256, n_experts=8, top_k=2, d_hidden=200, dtype=capmoe.DTYPE_BF16)
    a.update(more)
    return capmoe.make_desc(**a)


def _experts(**change):
    e = capmoe.MoeFp4Experts(P, P, P, P, P, P)
    for k, v in change.items():
        setattr(e, k, v)
    return e


def test_ffn_refusals():
    lib = capmoe.load()
    size = ctypes.c_size_t()

    def query(desc):
        return lib.moe_query_fp4(ctypes.byref(desc), ctypes.byref(size))

    assert query(_desc()) == OK and size.value >= capmoe.moe_query(_desc())[3]
    assert query(_desc(dtype=capmoe.DTYPE_F32)) == UNSUPPORTED and query(_desc(d_model=(1 << 21) + 8)) == UNSUPPORTED
    assert query(_desc(d_model=100)) == UNSUPPORTED and query(_desc(n_tokens=-1)) == INVALID
    assert query(_desc(n_tokens=1 << 25, d_model=1 << 21)) == UNSUPPORTED
    assert lib.moe_query_fp4(None, None) == INVALID
    need = capmoe.moe_query_fp4(_desc())
    good = dict(x=P, xs=None, off=P, token=P, experts=_experts(), yp=P, work=P, size=need)

    for gathered in (False, True):
        def call(desc=_desc(), **change):
            a = {**good, **change}
            e = ctypes.byref(a["experts"]) if a["experts"] is not None else None
            if gathered:
                return lib.moe_dispatch_ffn_fp4(ctypes.byref(desc), a["x"], a["xs"], a["off"], a["token"], e, a["yp"], a["work"], a["size"], None)
            return lib.moe_grouped_ffn_fp4(ctypes.byref(desc), a["x"], a["xs"], a["off"], e, a["yp"], a["work"], a["size"], None)

        for a in ("x", "off", "yp", "work", "experts") + (("token",) if gathered else ()):
            assert call(**{a: None}) == INVALID
        for a in ("x", "xs", "yp"):
            assert call(**{a: P + 8}) == INVALID
        assert call(work=P + 128) == INVALID and call(size=0) == SMALL
        for f, _ in capmoe.MoeFp4Experts._fields_:
            assert call(experts=_experts(**{f: None})) == INVALID and call(experts=_experts(**{f: P + 4})) == INVALID
        assert call(desc=_desc(dtype=capmoe.DTYPE_F32)) == UNSUPPORTED
        assert call(desc=_desc(gamma=0.0), x=None, token=None, yp=None) == OK  # no row can survive
    big = _desc(n_tokens=1 << 18, d_model=1 << 13)
    assert lib.moe_dispatch_ffn_fp4(ctypes.byref(big), P, None, P, P, ctypes.byref(_experts()), P, P, 1 << 50, None) == UNSUPPORTED
    # narrow rows of many tokens: 2^25 of 128 bytes pass the window that they are gathered through
    narrow = _desc(n_tokens=1 << 25, d_model=8, n_experts=8, top_k=1, d_hidden=8)
    for scale in (None, P):
        assert lib.moe_dispatch_ffn_fp4(ctypes.byref(narrow), P, scale, P, P, ctypes.byref(_experts()), P, P, 1 << 50, None) == UNSUPPORTED


def test_layer_refusals():
    lib = capmoe.load()
    names = ["x", "xq", "xs", "wr", "bias", "experts", "cls", "seed", "logits", "scores", "idx", "topk", "count", "seg", "off", "token", "weight",
             "pair", "yp", "y", "work", "size"]
    good = {n: P for n in names}
    good.update(xq=None, xs=None, experts=_experts(), seed=0, size=capmoe.moe_query_fp4(_desc()), bias=None, cls=None)

    def call(desc=_desc(), **change):
        a = {**good, **change}
        a["experts"] = ctypes.byref(a["experts"]) if a["experts"] is not None else None
        return lib.moe_layer_forward_fp4(ctypes.byref(desc), *[a[n] for n in names], None)

    for a in ("x", "wr", "experts", "logits", "scores", "idx", "topk", "count", "seg", "off", "token", "weight", "pair", "yp", "y", "work"):
        assert call(**{a: None}) == INVALID, a
    assert call(xq=P) == INVALID and call(xs=P) == INVALID  # both or neither
    for a in ("x", "wr", "yp", "y", "scores", "idx", "pair"):
        assert call(**{a: P + 8}) == INVALID, a
    assert call(xq=P + 8, xs=P) == INVALID and call(xq=P, xs=P + 4) == INVALID
    assert call(size=64) == SMALL and call(desc=_desc(dtype=capmoe.DTYPE_F32)) == UNSUPPORTED
    assert call(desc=_desc(n_tokens=1 << 25, d_model=8, n_experts=8, top_k=1, d_hidden=8), size=1 << 50) == UNSUPPORTED


def test_binding_refuses_tensors_that_do_not_fit():
    t = torch.uint8
    x = torch.zeros((4, 264), dtype=torch.bfloat16)
    q, s = torch.zeros((4, 256), dtype=t), torch.zeros((4, 16), dtype=t)
    for args in ((x.half(), q, s), (x.t(), q, s), (x, q[:, :128], s), (x, q, s[:, :8]), (x[:3], q, s), (x[None], q, s)):
        with pytest.raises(ValueError):
            capmoe.moe_quantize_rows_fp4(args[0], None, None, args[1], args[2])
    with pytest.raises(ValueError):
        capmoe.moe_quantize_rows_fp4(x, torch.zeros(3, dtype=torch.int32), None, q, s)
    with pytest.raises(ValueError):
        capmoe.moe_quantize_rows_fp4(x, None, torch.zeros(1), q, s)
    with pytest.raises(ValueError):
        capmoe.moe_quantize_weights_fp4(torch.zeros((2, 4, 264)), q, s)
    for y in (x.half(), x[:, :256], x[:3]):
        with pytest.raises(ValueError):
            capmoe.moe_dequantize_rows(8, q, s, y)
    norm = capmoe.make_norm(4, 264, bits=4)
    w = torch.zeros(264, dtype=torch.bfloat16)
    good = dict(x=x, residual=x, weight=w, row_count=None, sum=x, y=x.clone(), q=q, scale=s)
    for change in (dict(x=x.float()), dict(residual=x[:3]), dict(weight=w[:8]), dict(weight=w.float()), dict(sum=x.t()), dict(y=x[:, :8]),
                   dict(q=q[:, :8]), dict(scale=s[:2]), dict(row_count=torch.zeros(1))):
        with pytest.raises(ValueError):
            capmoe.moe_norm_rows(norm, **{**good, **change})
    with pytest.raises(ValueError):
        capmoe.moe_norm_rows(norm, **good, stream=Stream)  # host memory


def test_binding_refuses_products_that_do_not_fit():
    t = torch.uint8
    gemm = capmoe.make_gemm(5, 264, 136, 2)
    good = dict(x=torch.zeros((5, 256), dtype=t), x_scale=torch.zeros((5, 16), dtype=t), row_token=None,
                expert_offset=torch.zeros(3, dtype=torch.int32), w=torch.zeros((2, 256, 256), dtype=t), w_scale=torch.zeros((2, 256, 16), dtype=t),
                y=torch.zeros((5, 136), dtype=torch.bfloat16))
    for change in (dict(x=good["x"][:, :128]), dict(x_scale=good["x_scale"][:, :8]), dict(expert_offset=torch.zeros(2, dtype=torch.int32)),
                   dict(w=good["w"][:1]), dict(w_scale=good["w_scale"][:, :128]), dict(y=good["y"][:4]), dict(y=good["y"].float()),
                   dict(row_token=torch.zeros(4, dtype=torch.int32)), dict(w=None)):
        with pytest.raises(ValueError):
            capmoe.moe_grouped_gemm_fp4(gemm, **{**good, **change})
    with pytest.raises(ValueError):
        capmoe.moe_grouped_gemm_fp4(gemm, **good, stream=Stream)  # host memory


def test_experts_that_do_not_fit_each_other_or_their_layer():
    t = torch.uint8

    def parts(e=2, h=256, d=264):
        up = lambda n: -(-n // 128) * 128
        out = []
        for n, k in ((h, d), (h, d), (d, h)):
            pitch, scale = capmoe.moe_fp4_query(k)
            out += [torch.zeros((e, up(n), pitch), dtype=t), torch.zeros((e, up(n), scale), dtype=t)]
        return out

    experts = capmoe.Fp4Experts(*parts())
    assert experts.sizes == (2, 256, 384)
    experts.of(_desc(n_experts=2, d_hidden=200, d_model=264, top_k=1))
    for bad in (dict(n_experts=4), dict(d_hidden=264), dict(d_model=512)):
        with pytest.raises(ValueError):
            experts.of(_desc(**{**dict(n_experts=2, d_hidden=200, d_model=264, top_k=1), **bad}))
    for i in range(6):
        for bad in (parts()[i][:1], parts()[i][:, :128], parts()[i][..., :8], parts()[i].float()):
            p = parts()
            p[i] = bad
            with pytest.raises(ValueError):
                capmoe.Fp4Experts(*p)
