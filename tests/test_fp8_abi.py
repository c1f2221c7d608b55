"""The 8-bit experts without a GPU: sizes, refusals before anything is launched, and the reference's own format."""
import ctypes

import numpy as np
import pytest
import torch

import fp8_reference as ref
from paper_2503_05066_amd import capmoe

pytestmark = pytest.mark.usefixtures("built_library")
OK, INVALID, UNSUPPORTED, SMALL = 0, 1, 2, 3
P = 1 << 20  # an aligned address that nothing reads


def test_reference_values_are_those_of_the_type():
    bytes_ = torch.arange(256, dtype=torch.uint8)
    want = bytes_.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ref.E4M3, want, equal_nan=True)
    v = np.concatenate([np.random.default_rng(1).uniform(-448, 448, 20000), ref.E4M3[:126], (ref.E4M3[:126] + ref.E4M3[1:127]) / 2])
    got = ref.encode(np.float64(np.float32(v)))
    want = torch.from_numpy(np.float32(v)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(got, want)


@pytest.mark.parametrize("amax,byte", [(448.0, 127), (448.0001, 128), (1.75, 119), (1.75001, 120), (0.0, 0), (1e-45, 0),
                                       (3.4e38, 247), (448.0 * 2.0 ** -127, 0), (449.0 * 2.0 ** -127, 1)])
def test_reference_scales(amax, byte):
    assert ref.block_byte(np.array([amax]))[0] == byte


@pytest.mark.parametrize("cols,pitch,scale", [(1, 128, 4), (128, 128, 4), (129, 256, 4), (512, 512, 4), (520, 640, 8),
                                              (14336, 14336, 112), (1 << 21, 1 << 21, 1 << 14)])
def test_sizes(cols, pitch, scale):
    assert capmoe.moe_fp8_query(cols) == (pitch, scale)


def test_size_refusals():
    lib = capmoe.load()
    assert lib.moe_fp8_query(0, None, None) == INVALID
    assert lib.moe_fp8_query((1 << 21) + 1, None, None) == UNSUPPORTED


def test_quantize_rows_refusals():
    f = capmoe.load().moe_quantize_rows
    good = dict(dtype=1, x=P, n=4, cols=64, token=None, count=None, q=P, s=P)

    def call(**change):
        a = {**good, **change}
        return f(a["dtype"], a["x"], a["n"], a["cols"], a["token"], a["count"], a["q"], a["s"], None)

    assert call(dtype=2) == INVALID and call(dtype=-1) == INVALID
    assert call(n=-1) == INVALID and call(cols=0) == INVALID and call(cols=-8) == INVALID
    assert call(cols=12) == UNSUPPORTED and call(dtype=0, cols=6) == UNSUPPORTED
    assert call(cols=(1 << 21) + 8) == UNSUPPORTED
    assert call(n=1 << 31) == UNSUPPORTED and call(n=1 << 30, cols=256) == UNSUPPORTED and call(n=1 << 62, cols=1 << 20) == UNSUPPORTED
    for a in ("x", "q", "s"):
        assert call(**{a: None}) == INVALID
    assert call(x=P + 8) == INVALID and call(q=P + 8) == INVALID and call(s=P + 2) == INVALID
    assert call(n=0, x=None, q=None, s=None) == OK


def test_quantize_weights_refusals():
    f = capmoe.load().moe_quantize_weights
    good = dict(dtype=1, w=P, e=2, n=16, k=64, q=P, s=P)

    def call(**change):
        a = {**good, **change}
        return f(a["dtype"], a["w"], a["e"], a["n"], a["k"], a["q"], a["s"], None)

    assert call(dtype=7) == INVALID and call(e=0) == INVALID and call(n=0) == INVALID and call(k=0) == INVALID
    assert call(k=12) == UNSUPPORTED and call(dtype=0, k=3) == UNSUPPORTED and call(n=(1 << 21) + 1) == UNSUPPORTED
    assert call(e=1 << 10, n=1 << 21, k=1 << 21) == UNSUPPORTED and call(e=1 << 12, n=1 << 13, k=1 << 13) == UNSUPPORTED
    for a in ("w", "q", "s"):
        assert call(**{a: None}) == INVALID
    assert call(w=P + 4) == INVALID and call(q=P + 1) == INVALID and call(s=P + 1) == INVALID


def test_gemm_refusals():
    lib = capmoe.load()
    good = dict(rows=8, src=0, e=4, k=256, n=64, x=P, xs=P, token=None, off=P, w=P, ws=P, y=P, work=P, size=1 << 30)

    def call(**change):
        a = {**good, **change}
        g = capmoe.MoeGemm(a["rows"], a["src"], a["e"], a["k"], a["n"])
        return lib.moe_grouped_gemm_fp8(ctypes.byref(g), a["x"], a["xs"], a["token"], a["off"], a["w"], a["ws"], a["y"],
                                        a["work"], a["size"], None)

    for bad in (dict(rows=-1), dict(src=-1), dict(e=0), dict(k=0), dict(n=0), dict(token=P, src=0)):
        assert call(**bad) == INVALID
    for bad in (dict(e=257), dict(n=12), dict(n=(1 << 21) + 8), dict(k=(1 << 21) + 1), dict(token=P, src=1 << 20, k=1 << 13)):
        assert call(**bad) == UNSUPPORTED
    for a in ("x", "xs", "off", "w", "ws", "y"):
        assert call(**{a: None}) == INVALID
    for a in ("x", "w", "y"):
        assert call(**{a: P + 8}) == INVALID
    assert call(xs=P + 2) == INVALID and call(ws=P + 1) == INVALID
    assert call(rows=0) == OK  # nothing to do, nothing launched
    assert call(rows=0, **{a: None for a in ("x", "xs", "off", "w", "ws", "y")}) == OK  # tensors of no rows have no address
    assert capmoe.moe_gemm_query(capmoe.make_gemm(8, 256, 64, 4)) == 0 and call(rows=0, work=None, size=0) == OK
    assert lib.moe_grouped_gemm_fp8(None, P, P, None, P, P, P, P, P, 1 << 30, None) == INVALID
    assert lib.moe_gemm_query(None, None) == INVALID


def _desc(**more):
    a = dict(n_tokens=16, d_model=256, n_experts=8, top_k=2, d_hidden=200, dtype=capmoe.DTYPE_BF16)
    a.update(more)
    return capmoe.make_desc(**a)


def _experts(**change):
    e = capmoe.MoeFp8Experts(P, P, P, P, P, P)
    for k, v in change.items():
        setattr(e, k, v)
    return e


def test_ffn_refusals():
    lib = capmoe.load()

    def grouped(desc=None, x=P, off=P, experts=None, yp=P, work=P, size=1 << 40):
        return lib.moe_grouped_ffn_fp8(ctypes.byref(desc or _desc()), x, off, ctypes.byref(experts or _experts()), yp, work, size, None)

    def fused(desc=None, x=P, off=P, token=P, experts=None, yp=P, work=P, size=1 << 40):
        return lib.moe_dispatch_ffn_fp8(ctypes.byref(desc or _desc()), x, off, token, ctypes.byref(experts or _experts()), yp, work, size, None)

    for f in (grouped, fused):
        assert f(desc=_desc(dtype=capmoe.DTYPE_F32)) == UNSUPPORTED
        assert f(desc=_desc(d_hidden=(1 << 21) + 1)) == UNSUPPORTED
        assert f(desc=_desc(d_model=252)) == UNSUPPORTED  # no 16-byte pieces
        assert f(desc=_desc(top_k=9)) == INVALID
        for a in ("x", "off", "yp", "work"):
            assert f(**{a: None}) == INVALID
        assert f(x=P + 8) == INVALID and f(yp=P + 8) == INVALID and f(work=P + 8) == INVALID
        for name, _ in capmoe.MoeFp8Experts._fields_:
            assert f(experts=_experts(**{name: None})) == INVALID
            assert f(experts=_experts(**{name: P + 2})) == INVALID
        assert f(size=1024) == SMALL
        assert f(desc=_desc(gamma=0.0)) == OK  # no row can survive
    assert fused(token=None) == INVALID
    assert fused(desc=_desc(n_tokens=1 << 17, d_model=1 << 14)) == UNSUPPORTED
    # d fills 16 bytes a row of x, but 128 of its 8-bit form
    narrow = dict(n_tokens=1 << 25, d_model=8, n_experts=4, top_k=1, gamma=0.001)
    assert fused(desc=_desc(**narrow)) == UNSUPPORTED
    # more blocks of 128 than the quantising counts
    assert grouped(desc=_desc(n_tokens=1 << 20, d_model=1 << 15, top_k=8, mode=capmoe.MODE_NONE)) == UNSUPPORTED
    none = _desc(gamma=0.0)
    assert grouped(desc=none, x=None, yp=None) == OK and fused(desc=none, x=None, token=None, yp=None) == OK
    assert lib.moe_grouped_ffn_fp8(ctypes.byref(_desc()), P, P, None, P, P, 1 << 40, None) == INVALID


def test_layer_refusals():
    lib = capmoe.load()
    names = ("logits", "scores", "topk_idx", "topk_score", "expert_count", "seg_count", "expert_offset", "row_token",
             "row_weight", "pair_row", "yp", "y", "workspace")

    def call(desc=None, x=P, w_router=P, experts=None, size=1 << 40, **change):
        a = {**{n: P for n in names}, **change}
        return lib.moe_layer_forward_fp8(ctypes.byref(desc or _desc()), x, w_router, None, ctypes.byref(experts or _experts()), None, 0,
                                         *[a[n] for n in names], size, None)

    assert call(desc=_desc(dtype=capmoe.DTYPE_F32)) == UNSUPPORTED
    assert call(x=None) == INVALID and call(w_router=None) == INVALID and call(x=P + 8) == INVALID
    for n in names:
        assert call(**{n: None}) == INVALID, n
    for n in ("scores", "topk_idx", "pair_row", "yp", "y", "workspace"):
        assert call(**{n: P + 4}) == INVALID, n
    assert call(experts=_experts(down=None)) == INVALID
    assert call(desc=_desc(n_tokens=1 << 25, d_model=8, n_experts=4, top_k=1, gamma=0.001)) == UNSUPPORTED
    need = capmoe.moe_query_fp8(_desc())
    assert call(size=need - 1) == SMALL and need >= capmoe.moe_query(_desc())[3]


def test_query_refuses_other_types():
    with pytest.raises(capmoe.CapMoeError) as e:
        capmoe.moe_query_fp8(_desc(dtype=capmoe.DTYPE_F32))
    assert e.value.status == UNSUPPORTED


def test_binding_refuses_tensors_that_do_not_fit():
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    q, s = capmoe.fp8_row_buffers(4, 64, device="cpu")
    for bad in (lambda: capmoe.moe_quantize_rows(x, None, None, q[:, :64], s), lambda: capmoe.moe_quantize_rows(x, None, None, q, s[:2]),
                lambda: capmoe.moe_quantize_rows(x, None, None, torch.cat([q, q]), torch.cat([s, s])),
                lambda: capmoe.moe_quantize_rows(x.half(), None, None, q, s), lambda: capmoe.moe_quantize_rows(x.T, None, None, q, s),
                lambda: capmoe.moe_quantize_rows(x, torch.zeros(3, dtype=torch.int32), None, q, s),
                lambda: capmoe.moe_quantize_rows(x, torch.zeros(4, dtype=torch.int64), None, q, s)):
        with pytest.raises(ValueError):
            bad()
    w = torch.zeros((2, 8, 64), dtype=torch.bfloat16)
    q, s = capmoe.fp8_weight_buffers(2, 8, 64, device="cpu")
    for bad in (lambda: capmoe.moe_quantize_weights(w, q[:, :8], s), lambda: capmoe.moe_quantize_weights(w, q, s[:1]),
                lambda: capmoe.moe_quantize_weights(w.transpose(0, 1), q, s), lambda: capmoe.moe_quantize_weights(w[0], q, s)):
        with pytest.raises(ValueError):
            bad()


def test_experts_that_do_not_fit_are_refused():
    def made(e=2, h=200, d=72, **change):
        sizes = {"gate": (e, h, d), "up": (e, h, d), "down": (e, d, h), **change}
        parts = [t for n in ("gate", "up", "down") for t in capmoe.fp8_weight_buffers(*sizes[n], device="cpu")]
        return capmoe.Fp8Experts(*parts)

    good = made()
    assert good.sizes == (2, 256, 128)
    for bad in (dict(up=(2, 300, 72)), dict(up=(3, 200, 72)), dict(down=(2, 200, 72)), dict(down=(2, 72, 300)), dict(down=(1, 72, 200))):
        with pytest.raises(ValueError):
            made(**bad)
    t = list(good.tensors)
    for i, bad in ((0, t[0][:, :, :64]), (1, t[1][:, :1]), (4, t[4].transpose(1, 2)), (5, t[5].int()), (2, t[2].short())):
        with pytest.raises(ValueError):
            capmoe.Fp8Experts(*t[:i], bad, *t[i + 1:])
    x = torch.zeros((16, 72), dtype=torch.bfloat16)
    for desc in (_desc(d_model=72, n_experts=3), _desc(d_model=136, n_experts=2), _desc(d_model=72, n_experts=2, d_hidden=257)):
        for call in (lambda: capmoe.moe_grouped_ffn_fp8(desc, x, None, good, x, x), lambda: capmoe.moe_dispatch_ffn_fp8(desc, x, None, None, good, x, x)):
            with pytest.raises(ValueError):
                call()


class _NoStream:
    """A stream for calls that must be over before anything is enqueued on it."""

    cuda_stream = None
    device_index = -1  # that of tensors in host memory


def test_binding_passes_no_workspace_to_a_product():
    gemm = capmoe.make_gemm(0, 256, 64, 2)
    xq, xs = capmoe.fp8_row_buffers(0, 256, device="cpu")
    wq, ws = capmoe.fp8_weight_buffers(2, 64, 256, device="cpu")
    y, offset = torch.zeros((0, 64), dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    capmoe.moe_grouped_gemm_fp8(gemm, xq, xs, None, offset, wq, ws, y, None, stream=_NoStream)


def _product(rows=6, e=2, k=264, n=200, src=0):
    """Arguments of a product that belong together, on the host."""
    a = dict(gemm=capmoe.make_gemm(rows, k, n, e, src_rows=src), row_token=None, workspace=None)
    a["x"], a["x_scale"] = capmoe.fp8_row_buffers(src or rows, k, device="cpu")
    a["w"], a["w_scale"] = capmoe.fp8_weight_buffers(e, n, k, device="cpu")
    a["y"], a["expert_offset"] = torch.zeros((rows, n), dtype=torch.bfloat16), torch.zeros(e + 1, dtype=torch.int32)
    if src:
        a["row_token"] = torch.zeros(rows, dtype=torch.int32)
    return a


def test_binding_refuses_tensors_that_do_not_fit_a_product():
    def refused(**change):
        with pytest.raises(ValueError):
            capmoe.moe_grouped_gemm_fp8(**{**a, **change}, stream=_NoStream)

    a = _product(src=4)
    refused(x=a["x"][:, :256]), refused(x=a["x"].short()), refused(x=a["x"].T), refused(x=a["x"][0]), refused(x=a["x"].repeat(1, 2)[:, ::2])
    refused(x=a["x"][:3], x_scale=a["x_scale"][:3])  # fewer rows than the plan's tokens
    refused(x_scale=a["x_scale"][:3]), refused(x_scale=a["x_scale"].int()), refused(x_scale=a["x_scale"].repeat(1, 2))
    refused(w=a["w"][:, :200]), refused(w=a["w"][:1]), refused(w=a["w"][:, :, :264]), refused(w=a["w"].transpose(1, 2)), refused(w=a["w"].bfloat16())
    refused(w_scale=a["w_scale"][:, :1]), refused(w_scale=a["w_scale"].float()), refused(w_scale=a["w_scale"][0])
    refused(y=a["y"][:5]), refused(y=a["y"][:, :192]), refused(y=a["y"].float()), refused(y=a["y"].half()), refused(y=a["y"].T), refused(y=a["y"][0])
    refused(y=torch.zeros((6, 400), dtype=torch.bfloat16)[:, ::2])
    refused(expert_offset=a["expert_offset"][:2]), refused(expert_offset=a["expert_offset"].long())
    refused(expert_offset=torch.zeros(6, dtype=torch.int32)[::2])
    refused(row_token=a["row_token"][:5]), refused(row_token=a["row_token"].long()), refused(row_token=torch.zeros(12, dtype=torch.int32)[::2])
    for name in ("x", "x_scale", "expert_offset", "w", "w_scale", "y"):
        refused(**{name: None})
    a = _product()
    refused(x=a["x"][:, :256]), refused(x_scale=a["x_scale"][:5])


def test_product_without_rows_takes_no_tensors():
    a = _product(rows=0)
    capmoe.moe_grouped_gemm_fp8(a["gemm"], None, None, None, None, None, None, None, None, stream=_NoStream)
    for bad in (capmoe.make_gemm(-1, 256, 64), capmoe.make_gemm(4, 0, 64), capmoe.make_gemm(4, 256, 0), capmoe.make_gemm(4, 256, 64, 0),
                capmoe.make_gemm(4, 256, 12), capmoe.make_gemm(4, 256, 64, 257), capmoe.make_gemm(4, (1 << 21) + 8, 64)):
        with pytest.raises(capmoe.CapMoeError):  # the call's own refusals
            capmoe.moe_grouped_gemm_fp8(bad, **{k: v for k, v in a.items() if k != "gemm"}, stream=_NoStream)


class _GpuStream(_NoStream):
    device_index = 0


def test_binding_refuses_tensors_of_another_device():
    x, token, count = torch.zeros((4, 64), dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    q, s = capmoe.fp8_row_buffers(4, 64, device="cpu")
    w = torch.zeros((2, 8, 64), dtype=torch.bfloat16)
    wq, ws = capmoe.fp8_weight_buffers(2, 8, 64, device="cpu")
    for call in (lambda: capmoe.moe_quantize_rows(x, token, count, q, s, stream=_GpuStream),
                 lambda: capmoe.moe_quantize_rows(x, None, None, q, s, stream=_GpuStream),
                 lambda: capmoe.moe_quantize_weights(w, wq, ws, stream=_GpuStream),
                 lambda: capmoe.moe_grouped_gemm_fp8(**_product(), stream=_GpuStream),
                 lambda: capmoe.moe_grouped_gemm_fp8(**_product(src=4), stream=_GpuStream)):
        with pytest.raises(ValueError, match="device"):
            call()


def test_experts_lie_on_one_device():
    parts = [t for sizes in ((2, 200, 72), (2, 200, 72), (2, 72, 200)) for t in capmoe.fp8_weight_buffers(*sizes, device="cpu")]
    for i in range(6):
        with pytest.raises(ValueError, match="device"):
            capmoe.Fp8Experts(*parts[:i], parts[i].to("meta"), *parts[i + 1:])


def test_ffn_calls_refuse_tensors_of_another_device():
    desc = _desc(d_model=72, n_experts=2, top_k=1)
    parts = [t for sizes in ((2, 200, 72), (2, 200, 72), (2, 72, 200)) for t in capmoe.fp8_weight_buffers(*sizes, device="cpu")]
    experts, x = capmoe.Fp8Experts(*parts), torch.zeros((16, 72), dtype=torch.bfloat16)
    offset, token, work = torch.zeros(3, dtype=torch.int32), torch.zeros(16, dtype=torch.int32), torch.empty(1 << 20, dtype=torch.uint8)
    buf = capmoe.LayerBuffers(desc, device="cpu", fp8=True)
    router = torch.zeros((2, 72))
    for call in (lambda: capmoe.moe_grouped_ffn_fp8(desc, x, offset, experts, x, work, stream=_GpuStream),
                 lambda: capmoe.moe_dispatch_ffn_fp8(desc, x, offset, token, experts, x, work, stream=_GpuStream),
                 lambda: capmoe.moe_layer_forward_fp8(desc, x, router, None, experts, None, 0, buf, stream=_GpuStream)):
        with pytest.raises(ValueError, match="device"):
            call()


def test_binding_refuses_counts_that_are_no_int32():
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    q, s = capmoe.fp8_row_buffers(4, 64, device="cpu")
    # an empty tensor has no address: all rows would be done instead of none
    for bad in (torch.zeros(1), torch.zeros(1, dtype=torch.int64), torch.zeros(0, dtype=torch.int32)):
        with pytest.raises(ValueError, match="row_count"):
            capmoe.moe_quantize_rows(x, None, bad, q, s, stream=_NoStream)


def test_calls_that_ran_without_a_device_to_compare_still_run():
    class Handle:  # of a stream that something else made
        cuda_stream = None

    a = _product(rows=0)
    capmoe.moe_grouped_gemm_fp8(**a, stream=Handle)
    # a workspace of no bytes, wherever it is
    a["workspace"] = torch.empty(0, dtype=torch.uint8, device="meta")
    b = {k: v for k, v in a.items() if k in ("gemm", "row_token", "workspace")}
    capmoe.moe_grouped_gemm_fp8(**b, x=None, x_scale=None, expert_offset=None, w=None, w_scale=None, y=None, stream=_GpuStream)
