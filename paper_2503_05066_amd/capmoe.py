"""Thin binding to libcapmoe.so: same names as the C ABI, argument marshalling only.

Tensors are torch tensors on the GPU (PyTorch is used for device memory and streams, nothing
else); every step of the layer runs in the library's HIP kernels.  There is no fallback: if the
library has not been built, loading raises.
"""
from __future__ import annotations

import ctypes
import functools
import math
import os

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libcapmoe.so")

MOE_OK = 0
MODE_NONE, MODE_TOKEN_DROP, MODE_EXPANDED_DROP = 0, 1, 2
SCOPE_LOCAL, SCOPE_GLOBAL, SCOPE_LOCAL_DEVICE, SCOPE_GLOBAL_DEVICE = 0, 1, 2, 3
DTYPE_F32, DTYPE_BF16 = 0, 1
METRIC_SCORE, METRIC_ORDER, METRIC_REVERSE_ORDER, METRIC_RANDOM = 0, 1, 2, 3


class MoeDesc(ctypes.Structure):
    """moe_desc_t of include/capmoe.h."""

    _fields_ = [
        ("n_tokens", ctypes.c_int32), ("d_model", ctypes.c_int32), ("n_experts", ctypes.c_int32),
        ("top_k", ctypes.c_int32), ("d_hidden", ctypes.c_int32), ("device_groups", ctypes.c_int32),
        ("mode", ctypes.c_int32), ("capacity_scope", ctypes.c_int32), ("gamma", ctypes.c_double),
        ("dtype", ctypes.c_int32), ("metric", ctypes.c_int32),
        ("overselect", ctypes.c_int32), ("max_experts", ctypes.c_int32),
    ]


class MoeGemm(ctypes.Structure):
    """moe_gemm_t of include/capmoe.h."""

    _fields_ = [(n, ctypes.c_int32) for n in ("max_rows", "src_rows", "n_experts", "n_in", "n_out")]


class MoeFp8Experts(ctypes.Structure):
    """moe_fp8_experts_t of include/capmoe.h."""

    _fields_ = [(n, ctypes.c_void_p) for n in ("gate", "gate_scale", "up", "up_scale", "down", "down_scale")]


KERNELS = ("router_logits", "softmax_topk", "drop_prepare", "drop_select", "drop_emit", "dispatch", "ffn_schedule",
           "ffn_gate_up", "ffn_down", "combine", "drop_limit")


class MoeProfile(ctypes.Structure):
    """moe_profile_t of include/capmoe.h: event handles per kernel id and the library's launch counts."""

    _fields_ = [("start", ctypes.c_void_p * len(KERNELS)), ("stop", ctypes.c_void_p * len(KERNELS)),
                ("launches", ctypes.c_int64 * len(KERNELS))]

    def set_events(self, kernel: int, start_event, stop_event):
        """torch.cuda.Event pair (created with enable_timing) for one kernel id, or None, None."""
        def handle(ev):
            if ev is None:
                return None
            if not ev.cuda_event:      # torch creates the hipEvent lazily; recording once materialises it
                ev.record()
            return ev.cuda_event
        self.start[kernel] = handle(start_event)
        self.stop[kernel] = handle(stop_event)


class CapMoeError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {status_string(status)} (status {status})")


_lib = None


def load():
    """Load the shared library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2503_05066_amd.build` "
                               "(there is no fallback path)")
        lib = ctypes.CDLL(LIB_PATH)
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
        dp = ctypes.POINTER(MoeDesc)
        lib.moe_status_string.argtypes = [i32]
        lib.moe_status_string.restype = ctypes.c_char_p
        lib.moe_query.argtypes = [dp, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32),
                                  ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_size_t)]
        lib.moe_route_topk.argtypes = [dp, vp, vp, vp, i32, vp, vp, vp, vp, vp, sz, vp]
        lib.moe_route_topk_static.argtypes = [dp, vp, vp, vp, i32, vp, vp, vp, vp, vp]
        lib.moe_capacity_drop.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.moe_capacity_drop_ranked.argtypes = [dp, vp, vp, vp, ctypes.c_uint32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.moe_dispatch.argtypes = [dp, vp, vp, vp, vp, vp]
        lib.moe_grouped_ffn.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.moe_dispatch_ffn.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.moe_combine.argtypes = [dp, vp, vp, vp, vp, vp]
        lib.moe_layer_forward.argtypes = [dp] + [vp] * 7 + [ctypes.c_uint32] + [vp] * 13 + [sz, vp]
        lib.moe_layer_forward.restype = i32
        lib.moe_profile_attach.argtypes = [ctypes.POINTER(MoeProfile)]
        lib.moe_profile_attach.restype = i32
        lib.moe_ffn_schedule_query.argtypes = [ctypes.POINTER(MoeDesc), vp, i32, vp, vp]
        lib.moe_ffn_schedule_query.restype = i32
        lib.moe_probe_mfma_bf16.argtypes = [i32, i32, i32, vp, ctypes.POINTER(ctypes.c_int64), vp]
        lib.moe_probe_mfma_bf16.restype = i32
        gp, ep, i64 = ctypes.POINTER(MoeGemm), ctypes.POINTER(MoeFp8Experts), ctypes.c_int64
        lib.moe_fp8_query.argtypes = [ctypes.c_int32, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32)]
        lib.moe_quantize_rows.argtypes = [i32, vp, i64, ctypes.c_int32, vp, vp, vp, vp, vp]
        lib.moe_quantize_weights.argtypes = [i32, vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, vp, vp, vp]
        lib.moe_gemm_query.argtypes = [gp, ctypes.POINTER(ctypes.c_size_t)]
        lib.moe_grouped_gemm_fp8.argtypes = [gp] + [vp] * 8 + [sz, vp]
        lib.moe_query_fp8.argtypes = [dp, ctypes.POINTER(ctypes.c_size_t)]
        lib.moe_grouped_ffn_fp8.argtypes = [dp, vp, vp, ep, vp, vp, sz, vp]
        lib.moe_dispatch_ffn_fp8.argtypes = [dp, vp, vp, vp, ep, vp, vp, sz, vp]
        lib.moe_layer_forward_fp8.argtypes = [dp, vp, vp, vp, ep, vp, ctypes.c_uint32] + [vp] * 13 + [sz, vp]
        for f in ("moe_fp8_query", "moe_quantize_rows", "moe_quantize_weights", "moe_gemm_query", "moe_grouped_gemm_fp8",
                  "moe_query_fp8", "moe_grouped_ffn_fp8", "moe_dispatch_ffn_fp8", "moe_layer_forward_fp8"):
            getattr(lib, f).restype = i32
        for f in ("moe_query", "moe_route_topk", "moe_route_topk_static", "moe_capacity_drop", "moe_capacity_drop_ranked", "moe_dispatch",
                  "moe_grouped_ffn",
                  "moe_dispatch_ffn", "moe_combine"):
            getattr(lib, f).restype = i32
        _lib = lib
    return _lib


def status_string(status: int) -> str:
    return load().moe_status_string(int(status)).decode()


def make_desc(n_tokens, d_model, n_experts, top_k, d_hidden, device_groups=1, mode=MODE_TOKEN_DROP,
              capacity_scope=SCOPE_LOCAL, gamma=1.0, dtype=DTYPE_BF16, metric=METRIC_SCORE, overselect=0,
              max_experts=0) -> MoeDesc:
    return MoeDesc(n_tokens, d_model, n_experts, top_k, d_hidden, device_groups, mode, capacity_scope,
                   float(gamma), dtype, metric, overselect, int(max_experts))


def _ptr(t):
    return None if t is None else t.data_ptr()  # every argtype is declared, a number will do


def _stream(stream):
    if stream is None:
        import torch

        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def _stream_on(stream, *tensors):
    """_stream for calls that look at their tensors: all of them lie on the stream's device (host memory, or another GPU's, is
    no address of a kernel there).  A handle that names no device is not compared."""
    if stream is None:
        import torch

        stream = torch.cuda.current_stream(torch.cuda.current_device())  # 1.3 us; without the argument 2.6
    device = getattr(stream, "device_index", None)
    for t in tensors:
        if t is not None and t.get_device() != device and device is not None:
            raise ValueError(f"a tensor on {t.device}, a stream of device {device}")
    return stream.cuda_stream


def _check(status: int, what: str):
    if status != MOE_OK:
        raise CapMoeError(status, what)


def moe_query(desc: MoeDesc):
    """(cap, slots_per_token, max_rows, workspace_bytes) of a descriptor; host only."""
    cap, slots = ctypes.c_int32(), ctypes.c_int32()
    rows, ws = ctypes.c_int64(), ctypes.c_size_t()
    _check(load().moe_query(ctypes.byref(desc), ctypes.byref(cap), ctypes.byref(slots), ctypes.byref(rows),
                            ctypes.byref(ws)), "moe_query")
    return cap.value, slots.value, rows.value, ws.value


def moe_route_topk(desc, x, w_router, bias, use_given_logits, logits, scores, topk_idx, topk_score, workspace,
                   stream=None):
    _check(load().moe_route_topk(ctypes.byref(desc), _ptr(x), _ptr(w_router), _ptr(bias), int(use_given_logits),
                                 _ptr(logits), _ptr(scores), _ptr(topk_idx), _ptr(topk_score), _ptr(workspace),
                                 workspace.numel() * workspace.element_size() if workspace is not None else 0,
                                 _stream(stream)), "moe_route_topk")


def moe_route_topk_static(desc, x, w_router, bias, use_given_logits, logits, scores, topk_idx, topk_score, stream=None):
    _check(load().moe_route_topk_static(ctypes.byref(desc), _ptr(x), _ptr(w_router), _ptr(bias),
                                        int(use_given_logits), _ptr(logits), _ptr(scores), _ptr(topk_idx),
                                        _ptr(topk_score), _stream(stream)), "moe_route_topk_static")


def moe_capacity_drop(desc, scores, topk_idx, expert_count, seg_count, expert_offset, row_token, row_weight,
                      pair_row, workspace, stream=None):
    _check(load().moe_capacity_drop(ctypes.byref(desc), _ptr(scores), _ptr(topk_idx), _ptr(expert_count),
                                    _ptr(seg_count), _ptr(expert_offset), _ptr(row_token), _ptr(row_weight),
                                    _ptr(pair_row), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                    _stream(stream)), "moe_capacity_drop")


def moe_capacity_drop_ranked(desc, scores, topk_idx, token_class, seed, expert_count, seg_count, expert_offset,
                             row_token, row_weight, pair_row, workspace, stream=None):
    _check(load().moe_capacity_drop_ranked(ctypes.byref(desc), _ptr(scores), _ptr(topk_idx), _ptr(token_class),
                                           int(seed) & 0xFFFFFFFF, _ptr(expert_count), _ptr(seg_count),
                                           _ptr(expert_offset), _ptr(row_token), _ptr(row_weight), _ptr(pair_row),
                                           _ptr(workspace), workspace.numel() * workspace.element_size(),
                                           _stream(stream)), "moe_capacity_drop_ranked")


def moe_dispatch(desc, x, expert_offset, row_token, xp, stream=None):
    _check(load().moe_dispatch(ctypes.byref(desc), _ptr(x), _ptr(expert_offset), _ptr(row_token), _ptr(xp),
                               _stream(stream)), "moe_dispatch")


def moe_grouped_ffn(desc, xp, expert_offset, w_gate, w_up, w_down, yp, workspace, stream=None):
    _check(load().moe_grouped_ffn(ctypes.byref(desc), _ptr(xp), _ptr(expert_offset), _ptr(w_gate), _ptr(w_up),
                                  _ptr(w_down), _ptr(yp), _ptr(workspace),
                                  workspace.numel() * workspace.element_size(), _stream(stream)), "moe_grouped_ffn")


def moe_dispatch_ffn(desc, x, expert_offset, row_token, w_gate, w_up, w_down, yp, workspace, stream=None):
    _check(load().moe_dispatch_ffn(ctypes.byref(desc), _ptr(x), _ptr(expert_offset), _ptr(row_token), _ptr(w_gate),
                                   _ptr(w_up), _ptr(w_down), _ptr(yp), _ptr(workspace),
                                   workspace.numel() * workspace.element_size(), _stream(stream)), "moe_dispatch_ffn")


def moe_combine(desc, yp, row_weight, pair_row, y, stream=None):
    _check(load().moe_combine(ctypes.byref(desc), _ptr(yp), _ptr(row_weight), _ptr(pair_row), _ptr(y),
                              _stream(stream)), "moe_combine")


def moe_layer_forward(desc, x, w_router, bias, w_gate, w_up, w_down, token_class, seed, buf, stream=None):
    """The whole layer through the one-call entry point, into the buffers of a LayerBuffers."""
    ws = buf.workspace
    _check(load().moe_layer_forward(
        ctypes.byref(desc), _ptr(x), _ptr(w_router), _ptr(bias), _ptr(w_gate), _ptr(w_up), _ptr(w_down),
        _ptr(token_class), int(seed) & 0xFFFFFFFF, _ptr(buf.logits), _ptr(buf.scores), _ptr(buf.topk_idx),
        _ptr(buf.topk_score), _ptr(buf.expert_count), _ptr(buf.seg_count), _ptr(buf.expert_offset),
        _ptr(buf.row_token), _ptr(buf.row_weight), _ptr(buf.pair_row), _ptr(buf.yp), _ptr(buf.y), _ptr(ws),
        ws.numel() * ws.element_size(), _stream(stream)), "moe_layer_forward")
    return buf.y


def moe_fp8_query(cols: int):
    """(pitch, scale_pitch) in bytes of an 8-bit matrix of this many columns; host only."""
    pitch, scale_pitch = ctypes.c_int32(), ctypes.c_int32()
    _check(load().moe_fp8_query(int(cols), ctypes.byref(pitch), ctypes.byref(scale_pitch)), "moe_fp8_query")
    return pitch.value, scale_pitch.value


def _fits(ok, what):
    """The quantising calls read their sizes off the tensors, so a tensor that does not fit them is refused here."""
    if not ok:
        raise ValueError(what)


@functools.lru_cache(maxsize=None)
def _product_dtypes():
    import torch

    return torch.bfloat16, torch.int32


_value_dtypes = {}


def _value_dtype(t, dims, what):
    if not _value_dtypes:
        import torch

        _value_dtypes.update({torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16, "int32": torch.int32})
    dtype = _value_dtypes.get(t.dtype)
    if dtype is None or t.dim() != dims or not t.is_contiguous():
        raise ValueError(f"{what}: a dense bf16 or fp32 tensor of {dims} dimensions")
    return dtype


def _fits_fp8(t, shape, what):
    if t.shape != shape or t.element_size() != 1 or not t.is_contiguous():
        raise ValueError(f"{what}: a dense tensor of {shape} bytes")


_fp8_pitches = functools.lru_cache(maxsize=256)(lambda cols: moe_fp8_query(cols))


def moe_quantize_rows(x, row_token, row_count, q, scale, stream=None):
    """x [*, cols] (bf16 or fp32) into the 8-bit rows q [n_rows, pitch], scale [n_rows, scale_pitch]."""
    dtype = _value_dtype(x, 2, "x")
    n_rows, cols = q.shape[0], x.shape[1]
    pitch, scale_pitch = _fp8_pitches(cols)
    _fits_fp8(q, (n_rows, pitch), "q")
    _fits_fp8(scale, (n_rows, scale_pitch), "scale")
    if row_token is None:
        _fits(x.shape[0] >= n_rows, "x: a row for every row of q")
    else:
        _fits(row_token.dtype == _value_dtypes["int32"] and row_token.numel() >= n_rows and row_token.is_contiguous(),
              "row_token: a dense int32 for every row of q")
    if row_count is not None:
        _fits(row_count.dtype == _value_dtypes["int32"] and row_count.numel() > 0, "row_count: an int32")
    _check(load().moe_quantize_rows(dtype, _ptr(x), n_rows, cols, _ptr(row_token), _ptr(row_count), _ptr(q), _ptr(scale),
                                    _stream_on(stream, x, row_token, row_count, q, scale)), "moe_quantize_rows")


def moe_quantize_weights(w, q, scale, stream=None):
    """w [E, n_out, n_in] (bf16 or fp32) into the 8-bit weights q, scale (see fp8_weight_buffers)."""
    dtype = _value_dtype(w, 3, "w")
    e, n_out, n_in = w.shape
    pitch, scale_pitch = _fp8_pitches(n_in)
    blocks = -(-n_out // 128)
    _fits_fp8(q, (e, blocks * 128, pitch), "q")
    _fits_fp8(scale, (e, blocks, scale_pitch), "scale")
    _check(load().moe_quantize_weights(dtype, _ptr(w), e, n_out, n_in, _ptr(q), _ptr(scale), _stream_on(stream, w, q, scale)),
           "moe_quantize_weights")


def fp8_row_buffers(n_rows: int, cols: int, device="cuda"):
    """(values, scales) of the 8-bit form of [n_rows, cols], uninitialised."""
    import torch

    pitch, scale_pitch = moe_fp8_query(cols)
    return (torch.empty((n_rows, pitch), dtype=torch.uint8, device=device),
            torch.empty((n_rows, scale_pitch), dtype=torch.uint8, device=device))


def fp8_weight_buffers(n_experts: int, n_out: int, n_in: int, device="cuda"):
    """(values, scales) of the 8-bit form of expert weights [n_experts, n_out, n_in], uninitialised."""
    import torch

    pitch, scale_pitch = moe_fp8_query(n_in)
    blocks = -(-n_out // 128)
    return (torch.empty((n_experts, blocks * 128, pitch), dtype=torch.uint8, device=device),
            torch.empty((n_experts, blocks, scale_pitch), dtype=torch.uint8, device=device))


class Fp8Experts:
    """The 8-bit weights of a layer's experts (keeps the tensors alive; allocation and marshalling only)."""

    def __init__(self, gate, gate_scale, up, up_scale, down, down_scale):
        e, h, d = gate.shape
        for q, scale, n, k in ((gate, gate_scale, h, d), (up, up_scale, h, d), (down, down_scale, d, h)):
            if tuple(q.shape) != (e, n, k) or n % 128 or k % 128 or q.element_size() != 1 or not q.is_contiguous():
                raise ValueError(f"8-bit expert weights {tuple(q.shape)}: expected {(e, n, k)}, multiples of 128, one byte, contiguous")
            if tuple(scale.shape) != (e, n // 128, -(-k // 512) * 4) or scale.element_size() != 1 or not scale.is_contiguous():
                raise ValueError(f"scales {tuple(scale.shape)} of expert weights {(e, n, k)}")
            if q.device != gate.device or scale.device != gate.device:
                raise ValueError("8-bit expert weights on more than one device")
        self.sizes = (e, h, d)  # filled up to multiples of 128
        self.tensors = (gate, gate_scale, up, up_scale, down, down_scale)
        self.struct = MoeFp8Experts(*[t.data_ptr() for t in self.tensors])

    def of(self, desc: MoeDesc):
        """The struct for a call of that layer."""
        if self.sizes != (desc.n_experts, -(-desc.d_hidden // 128) * 128, -(-desc.d_model // 128) * 128):
            raise ValueError(f"8-bit experts of {self.sizes} do not belong to this layer")
        return ctypes.byref(self.struct)

    @classmethod
    def quantized(cls, w_gate, w_up, w_down, stream=None):
        """From w_gate, w_up [E,h,d] and w_down [E,d,h] in bf16 or fp32 (as at model load).  The tensors belong to `stream`:
        work on others that uses them waits for it."""
        import torch

        tensors = []
        with torch.cuda.stream(stream):  # their memory too: what another stream gave back, its work may still write
            for w in (w_gate, w_up, w_down):
                q, scale = fp8_weight_buffers(*w.shape, device=w.device)
                moe_quantize_weights(w, q, scale, stream)
                tensors += [q, scale]
        return cls(*tensors)


def make_gemm(max_rows, n_in, n_out, n_experts=1, src_rows=0) -> MoeGemm:
    return MoeGemm(max_rows, src_rows, n_experts, n_in, n_out)


def moe_gemm_query(gemm: MoeGemm) -> int:
    """Workspace bytes of moe_grouped_gemm_fp8; host only."""
    ws = ctypes.c_size_t()
    _check(load().moe_gemm_query(ctypes.byref(gemm), ctypes.byref(ws)), "moe_gemm_query")
    return ws.value


@functools.lru_cache(maxsize=256)
def _product_sizes(gemm: bytes):
    """The fields of a MoeGemm that the call accepts, and what they say of the tensors."""
    sizes = MoeGemm.from_buffer_copy(gemm)
    moe_gemm_query(sizes)  # refuses sizes that the call refuses
    pitch, scale_pitch = moe_fp8_query(sizes.n_in)
    w = (sizes.n_experts, -(-sizes.n_out // 128) * 128, pitch)
    w_bytes, w_scale_bytes = math.prod(w), w[0] * (w[1] // 128) * scale_pitch
    return sizes.max_rows, sizes.src_rows, 4 * (sizes.n_experts + 1), sizes.n_out, pitch, scale_pitch, w, w_bytes, w_scale_bytes


def _fits_product(gemm, x, x_scale, row_token, expert_offset, w, w_scale, y):
    """False if there are no rows, else every tensor against the sizes of the call.  (Of rows that are not gathered, x holds as
    many as expert_offset ends with, known on the device only.)  In one expression, 1.2 us: one by one the checks took 2 us more, of
    8 for a token's experts."""
    max_rows, src_rows, offset_bytes, n_out, pitch, scale_pitch, w_shape, w_bytes, w_scale_bytes = _product_sizes(bytes(gemm))
    if max_rows == 0:
        return False
    bf16, int32 = _product_dtypes()
    try:
        (rows, cols), (y_rows, y_cols) = x.shape, y.shape
        fits = (cols == pitch and x.nbytes == rows * pitch and x.is_contiguous() and
                x_scale.nbytes == rows * scale_pitch and x_scale.is_contiguous() and
                w.shape == w_shape and w.nbytes == w_bytes and w.is_contiguous() and
                w_scale.nbytes == w_scale_bytes and w_scale.is_contiguous() and
                y.dtype is bf16 and y_cols == n_out and y_rows >= max_rows and y.is_contiguous() and
                expert_offset.dtype is int32 and expert_offset.nbytes >= offset_bytes and expert_offset.is_contiguous() and
                (row_token is None or rows >= src_rows and row_token.dtype is int32 and row_token.nbytes >= 4 * max_rows and
                 row_token.is_contiguous()))
    except (AttributeError, ValueError):  # no tensor, or not of two dimensions
        fits = False
    if not fits:
        raise ValueError(f"a product of {max_rows} rows (of {src_rows}, with row_token) takes dense tensors: x bytes [rows, {pitch}], x_scale "
                         f"bytes [rows, {scale_pitch}], w bytes {list(w_shape)}, w_scale {w_scale_bytes} bytes, y bf16 [max_rows, {n_out}], "
                         f"expert_offset int32 [{offset_bytes // 4}], row_token int32 [max_rows]")
    return True


def moe_grouped_gemm_fp8(gemm, x, x_scale, row_token, expert_offset, w, w_scale, y, workspace, stream=None):
    """workspace may be None where moe_gemm_query answers 0.  A tensor that does not fit the sizes of gemm is refused."""
    arrays = (None,) * 7  # without rows none is read
    if _fits_product(gemm, x, x_scale, row_token, expert_offset, w, w_scale, y):
        arrays = (x.data_ptr(), x_scale.data_ptr(), None if row_token is None else row_token.data_ptr(), expert_offset.data_ptr(),
                  w.data_ptr(), w_scale.data_ptr(), y.data_ptr())
    _check(load().moe_grouped_gemm_fp8(ctypes.byref(gemm), *arrays, _ptr(workspace),
                                       workspace.numel() * workspace.element_size() if workspace is not None else 0,
                                       _stream_on(stream, x, x_scale, row_token, expert_offset, w, w_scale, y)), "moe_grouped_gemm_fp8")


def moe_query_fp8(desc: MoeDesc) -> int:
    """Workspace bytes of a layer with 8-bit experts; host only."""
    ws = ctypes.c_size_t()
    _check(load().moe_query_fp8(ctypes.byref(desc), ctypes.byref(ws)), "moe_query_fp8")
    return ws.value


def moe_grouped_ffn_fp8(desc, xp, expert_offset, experts: Fp8Experts, yp, workspace, stream=None):
    _check(load().moe_grouped_ffn_fp8(ctypes.byref(desc), _ptr(xp), _ptr(expert_offset), experts.of(desc),
                                      _ptr(yp), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                      _stream_on(stream, xp, expert_offset, yp, workspace, experts.tensors[0])), "moe_grouped_ffn_fp8")


def moe_dispatch_ffn_fp8(desc, x, expert_offset, row_token, experts: Fp8Experts, yp, workspace, stream=None):
    _check(load().moe_dispatch_ffn_fp8(ctypes.byref(desc), _ptr(x), _ptr(expert_offset), _ptr(row_token),
                                       experts.of(desc), _ptr(yp), _ptr(workspace),
                                       workspace.numel() * workspace.element_size(),
                                       _stream_on(stream, x, expert_offset, row_token, yp, workspace, experts.tensors[0])),
           "moe_dispatch_ffn_fp8")


def moe_layer_forward_fp8(desc, x, w_router, bias, experts: Fp8Experts, token_class, seed, buf, stream=None):
    """The whole layer with 8-bit experts, into the buffers of a LayerBuffers made with fp8=True."""
    ws = buf.workspace
    _check(load().moe_layer_forward_fp8(
        ctypes.byref(desc), _ptr(x), _ptr(w_router), _ptr(bias), experts.of(desc), _ptr(token_class),
        int(seed) & 0xFFFFFFFF, _ptr(buf.logits), _ptr(buf.scores), _ptr(buf.topk_idx), _ptr(buf.topk_score),
        _ptr(buf.expert_count), _ptr(buf.seg_count), _ptr(buf.expert_offset), _ptr(buf.row_token),
        _ptr(buf.row_weight), _ptr(buf.pair_row), _ptr(buf.yp), _ptr(buf.y), _ptr(ws),
        ws.numel() * ws.element_size(), _stream_on(stream, x, w_router, bias, token_class, ws, experts.tensors[0])),
        "moe_layer_forward_fp8")
    return buf.y


def moe_profile_attach(table: "MoeProfile | None"):
    """Attach the caller's profile table to this thread (None detaches).  The caller keeps the table alive."""
    _check(load().moe_profile_attach(ctypes.byref(table) if table is not None else None), "moe_profile_attach")


def moe_ffn_schedule_query(desc: MoeDesc, expert_count, compute_units: int = 256):
    """What the tile schedule of the expert GEMMs decides for these rows per expert (host only, nothing is launched):
    ((big tiles, short tiles), [gate/up header of 8 ints, down header of 8 ints])."""
    counts = (ctypes.c_int32 * desc.n_experts)(*[int(c) for c in expert_count])
    tiles = (ctypes.c_int32 * 2)()
    header = (ctypes.c_int32 * 16)()
    _check(load().moe_ffn_schedule_query(ctypes.byref(desc), counts, int(compute_units), tiles, header),
           "moe_ffn_schedule_query")
    return (tiles[0], tiles[1]), [list(header[:8]), list(header[8:])]


def moe_probe_mfma_bf16(blocks: int, iterations: int, sink, random_operands: bool = False, stream=None) -> int:
    """Launch the matrix-core probe; returns the flops of the launch (the caller times it)."""
    flops = ctypes.c_int64(0)
    assert sink.numel() >= blocks * 256
    _check(load().moe_probe_mfma_bf16(int(blocks), int(iterations), int(bool(random_operands)), _ptr(sink),
                                      ctypes.byref(flops), _stream(stream)), "moe_probe_mfma_bf16")
    return int(flops.value)


class LayerBuffers:
    """Device buffers of one layer call, sized by moe_query (allocation only, no arithmetic)."""

    def __init__(self, desc: MoeDesc, device="cuda", fp8=False):
        import torch

        self.desc = desc
        self.cap, self.slots, self.max_rows, self.workspace_bytes = moe_query(desc)
        if fp8:  # for the calls with 8-bit experts as well
            self.workspace_bytes = moe_query_fp8(desc)
        n, e, k, d = desc.n_tokens, desc.n_experts, desc.top_k + desc.overselect, desc.d_model
        blocks = desc.device_groups if desc.capacity_scope in (SCOPE_LOCAL, SCOPE_LOCAL_DEVICE) else 1
        act = torch.bfloat16 if desc.dtype == DTYPE_BF16 else torch.float32
        rows = max(self.max_rows, 1)
        i32, f32 = torch.int32, torch.float32
        mk = lambda shape, dt: torch.empty(shape, dtype=dt, device=device)
        self.logits, self.scores = mk((n, e), f32), mk((n, e), f32)
        self.topk_idx, self.topk_score = mk((n, k), i32), mk((n, k), f32)
        self.expert_count, self.seg_count = mk((e,), i32), mk((blocks, e), i32)
        self.expert_offset = mk((e + 1,), i32)
        self.row_token, self.row_weight = mk((rows,), i32), mk((rows,), f32)
        self.pair_row = mk((n, self.slots), i32)
        self.xp, self.yp = mk((rows, d), act), mk((rows, d), act)
        self.y = mk((n, d), act)
        self.workspace = mk((max(self.workspace_bytes, 256),), torch.uint8)


def layer_forward(buf: LayerBuffers, x, w_router, bias, w_gate, w_up, w_down, given_logits=None, stream=None,
                  fused_dispatch=False, token_class=None, seed=0):
    """The calls of one layer, enqueued back to back on one stream; returns buf.y.

    fused_dispatch=False: the five calls route_topk, capacity_drop, dispatch, grouped_ffn, combine.
    fused_dispatch=True: dispatch and grouped_ffn are replaced by moe_dispatch_ffn (xp is not written).
    """
    d = buf.desc
    if given_logits is not None:
        buf.logits.copy_(given_logits)
    moe_route_topk(d, x, w_router, bias, given_logits is not None, buf.logits, buf.scores, buf.topk_idx,
                   buf.topk_score, buf.workspace, stream)
    if token_class is None and seed == 0:
        moe_capacity_drop(d, buf.scores, buf.topk_idx, buf.expert_count, buf.seg_count, buf.expert_offset,
                          buf.row_token, buf.row_weight, buf.pair_row, buf.workspace, stream)
    else:
        moe_capacity_drop_ranked(d, buf.scores, buf.topk_idx, token_class, seed, buf.expert_count, buf.seg_count,
                                 buf.expert_offset, buf.row_token, buf.row_weight, buf.pair_row, buf.workspace, stream)
    if fused_dispatch:
        moe_dispatch_ffn(d, x, buf.expert_offset, buf.row_token, w_gate, w_up, w_down, buf.yp, buf.workspace, stream)
    else:
        moe_dispatch(d, x, buf.expert_offset, buf.row_token, buf.xp, stream)
        moe_grouped_ffn(d, buf.xp, buf.expert_offset, w_gate, w_up, w_down, buf.yp, buf.workspace, stream)
    moe_combine(d, buf.yp, buf.row_weight, buf.pair_row, buf.y, stream)
    return buf.y


def is_unbounded(gamma) -> bool:
    return math.isinf(gamma)
