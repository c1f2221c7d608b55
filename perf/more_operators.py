"""The operators of 4-bit experts and of the norm ahead of them, as timed cases.

A case names one operator:

  "norm"     moe_norm_rows: the residual's addition and the root-mean-square norm, with an output in 8 or 4 bits
  "rows"     moe_quantize_rows_fp4: activations to e2m1 with a power-of-two scale per row and 32 columns, permuted or not
  "weights"  moe_quantize_weights_fp4: expert weights to the same format (model load)
  "gemm"     moe_grouped_gemm_fp4: the product of 4-bit rows, grouped by expert with ragged sizes, and 4-bit weights
  "ffn"      moe_dispatch_ffn_fp4: the SwiGLU expert FFN on 4-bit weights, from tokens to bf16 expert outputs

What a case leaves in 8 or 4 bits it returns as the values that it stands for, in bf16, which holds them all
(moe_dequantize_rows).  Sizes are those of the workloads in paper_2503_05066_amd/synth.py, of the tests and of bench.py, with
ragged ones of the same families between them.

A 4-bit matrix of c columns has rows of 128 * ceil(c / 256) bytes, two values each, the lower column in the lower four bits,
zero behind the columns, and 16 * ceil(c / 512) scale bytes per row: byte 4 * (b % 4) + b / 4 of a group of 16 belongs to the
group's b-th 32 columns and stands for 2^(byte - 127), 255 for no number.  Weights have a multiple of 128 rows, filled up with
zeros.  An 8-bit matrix has rows of 128 * ceil(c / 128) bytes and 4 * ceil(c / 512) scale bytes, one per 128 columns.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _up(n, m):
    return -(-n // m) * m


def _norm_case(name, dtype, rows, cols, residual, y, bits):
    return {"name": name, "op": "norm", "dtype": dtype, "rows": rows, "cols": cols, "residual": residual, "y": y, "bits": bits}


def _rows_case(name, dtype, rows, cols, tokens=0):
    return {"name": name, "op": "rows", "dtype": dtype, "rows": rows, "cols": cols, "tokens": tokens}


def _weights_case(name, dtype, e, n_out, n_in):
    return {"name": name, "op": "weights", "dtype": dtype, "experts": e, "n_out": n_out, "n_in": n_in}


def _gemm_case(name, tokens, e, k, n_in, n_out, gather=False, gamma=0.0, skew="normal", skew_param=1.0):
    return {"name": name, "op": "gemm", "tokens": tokens, "experts": e, "top_k": k, "n_in": n_in,
            "n_out": n_out, "gather": gather, "gamma": gamma, "skew": skew, "skew_param": skew_param}


def _ffn_case(name, tokens, d, e, k, h, small_rows=False, gamma=0.0, skew="normal", skew_param=1.0):
    return {"name": name, "op": "ffn", "tokens": tokens, "experts": e, "top_k": k, "n_in": d, "n_out": h,
            "small_rows": small_rows, "gamma": gamma, "skew": skew, "skew_param": skew_param}


def listed():
    return [
        # ahead of a layer in a decoding batch: latency
        _norm_case("norm_37_decode", "bf16", 37, 4096, True, True, 4),
        # ahead of a layer of a long prompt batch: the router reads bf16, the experts 4 bits
        _norm_case("norm_8192", "bf16", 8192, 4096, True, True, 4),
        # fp32 activations of a width that divides nothing, for a product on 8-bit weights alone
        _norm_case("norm_f32_odd", "f32", 3001, 1416, False, False, 8),
        # a prompt batch permuted into expert-major order on the way: 13 k kept pairs of 4096 tokens
        _rows_case("rows_13000_permuted", "bf16", 13000, 2048, tokens=4096),
        # loading a layer of many small experts
        _weights_case("weights_64_experts", "bf16", 64, 1024, 2048),
        # one projection of a single token's eight experts: latency and the weight stream
        _gemm_case("gemm_1_token", 1, 64, 8, 2048, 1024, skew="zipf", skew_param=1.1),
        # an expert that all tokens share (a dense product) in a short batch, sizes that are no multiples of 128
        _gemm_case("gemm_shared_odd", 203, 1, 1, 2056, 5640),
        # few wide experts, long sums: the matrix cores bind
        _gemm_case("gemm_8192_wide", 8192, 8, 2, 14336, 4096, gamma=1.0, skew_param=1.5),
        # decoding a small batch with few, wide experts: streams nearly all weights for sixteen tokens
        _ffn_case("ffn_16_wide", 16, 4096, 8, 2, 14336, skew_param=0.5),
        # a short ragged prompt on a layer whose counts divide nothing
        _ffn_case("ffn_1531_odd", 1531, 2048, 60, 4, 1408, gamma=1.25, skew="zipf", skew_param=1.0),
        # an ordinary prompt batch, skewed routing under a capacity, tokens that the norm left in 4 bits
        _ffn_case("ffn_4096_rows", 4096, 2048, 64, 8, 1024, small_rows=True, gamma=1.0, skew="zipf", skew_param=1.1),
        # few wide experts, a long prompt batch: the matrix cores bind
        _ffn_case("ffn_8192_wide", 8192, 4096, 8, 2, 14336, gamma=1.0, skew_param=1.5),
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _width(rng, low, high):
    """A row length: a multiple of 128 as models have them, or of 8."""
    n = _log_int(rng, low, high)
    return max(low, _up(n, 128) if rng.random() < 0.6 else _up(n, 8))


def draw(rng):
    op = rng.choice(["norm", "norm", "rows", "weights", "gemm", "gemm", "ffn", "ffn"])
    while True:
        dtype = rng.choice(["bf16", "bf16", "f32"])
        e = rng.choice([1, 4, 8, 16, 32, 60, 64, 96, 128])
        if op == "norm":
            rows, cols, bits = _log_int(rng, 1, 32768), _width(rng, 64, 14336), rng.choice([0, 4, 4, 8])
            c = _norm_case("", dtype, rows, cols, rng.random() < 0.7, bits == 0 or rng.random() < 0.7, bits)
            if rows * cols > 1 << 26:
                continue
        elif op == "rows":
            rows, cols = _log_int(rng, 1, 32768), _width(rng, 64, 14336)
            tokens = rng.choice([0, max(1, rows // rng.choice([1, 2, 5]))])
            c = _rows_case("", dtype, rows, cols, tokens)
            if rows * cols > 1 << 27:
                continue
        elif op == "weights":
            c = _weights_case("", dtype, e, _width(rng, 64, 14336), _width(rng, 64, 14336))
            if e * c["n_out"] * c["n_in"] > 1 << 28:
                continue
        else:
            n = _log_int(rng, 1, 16384)
            k = min(e, rng.choice([1, 2, 4, 6, 8]))
            gamma = rng.choice([0.0, 1.0, 1.5]) if n >= 64 else 0.0
            skew = rng.choice(["normal", "zipf", "one_hot"])
            param = {"normal": round(rng.uniform(0.5, 1.5), 2), "zipf": round(rng.uniform(0.8, 1.2), 2), "one_hot": 3.0}[skew]
            a, b = _width(rng, 256, 8192), _width(rng, 256, 14336)
            if op == "gemm":
                if rng.random() < 0.5:
                    a, b = b, a
                c = _gemm_case("", n, e, k, a, b, rng.random() < 0.5, gamma, skew, param)
            else:
                c = _ffn_case("", n, a, e, k, b, rng.random() < 0.4, gamma, skew, param)
            mats = 3 if op == "ffn" else 1
            if mats * e * a * b > 3 * 8 * 4096 * 14336 or sum(_counts(c)) * mats * a * b > 10 ** 12 or n * k * max(a, b) > 1 << 28:
                continue
            if e * max(_counts(c)) * max(a, b) > 1 << 30:  # the plain form holds every expert's rows up to the longest
                continue
        del c["name"]
        return c


def _counts(case):
    """Rows of each expert: its share of the token-expert pairs under the case's skew, at most the capacity."""
    e, n, p = case["experts"], case["tokens"], case["skew_param"]
    if case["skew"] == "zipf":
        w = np.arange(1, e + 1, dtype=np.float64) ** -p
    elif case["skew"] == "one_hot":
        w = np.ones(e)
        w[0] = math.exp(p)
    else:
        w = np.exp(np.random.default_rng(e).standard_normal(e) * p)
    pairs = n * case["top_k"]
    ends = np.round(np.cumsum(w / w.sum()) * pairs).astype(int)
    cap = n if case["gamma"] == 0.0 else min(n, int(case["gamma"] * pairs / e))
    return [int(min(c, cap)) for c in np.diff(ends, prepend=0)]


# ---------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------
def _two_to(e):
    """2^e, e whole numbers of at least -127, exactly."""
    return torch.where(e > -127, (e + 127).int() << 23, 1 << 22).to(torch.int32).view(torch.float32)


def _blocks(x, block):
    """x [..., c] as fp32 [..., blocks, block], zero behind the columns."""
    v = torch.zeros(x.shape[:-1] + (_up(x.shape[-1], block),), dtype=torch.float32, device=x.device)
    v[..., : x.shape[-1]] = x
    return v.view(x.shape[:-1] + (-1, block))


def _fp4(x):
    """x [..., c] -> codes (0 to 15) [..., c up to a multiple of 32], scale bytes [..., blocks of 32].

    The byte of a block is the smallest b >= 0 with amax <= 6 * 2^(b - 127); a block that holds a NaN or an infinity has 255 and
    zeros.  Values divided by 2^(b - 127) are rounded once, to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6, ties to the even code."""
    v = _blocks(x, 32)
    fine = torch.isfinite(v).all(-1)
    v = torch.where(fine[..., None], v, 0.0)
    frac, exp = torch.frexp(v.abs().amax(-1))  # amax = frac * 2^exp, 6 = 0.75 * 2^3
    b = (exp - 3 + (frac > 0.75) + 127).clamp(min=0)
    a = v.abs() * _two_to(127 - b)[..., None]
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    code = code + 8 * torch.signbit(v)
    return code.view(code.shape[:-2] + (-1,)), torch.where(fine, b, 255).to(torch.uint8)


def _fp4_value(code, b):
    """fp32 values of codes [..., c] and scale bytes [..., blocks of 32]."""
    levels = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=code.device)
    levels = torch.cat([levels, -levels])
    scale = torch.where(b < 255, _two_to(b.int() - 127), float("nan"))
    return (levels[code.long()].view(b.shape + (32,)) * scale[..., None]).view(code.shape)


def _fp8_value(x):
    """fp32 values of the 8-bit form of x [R, c]: e4m3 with the smallest power of two that holds a block of 128."""
    v = _blocks(x, 128)
    fine = torch.isfinite(v)
    frac, exp = torch.frexp(torch.where(fine, v, 0.0).abs().amax(-1))  # 448 = 0.875 * 2^9
    b = (exp - 9 + (frac > 0.875) + 127).clamp(min=0)
    q = torch.where(fine, v * _two_to(127 - b)[..., None], float("nan")).to(torch.float8_e4m3fn).float()
    return (q * _two_to(b - 127)[..., None]).view(v.shape[0], -1)[:, : x.shape[1]]


def _value4(x):
    """fp32 values of the 4-bit form of x [R, c]."""
    return _fp4_value(*_fp4(x))[..., : x.shape[-1]]


def _pack(code, b, rows):
    """The layout of a 4-bit matrix [..., n, c] with `rows` rows: bytes [..., rows, pitch], scales [..., rows, scale pitch]."""
    lead, n = code.shape[:-2], code.shape[-2]
    full = torch.zeros(lead + (rows, _up(code.shape[-1], 256)), dtype=torch.uint8, device=code.device)
    full[..., :n, : code.shape[-1]] = code
    scale = torch.zeros(lead + (rows, _up(b.shape[-1], 16)), dtype=torch.uint8, device=code.device)
    scale[..., :n, : b.shape[-1]] = b
    scale = scale.view(lead + (rows, -1, 4, 4)).transpose(-1, -2).reshape(scale.shape)
    return full[..., 0::2] | full[..., 1::2] << 4, scale


def _unpack(q, scale):
    """Codes [..., rows, columns up to a multiple of 256] and scale bytes of a 4-bit matrix."""
    code = torch.stack([q & 15, q >> 4], dim=-1).view(q.shape[:-1] + (-1,))
    b = scale.view(scale.shape[:-1] + (-1, 4, 4)).transpose(-1, -2).reshape(scale.shape)
    return code, b[..., : code.shape[-1] // 32]


def _matrix(q, scale):
    """fp32 values of a 4-bit matrix, with the columns that fill it up."""
    return _fp4_value(*_unpack(q, scale))


def _by_expert(x, s):
    """Rows of x as [E, most rows of an expert, k], zero behind an expert's rows."""
    out = torch.zeros((s["experts"], s["most"], x.shape[1]), dtype=torch.float32, device=x.device)
    out[s["row_expert"], s["row_place"]] = x
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(shape, std, dtype):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)

    def stream(r, c):
        """activations: a row's values are of one size, rows differ, and a few channels stand out"""
        x = normal((r, c), 1.0, torch.float32)
        x *= torch.exp(normal((r, 1), 1.0, torch.float32))
        x[:, torch.randint(0, c, (max(1, c // 256),), generator=gen, device="cuda")] *= 20.0
        return x.to(DTYPES[case["dtype"]])

    def experts(e, n, k, std):
        """4-bit weights of a layer, quantised once as at model load (a few experts at a time: memory)."""
        step = max(1, (1 << 27) // (n * k))
        parts = [_pack(*_fp4(normal((min(step, e - i), n, k), std, torch.bfloat16)), _up(n, 128)) for i in range(0, e, step)]
        return torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])

    def four(r, c):
        return (torch.zeros((r, _up(c, 256) // 2), dtype=torch.uint8, device="cuda"),
                torch.zeros((r, _up(c, 512) // 32), dtype=torch.uint8, device="cuda"))

    s = {"case": dict(case)}
    op = case["op"]
    if op == "norm":
        r, c, dtype = case["rows"], case["cols"], DTYPES[case["dtype"]]
        s["x"] = normal((r, c), 1.0, dtype) if case["residual"] else stream(r, c)
        s["residual"] = stream(r, c) if case["residual"] else None
        s["weight"] = (1.0 + 0.2 * normal((c,), 1.0, torch.float32)).to(dtype)
        s["eps"] = 1e-6
        s["sum"] = torch.zeros((r, c), dtype=dtype, device="cuda") if case["residual"] else None
        s["y"] = torch.zeros((r, c), dtype=dtype, device="cuda") if case["y"] else None
        s["q"], s["scale"] = None, None
        if case["bits"] == 8:
            s["q"] = torch.zeros((r, _up(c, 128)), dtype=torch.uint8, device="cuda")
            s["scale"] = torch.zeros((r, 4 * -(-c // 512)), dtype=torch.uint8, device="cuda")
        elif case["bits"] == 4:
            s["q"], s["scale"] = four(r, c)
        s["values"] = torch.zeros((r, c), dtype=torch.bfloat16, device="cuda") if case["bits"] else None
        return s
    if op == "rows":
        r, c, t = case["rows"], case["cols"], case["tokens"]
        s["x"] = stream(t or r, c)
        s["row_token"] = torch.randint(0, t, (r,), generator=gen, device="cuda", dtype=torch.int32) if t else None
        s["q"], s["scale"] = four(r, c)
        s["values"] = torch.zeros((r, c), dtype=torch.bfloat16, device="cuda")
        return s
    if op == "weights":
        e, n, k = case["experts"], case["n_out"], case["n_in"]
        s["w"] = normal((e, n, k), k ** -0.5, DTYPES[case["dtype"]])
        q, scale = four(e * _up(n, 128), k)
        s["q"], s["scale"] = q.view(e, _up(n, 128), -1), scale.view(e, _up(n, 128), -1)
        s["values"] = torch.zeros((e, _up(n, 128), k), dtype=torch.bfloat16, device="cuda")
        return s
    e, t = case["experts"], case["tokens"]
    counts = torch.tensor(_counts(case))[torch.randperm(e, generator=gen, device="cuda").cpu()]
    # every expert takes that many of the tokens, ascending
    rank = torch.rand((e, t), generator=gen, device="cuda").argsort(dim=1).argsort(dim=1)
    expert, token = torch.nonzero(rank < counts.cuda()[:, None], as_tuple=True)
    s["experts"], s["most"], s["rows"] = e, int(counts.max()), int(counts.sum())
    ends = torch.cumsum(counts, 0)
    s["expert_offset"] = torch.cat([torch.zeros(1, dtype=torch.int64), ends]).to(torch.int32).cuda()
    s["row_expert"], s["row_place"] = expert, torch.arange(s["rows"], device="cuda") - (ends - counts).cuda()[expert]
    s["row_token"] = token.to(torch.int32)
    d, h = case["n_in"], case["n_out"]
    if op == "gemm":
        r = t if case["gather"] else s["rows"]
        s["xq"], s["xs"] = _pack(*_fp4(normal((r, d), 1.0, torch.bfloat16)), r)
        s["w"] = experts(e, h, d, d ** -0.5)
        s["y"] = torch.zeros((s["rows"], h), dtype=torch.bfloat16, device="cuda")
    else:
        s["x"], s["xs"] = normal((t, d), 1.0, torch.bfloat16), None
        if case["small_rows"]:
            s["x"], s["xs"] = _pack(*_fp4(s["x"]), t)
        s["gate"], s["up"], s["down"] = experts(e, h, d, d ** -0.5), experts(e, h, d, d ** -0.5), experts(e, d, h, h ** -0.5)
        # the plan's arrays and the output hold the most rows that the layer may have
        s["row_token"] = torch.zeros((t * case["top_k"],), dtype=torch.int32, device="cuda")
        s["row_token"][: s["rows"]] = token
        s["y"] = torch.zeros((t * case["top_k"], d), dtype=torch.bfloat16, device="cuda")
    return s


def _plain(s):
    case = s["case"]
    if case["op"] == "norm":
        dtype = DTYPES[case["dtype"]]
        h = s["x"].float()
        if case["residual"]:
            h = (h + s["residual"].float()).to(dtype).float()
        y = (h * torch.rsqrt((h * h).mean(dim=1, keepdim=True) + s["eps"]) * s["weight"].float()).to(dtype)
        values = {0: lambda v: None, 4: _value4, 8: _fp8_value}[case["bits"]](y)
        return (h.to(dtype) if case["residual"] else None, y if case["y"] else None,
                None if values is None else values.to(torch.bfloat16))
    if case["op"] == "rows":
        return _value4(s["x"] if s["row_token"] is None else s["x"][s["row_token"].long()]).to(torch.bfloat16)
    if case["op"] == "weights":
        s["values"][:, : case["n_out"]] = _value4(s["w"])
        return s["values"]
    token = s["row_token"][: s["rows"]].long()
    if case["op"] == "gemm":
        x = _matrix(s["xq"], s["xs"])
        x = _by_expert(x[token] if case["gather"] else x, s)
        y = torch.bmm(x, _matrix(*s["w"]).transpose(1, 2))[s["row_expert"], s["row_place"], : case["n_out"]]
        s["y"].copy_(y)
        return s["y"]
    x = _matrix(s["x"], s["xs"]) if case["small_rows"] else _fp4_value(*_fp4(s["x"]))
    x = _by_expert(x[token], s)
    gate, up = (torch.bmm(x, _matrix(*s[name])[..., : x.shape[2]].transpose(1, 2)) for name in ("gate", "up"))
    hidden = (gate / (1.0 + torch.exp(-gate)) * up).to(torch.bfloat16)  # rounded to bf16, then to 4 bits
    hidden = _fp4_value(*_fp4(hidden))
    y = torch.bmm(hidden, _matrix(*s["down"])[..., : hidden.shape[2]].transpose(1, 2))
    s["y"][: s["rows"]] = y[s["row_expert"], s["row_place"], : case["n_in"]].to(torch.bfloat16)
    return s["y"]


def run(s):
    if not own:
        return _plain(s)
    from paper_2503_05066_amd import capmoe

    case = s["case"]
    if case["op"] == "norm":
        if "norm" not in s:  # what a program sets up once
            s["norm"] = capmoe.make_norm(case["rows"], case["cols"], s["eps"], bits=case["bits"],
                                         dtype=capmoe.DTYPE_BF16 if case["dtype"] == "bf16" else capmoe.DTYPE_F32)
        capmoe.moe_norm_rows(s["norm"], s["x"], s["residual"], s["weight"], None, s["sum"], s["y"], s["q"], s["scale"])
        if case["bits"]:
            capmoe.moe_dequantize_rows(case["bits"], s["q"], s["scale"], s["values"])
        return s["sum"], s["y"], s["values"]
    if case["op"] == "rows":
        capmoe.moe_quantize_rows_fp4(s["x"], s["row_token"], None, s["q"], s["scale"])
        capmoe.moe_dequantize_rows(4, s["q"], s["scale"], s["values"])
        return s["values"]
    if case["op"] == "weights":
        capmoe.moe_quantize_weights_fp4(s["w"], s["q"], s["scale"])
        capmoe.moe_dequantize_rows(4, s["q"].flatten(0, 1), s["scale"].flatten(0, 1), s["values"].flatten(0, 1))
        return s["values"]
    if case["op"] == "gemm":
        if "gemm" not in s:
            s["gemm"] = capmoe.make_gemm(s["rows"], case["n_in"], case["n_out"], case["experts"],
                                         src_rows=case["tokens"] if case["gather"] else 0)
        capmoe.moe_grouped_gemm_fp4(s["gemm"], s["xq"], s["xs"], s["row_token"] if case["gather"] else None,
                                    s["expert_offset"], s["w"][0], s["w"][1], s["y"])
        return s["y"]
    if "desc" not in s:
        s["desc"] = capmoe.make_desc(case["tokens"], case["n_in"], case["experts"], case["top_k"], case["n_out"],
                                     mode=capmoe.MODE_NONE)
        s["weights"] = capmoe.Fp4Experts(*s["gate"], *s["up"], *s["down"])
        s["workspace"] = torch.empty(capmoe.moe_query_fp4(s["desc"]), dtype=torch.uint8, device="cuda")
    capmoe.moe_dispatch_ffn_fp4(s["desc"], s["x"], s["xs"], s["expert_offset"], s["row_token"], s["weights"], s["y"], s["workspace"])
    return s["y"]


def work(case):
    if case["op"] in ("norm", "rows", "weights"):
        elem = 2 if case["dtype"] == "bf16" else 4
        if case["op"] == "norm":
            n = case["rows"] * case["cols"]
            bits = {0: 0.0, 4: 4.25, 8: 8.0625}[case["bits"]]
            moved = elem * (1 + 2 * case["residual"] + case["y"]) + bits / 8 + (2 if bits else 0)
            return {"bytes": n * moved + case["cols"] * elem, "flops": 0}
        if case["op"] == "rows":
            r, c = case["rows"], case["cols"]
            return {"bytes": min(r, case["tokens"] or r) * c * elem + r * c * (4.25 / 8 + 2), "flops": 0}
        n = case["experts"] * case["n_out"] * case["n_in"]
        return {"bytes": n * (elem + 4.25 / 8 + 2), "flops": 0}
    counts = _counts(case)
    rows, active = sum(counts), sum(c > 0 for c in counts)
    d, h, t = case["n_in"], case["n_out"], case["tokens"]
    four = 4.25 / 8  # bytes of a value and its share of a scale
    if case["op"] == "gemm":
        return {"bytes": active * d * h * four + (min(rows, t) if case["gather"] else rows) * d * four + rows * h * 2,
                "flops": 2 * rows * d * h}
    return {"bytes": 3 * active * d * h * four + min(rows, t) * d * (four if case["small_rows"] else 2) + rows * d * 2,
            "flops": 6 * rows * d * h}


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------
def _power(e):
    """2^e in 64 bits, e whole numbers."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _nearest(v, bits, lowest):
    """v rounded to a float with `bits` bits behind the leading one, whose smallest normal is 2^lowest; ties to even."""
    _, exp = torch.frexp(v)
    step = _power((exp - 1).clamp(min=lowest) - bits)
    return torch.round(v / step) * step


_FORMATS = {4: (32, 6.0, 1, 0), 8: (128, 448.0, 3, -6)}  # block, largest value, bits, lowest


def _exact_form(v, bits):
    """The values that the 4- or 8-bit form of v [..., c] (64 bits, finite) stands for."""
    block, top, mantissa, lowest = _FORMATS[bits]
    c = v.shape[-1]
    v = torch.nn.functional.pad(v, (0, _up(c, block) - c)).unflatten(-1, (-1, block))
    amax = v.abs().amax(dim=-1, keepdim=True)
    exp = torch.ceil(torch.log2(amax / top)).clamp(min=-127.0)
    exp = torch.where(amax <= top * _power(exp - 1), exp - 1, exp).clamp(min=-127.0)  # where the logarithm was rounded up
    exp = torch.where(amax > top * _power(exp), exp + 1, exp)
    return (_nearest(v / _power(exp), mantissa, lowest) * _power(exp)).flatten(-2)[..., :c]


def exact(case, seed):
    s = prepare(case, seed)
    levels = torch.tensor([0, 1, 2, 3, 4, 6, 8, 12], dtype=torch.float64, device="cuda") / 2
    levels = torch.cat([levels, -levels])

    def matrix(q, scale):
        """4-bit rows [n, pitch] as 64-bit values"""
        block = torch.arange(q.shape[-1] // 16, device="cuda")
        at = block // 16 * 16 + block % 4 * 4 + block % 16 // 4
        power = _power(scale.long()[:, at] - 127).repeat_interleave(32, 1)
        return torch.stack([levels[(q & 15).long()], levels[(q >> 4).long()]], dim=2).flatten(1) * power

    if case["op"] == "norm":
        bits = (7, -126) if case["dtype"] == "bf16" else (23, -126)
        h = s["x"].double()
        if case["residual"]:
            h = _nearest(h + s["residual"].double(), *bits)
        y = h / torch.sqrt((h ** 2).mean(dim=1, keepdim=True) + s["eps"]) * s["weight"].double()
        return (h if case["residual"] else None, y if case["y"] else None,
                _exact_form(_nearest(y, *bits), case["bits"]) if case["bits"] else None)
    if case["op"] == "rows":
        x = s["x"] if s["row_token"] is None else s["x"][s["row_token"].long()]
        return _exact_form(x.double(), 4) if x.numel() <= 1 << 27 else None
    if case["op"] == "weights":
        y = torch.zeros(s["values"].shape, dtype=torch.float64, device="cuda")
        y[:, : case["n_out"]] = _exact_form(s["w"].double(), 4)
        return y
    offset, token = s["expert_offset"].tolist(), s["row_token"][: s["rows"]].long()
    y = torch.zeros(s["y"].shape, dtype=torch.float64, device="cuda")
    if case["op"] == "gemm":
        x = matrix(s["xq"], s["xs"])
    else:
        x = matrix(s["x"], s["xs"]) if case["small_rows"] else _exact_form(s["x"].double(), 4)
    for i in range(case["experts"]):
        lo, hi = offset[i], offset[i + 1]
        if lo == hi:
            continue
        if case["op"] == "gemm":
            w = matrix(s["w"][0][i], s["w"][1][i])
            y[lo:hi] = ((x[token[lo:hi]] if case["gather"] else x[lo:hi]) @ w.T)[:, : case["n_out"]]
            continue
        xe = x[token[lo:hi], : case["n_in"]]
        gate, up = (xe @ matrix(s[name][0][i], s[name][1][i])[: case["n_out"], : case["n_in"]].T for name in ("gate", "up"))
        hidden = _exact_form(_nearest(gate * up / (1.0 + torch.exp(-gate)), 7, -126), 4)
        y[lo:hi] = (hidden @ matrix(s["down"][0][i], s["down"][1][i])[: case["n_in"], : case["n_out"]].T)
    return y
