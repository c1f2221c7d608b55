"""The operators of 8-bit experts, as timed cases.

A case names one operator:

  "rows"     moe_quantize_rows: activations to e4m3 with a power-of-two scale per row and 128 columns, with or without the
             permutation into expert-major order
  "weights"  moe_quantize_weights: expert weights to e4m3 with a power-of-two scale per 128 x 128 block (model load)
  "gemm"     moe_grouped_gemm_fp8: the product of 8-bit rows, grouped by expert with ragged sizes, and 8-bit weights
  "ffn"      moe_dispatch_ffn_fp8: the SwiGLU expert FFN on 8-bit weights, from bf16 tokens to bf16 expert outputs

Sizes are those of the workloads in paper_2503_05066_amd/synth.py, of the tests and of bench.py, with ragged ones of the
same families between them.  An 8-bit matrix of c columns has rows of 128 * ceil(c / 128) bytes, zero behind the columns,
and 4 * ceil(c / 512) scale bytes per row (per 128 rows for weights, whose rows are filled up to a multiple of 128 too);
scale byte b stands for 2^(b - 127).
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BLOCK = 128


def _up(n, m):
    return -(-n // m) * m


def _rows_case(name, dtype, rows, cols, tokens=0):
    return {"name": name, "op": "rows", "dtype": dtype, "rows": rows, "cols": cols, "tokens": tokens}


def _weights_case(name, dtype, e, n_out, n_in):
    return {"name": name, "op": "weights", "dtype": dtype, "experts": e, "n_out": n_out, "n_in": n_in}


def _gemm_case(name, tokens, e, k, n_in, n_out, gather=False, gamma=0.0, skew="normal", skew_param=1.0):
    return {"name": name, "op": "gemm", "tokens": tokens, "experts": e, "top_k": k, "n_in": n_in,
            "n_out": n_out, "gather": gather, "gamma": gamma, "skew": skew, "skew_param": skew_param}


def _ffn_case(name, tokens, d, e, k, h, gamma=0.0, skew="normal", skew_param=1.0):
    return {"name": name, "op": "ffn", "tokens": tokens, "experts": e, "top_k": k, "n_in": d, "n_out": h,
            "gamma": gamma, "skew": skew, "skew_param": skew_param}


def listed():
    return [
        # the activations of a small decoding batch: latency
        _rows_case("rows_37_decode", "bf16", 37, 4096),
        # a prompt batch permuted into expert-major order on the way: 13 k kept pairs of 4096 tokens
        _rows_case("rows_13000_permuted", "bf16", 13000, 2048, tokens=4096),
        # loading a layer of many small experts
        _weights_case("weights_64_experts", "bf16", 64, 1024, 2048),
        # loading fp32 experts whose sizes divide nothing
        _weights_case("weights_f32_odd", "f32", 7, 1000, 1416),
        # one projection of a single token's eight experts: latency and the weight stream
        _gemm_case("gemm_1_token", 1, 64, 8, 2048, 1024, skew="zipf", skew_param=1.1),
        # an expert that all tokens share (a dense product) in a decoding batch, sizes that are no multiples of 128
        _gemm_case("gemm_shared_odd", 203, 1, 1, 2056, 5640),
        # one projection of a skewed prompt batch, rows fetched through the plan
        _gemm_case("gemm_4096_ragged", 4096, 64, 8, 2048, 1024, gather=True, gamma=1.0, skew="zipf", skew_param=1.1),
        # few wide experts, long sums: the matrix cores bind
        _gemm_case("gemm_8192_wide", 8192, 8, 2, 14336, 4096, gamma=1.0, skew_param=1.5),
        # decoding a small batch with few, wide experts: streams nearly all weights for sixteen tokens
        _ffn_case("ffn_16_wide", 16, 4096, 8, 2, 14336, skew_param=0.5),
        # a short ragged prompt on a layer whose counts divide nothing
        _ffn_case("ffn_1531_odd", 1531, 2048, 60, 4, 1408, gamma=1.25, skew="zipf", skew_param=1.0),
        # an ordinary prompt batch, skewed routing under a capacity
        _ffn_case("ffn_4096", 4096, 2048, 64, 8, 1024, gamma=1.0, skew="zipf", skew_param=1.1),
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
    op = rng.choice(["rows", "weights", "gemm", "gemm", "ffn", "ffn"])
    while True:
        dtype = rng.choice(["bf16", "bf16", "f32"])
        e = rng.choice([1, 4, 8, 16, 32, 60, 64, 96, 128])
        if op == "rows":
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
                c = _ffn_case("", n, a, e, k, b, gamma, skew, param)
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


def _scale_bytes(amax):
    """The smallest b >= 0 with amax <= 448 * 2^(b - 127)."""
    frac, exp = torch.frexp(amax)  # amax = frac * 2^exp, 448 = 0.875 * 2^9
    return (exp - 9 + (frac > 0.875) + 127).clamp(min=0)


def _two_to(e):
    """2^e, e whole numbers of at least -127, exactly."""
    return torch.where(e > -127, (e + 127).int() << 23, 1 << 22).to(torch.int32).view(torch.float32)


def _e4m3(v):
    """fp32 values of magnitude up to 448 (or NaN), rounded."""
    return v.to(torch.float8_e4m3fn)


def _pad(x, rows, cols):
    out = torch.zeros(x.shape[:-2] + (rows, cols), dtype=torch.float32, device=x.device)
    out[..., : x.shape[-2], : x.shape[-1]] = x
    return out


def _quantize_rows(x):
    """x [R, c] -> e4m3 [R, pitch], scale bytes [R, scale pitch]; NaN and infinities become NaN and do not count for the scale."""
    r, c = x.shape
    v = _pad(x, r, _up(c, BLOCK)).view(r, -1, BLOCK)
    fine = torch.isfinite(v)
    b = _scale_bytes(torch.where(fine, v, 0.0).abs().amax(-1))
    q = torch.where(fine, v * _two_to(127 - b)[..., None], float("nan"))
    s = torch.zeros((r, 4 * -(-c // 512)), dtype=torch.uint8, device=x.device)
    s[:, : b.shape[1]] = b.to(torch.uint8)
    return _e4m3(q).view(r, -1), s


def _quantize_weights(w):
    """w [E, n, k] -> e4m3 [E, n up to a multiple of 128, pitch], scale bytes [E, blocks of n, scale pitch]."""
    e, n, k = w.shape
    nb, kb = -(-n // BLOCK), -(-k // BLOCK)
    v = _pad(w, nb * BLOCK, kb * BLOCK).view(e, nb, BLOCK, kb, BLOCK)
    fine = torch.isfinite(v)
    b = _scale_bytes(torch.where(fine, v, 0.0).abs().amax(dim=(2, 4)))
    q = torch.where(fine, v * _two_to(127 - b)[:, :, None, :, None], float("nan"))
    s = torch.zeros((e, nb, 4 * -(-k // 512)), dtype=torch.uint8, device=w.device)
    s[:, :, :kb] = b.to(torch.uint8)
    return _e4m3(q).view(e, nb * BLOCK, kb * BLOCK), s


def _rows_value(q, s):
    kb = q.shape[-1] // BLOCK
    scale = _two_to(s[..., :kb].int() - 127)
    return (q.float().view(q.shape[:-1] + (kb, BLOCK)) * scale[..., None]).view(q.shape)


def _weights_value(q, s):
    e, n, k = q.shape
    scale = _two_to(s[..., : k // BLOCK].int() - 127)
    return (q.float().view(e, n // BLOCK, BLOCK, k // BLOCK, BLOCK) * scale[:, :, None, :, None]).view(e, n, k)


def _by_expert(x, s):
    """Rows of x as [E, most rows of an expert, k], zero behind an expert's rows."""
    out = torch.zeros((s["experts"], s["most"], x.shape[1]), dtype=torch.float32, device=x.device)
    out[s["row_expert"], s["row_place"]] = x
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(shape, std, dtype):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)

    def experts(e, n, k, std):
        """8-bit weights of a layer, quantised once as at model load (a few experts at a time: memory)."""
        step = max(1, (1 << 28) // (n * k))
        parts = [_quantize_weights(normal((min(step, e - i), n, k), std, torch.bfloat16)) for i in range(0, e, step)]
        return torch.cat([p[0].view(torch.uint8) for p in parts]), torch.cat([p[1] for p in parts])

    s = {"case": dict(case)}
    op = case["op"]
    if op == "rows":
        r, c, t = case["rows"], case["cols"], case["tokens"]
        # activations behind a norm: a row's values are of one size, rows differ, and a few channels stand out
        s["x"] = normal((t or r, c), 1.0, torch.float32)
        s["x"] *= torch.exp(normal((t or r, 1), 1.0, torch.float32))
        s["x"][:, torch.randint(0, c, (max(1, c // 256),), generator=gen, device="cuda")] *= 20.0
        s["x"] = s["x"].to(DTYPES[case["dtype"]])
        s["row_token"] = torch.randint(0, t, (r,), generator=gen, device="cuda", dtype=torch.int32) if t else None
        s["q"] = torch.zeros((r, _up(c, BLOCK)), dtype=torch.uint8, device="cuda")
        s["scale"] = torch.zeros((r, 4 * -(-c // 512)), dtype=torch.uint8, device="cuda")
        return s
    if op == "weights":
        e, n, k = case["experts"], case["n_out"], case["n_in"]
        s["w"] = normal((e, n, k), k ** -0.5, DTYPES[case["dtype"]])
        s["q"] = torch.zeros((e, _up(n, BLOCK), _up(k, BLOCK)), dtype=torch.uint8, device="cuda")
        s["scale"] = torch.zeros((e, -(-n // BLOCK), 4 * -(-k // 512)), dtype=torch.uint8, device="cuda")
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
        x = normal((t if case["gather"] else s["rows"], d), 1.0, torch.bfloat16)
        s["xq"], s["xs"] = (v.view(torch.uint8) for v in _quantize_rows(x))
        s["w"] = experts(e, h, d, d ** -0.5)
        s["y"] = torch.zeros((s["rows"], h), dtype=torch.bfloat16, device="cuda")
    else:
        s["x"] = normal((t, d), 1.0, torch.bfloat16)
        s["gate"], s["up"], s["down"] = experts(e, h, d, d ** -0.5), experts(e, h, d, d ** -0.5), experts(e, d, h, h ** -0.5)
        # the plan's arrays and the output hold the most rows that the layer may have
        s["row_token"] = torch.zeros((t * case["top_k"],), dtype=torch.int32, device="cuda")
        s["row_token"][: s["rows"]] = token
        s["y"] = torch.zeros((t * case["top_k"], d), dtype=torch.bfloat16, device="cuda")
    return s


def _plain(s):
    case = s["case"]
    f8 = torch.float8_e4m3fn
    if case["op"] == "rows":
        return _quantize_rows(s["x"] if s["row_token"] is None else s["x"][s["row_token"].long()])
    if case["op"] == "weights":
        return _quantize_weights(s["w"])
    token = s["row_token"][: s["rows"]].long()
    if case["op"] == "gemm":
        x = _rows_value(s["xq"].view(f8), s["xs"])
        x = _by_expert(x[token] if case["gather"] else x, s)
        w = _weights_value(s["w"][0].view(f8), s["w"][1])
        y = torch.bmm(x, w.transpose(1, 2))[s["row_expert"], s["row_place"], : case["n_out"]]
        s["y"].copy_(y)
        return s["y"]
    x = _by_expert(_rows_value(*_quantize_rows(s["x"]))[token], s)
    gate = torch.bmm(x, _weights_value(s["gate"][0].view(f8), s["gate"][1]).transpose(1, 2))
    up = torch.bmm(x, _weights_value(s["up"][0].view(f8), s["up"][1]).transpose(1, 2))
    hidden = (gate / (1.0 + torch.exp(-gate)) * up).to(torch.bfloat16)  # rounded to bf16, then to 8 bits
    q, qs = _quantize_rows(hidden.view(-1, hidden.shape[2]))
    hidden = _rows_value(q, qs).view(hidden.shape)
    y = torch.bmm(hidden, _weights_value(s["down"][0].view(f8), s["down"][1]).transpose(1, 2))
    s["y"][: s["rows"]] = y[s["row_expert"], s["row_place"], : case["n_in"]].to(torch.bfloat16)
    return s["y"]


def run(s):
    if not own:
        return _plain(s)
    from paper_2503_05066_amd import capmoe

    case = s["case"]
    if case["op"] == "rows":
        capmoe.moe_quantize_rows(s["x"], s["row_token"], None, s["q"], s["scale"])
        return s["q"].view(torch.float8_e4m3fn), s["scale"]
    if case["op"] == "weights":
        capmoe.moe_quantize_weights(s["w"], s["q"], s["scale"])
        return s["q"].view(torch.float8_e4m3fn), s["scale"]
    if case["op"] == "gemm":
        if "gemm" not in s:  # what a program sets up once
            s["gemm"] = capmoe.make_gemm(s["rows"], case["n_in"], case["n_out"], case["experts"],
                                         src_rows=case["tokens"] if case["gather"] else 0)
            s["workspace"] = torch.empty(capmoe.moe_gemm_query(s["gemm"]), dtype=torch.uint8, device="cuda")
        capmoe.moe_grouped_gemm_fp8(s["gemm"], s["xq"], s["xs"], s["row_token"] if case["gather"] else None,
                                    s["expert_offset"], s["w"][0], s["w"][1], s["y"], s["workspace"])
        return s["y"]
    if "desc" not in s:
        s["desc"] = capmoe.make_desc(case["tokens"], case["n_in"], case["experts"], case["top_k"], case["n_out"],
                                     mode=capmoe.MODE_NONE)
        s["weights"] = capmoe.Fp8Experts(*s["gate"], *s["up"], *s["down"])
        s["workspace"] = torch.empty(capmoe.moe_query_fp8(s["desc"]), dtype=torch.uint8, device="cuda")
    capmoe.moe_dispatch_ffn_fp8(s["desc"], s["x"], s["expert_offset"], s["row_token"], s["weights"], s["y"], s["workspace"])
    return s["y"]


def work(case):
    if case["op"] == "rows":
        r, c = case["rows"], case["cols"]
        elem = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": min(r, case["tokens"] or r) * c * elem + r * (c + c // BLOCK), "flops": 0}
    if case["op"] == "weights":
        n = case["experts"] * case["n_out"] * case["n_in"]
        return {"bytes": n * (3 if case["dtype"] == "bf16" else 5) + n // BLOCK ** 2, "flops": 0}
    counts = _counts(case)
    rows, active = sum(counts), sum(c > 0 for c in counts)
    d, h, t = case["n_in"], case["n_out"], case["tokens"]
    if case["op"] == "gemm":
        return {"bytes": active * d * h + (min(rows, t) if case["gather"] else rows) * d + rows * h * 2, "flops": 2 * rows * d * h}
    return {"bytes": 3 * active * d * h + min(rows, t) * d * 2 + rows * d * 2, "flops": 6 * rows * d * h}


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


def _exact_blocks(v, dims):
    """(e4m3 values, scales' exponents) of 64-bit values whose blocks lie along dims."""
    fine = torch.isfinite(v)
    amax = torch.where(fine, v, 0.0).abs().amax(dim=dims, keepdim=True)
    exp = torch.ceil(torch.log2(amax / 448.0)).clamp(min=-127.0)
    exp = torch.where(amax <= 448.0 * _power(exp - 1), exp - 1, exp).clamp(min=-127.0)  # where the logarithm was rounded up
    exp = torch.where(amax > 448.0 * _power(exp), exp + 1, exp)
    return torch.where(fine, _nearest(v / _power(exp), 3, -6), float("nan")), exp


def _exact_rows(x):
    r, c = x.shape
    v = torch.zeros((r, _up(c, BLOCK)), dtype=torch.float64, device=x.device)
    v[:, :c] = x
    q, exp = _exact_blocks(v.view(r, -1, BLOCK), (2,))
    return q, exp


def exact(case, seed):
    s = prepare(case, seed)
    f8 = torch.float8_e4m3fn
    if case["op"] == "rows":
        x = s["x"] if s["row_token"] is None else s["x"][s["row_token"].long()]
        if x.numel() > 1 << 26:
            return None
        q, exp = _exact_rows(x)
        scale = torch.zeros_like(s["scale"])
        scale[:, : exp.shape[1]] = (exp[..., 0] + 127).to(torch.uint8)
        return q.reshape(s["q"].shape), scale
    if case["op"] == "weights":
        e, n, k = s["w"].shape
        q = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        q[:, :n, :k] = s["w"]
        q, exp = _exact_blocks(q.view(e, -1, BLOCK, q.shape[2] // BLOCK, BLOCK), (2, 4))
        scale = torch.zeros_like(s["scale"])
        scale[:, :, : exp.shape[3]] = (exp[:, :, 0, :, 0] + 127).to(torch.uint8)
        return q.reshape(s["q"].shape), scale

    def expert(w, i):
        q, b = w
        scale = _power(b[i].long() - 127)[:, : q.shape[2] // BLOCK]
        return q[i].view(f8).double() * scale.repeat_interleave(BLOCK, 0).repeat_interleave(BLOCK, 1)

    offset, token = s["expert_offset"].tolist(), s["row_token"][: s["rows"]].long()
    y = torch.zeros(s["y"].shape, dtype=torch.float64, device="cuda")
    if case["op"] == "gemm":
        x = s["xq"].view(f8).double()
        x = x * _power(s["xs"].long() - 127)[:, : x.shape[1] // BLOCK].repeat_interleave(BLOCK, 1)
    else:
        q, exp = _exact_rows(s["x"].double())
        x = (q * _power(exp)).reshape(case["tokens"], -1)
    for i in range(case["experts"]):
        lo, hi = offset[i], offset[i + 1]
        if lo == hi:
            continue
        if case["op"] == "gemm":
            y[lo:hi] = ((x[token[lo:hi]] if case["gather"] else x[lo:hi]) @ expert(s["w"], i).T)[:, : case["n_out"]]
            continue
        xe = x[token[lo:hi]]
        gate, up = xe @ expert(s["gate"], i).T, xe @ expert(s["up"], i).T
        hidden = _nearest(gate * up / (1.0 + torch.exp(-gate)), 7, -126)
        q, exp = _exact_rows(hidden)
        y[lo:hi] = ((q * _power(exp)).reshape(hi - lo, -1) @ expert(s["down"], i).T)[:, : case["n_in"]]
    return y
