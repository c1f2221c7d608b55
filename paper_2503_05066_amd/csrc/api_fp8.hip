// The entry points of the 8-bit experts: argument validation, workspace layout, the calls' launches.
#include <algorithm>

#include "fp8.h"

namespace capmoe {

// Workspace of a layer's FFN.  (A product by itself needs none.)
struct Fp8Workspace {
    void* hidden;           // [P_max, h filled up] bf16, or 8-bit values and behind them their scales
    uint8_t* hidden_scale;
    void* xq;               // [rows of x, pitch]
    uint8_t* xs;
    size_t bytes;
};

static Fp8Workspace ffn_fp8_workspace(const moe_desc_t& d, const Sizes& s, void* base) {
    Fp8Workspace w;
    char* p = (char*)base;
    size_t off = 0;
    const int64_t rows = std::max<int64_t>(s.max_rows, 1);
    const size_t hidden = align256((size_t)rows * fp8_pitch(d.d_hidden));
    w.hidden = p;
    w.hidden_scale = (uint8_t*)(p + hidden);
    off += 2 * hidden;
    static_assert(kFp8Block >= 4, "a row's scale bytes fit where its second byte per value would be");
    const int64_t x_rows = std::max<int64_t>(rows, d.n_tokens);
    w.xq = p + off;
    off += align256((size_t)x_rows * fp8_pitch(d.d_model));
    w.xs = (uint8_t*)(p + off);
    off += align256((size_t)x_rows * fp8_scale_pitch(d.d_model));
    w.bytes = off;
    return w;
}

static int validate_gemm(const moe_gemm_t* g) {
    if (!g || g->max_rows < 0 || g->src_rows < 0 || g->n_experts < 1 || g->n_in < 1 || g->n_out < 1) return MOE_ERR_INVALID_ARG;
    if (g->n_experts > kMaxExperts || g->n_in > kFp8MaxWidth || g->n_out > kFp8MaxWidth || g->n_out % 8 != 0) return MOE_ERR_UNSUPPORTED;
    return MOE_OK;
}

static bool misaligned16(const void* p) { return ((uintptr_t)p & 15) != 0; }
static bool misaligned4(const void* p) { return ((uintptr_t)p & 3) != 0; }

static int validate_fp8(const moe_desc_t* d) {
    const int v = validate(d);
    if (v != MOE_OK) return v;
    if (d->dtype != MOE_DTYPE_BF16 || d->d_model > kFp8MaxWidth || d->d_hidden > kFp8MaxWidth) return MOE_ERR_UNSUPPORTED;
    const int64_t rows = derive(*d).max_rows, blocks = fp8_blocks(std::max(d->d_model, d->d_hidden));
    if (rows >= (int64_t)1 << 31 || rows * blocks >= (int64_t)1 << 31) return MOE_ERR_UNSUPPORTED;
    return MOE_OK;
}

// The first product addresses all of x, as bf16 or as 8-bit rows, through one window of 4 GiB.
static bool too_large_to_gather(const moe_desc_t* d) {
    return (uint64_t)d->n_tokens * (uint64_t)d->d_model >= (1ull << 31) ||
           (uint64_t)d->n_tokens * (uint64_t)fp8_pitch(d->d_model) > kBeyond;
}

static int validate_experts(const moe_fp8_experts_t* w) {
    if (!w || !w->gate || !w->gate_scale || !w->up || !w->up_scale || !w->down || !w->down_scale) return MOE_ERR_INVALID_ARG;
    if (misaligned16(w->gate) || misaligned16(w->up) || misaligned16(w->down)) return MOE_ERR_INVALID_ARG;
    if (misaligned4(w->gate_scale) || misaligned4(w->up_scale) || misaligned4(w->down_scale)) return MOE_ERR_INVALID_ARG;
    return MOE_OK;
}

// One product on high row tiles (fp8.hip).
static void launch_fp8_tiles(const Fp8Gemm& g, const int32_t* expert_offset, const void* x, const uint8_t* x_scale,
                             int64_t x_rows, const int32_t* gather, const void* w, const uint8_t* w_scale, const void* up,
                             const uint8_t* up_scale, void* y, uint8_t* y_scale, bool stream, hipStream_t st) {
    Fp8Args p;
    p.x = (const uint8_t*)x, p.x_scale = x_scale, p.x_rows = x_rows, p.gather = gather;
    p.w[0] = (const uint8_t*)w, p.w[1] = (const uint8_t*)up;
    p.w_scale[0] = w_scale, p.w_scale[1] = up_scale;
    p.y = (uint8_t*)y, p.y_scale = y_scale;
    p.expert_offset = expert_offset, p.max_rows = g.max_rows, p.experts = g.experts;
    p.pitch = g.pitch, p.scale_pitch = fp8_scale_pitch(g.k);
    p.n = g.n, p.n_pad = g.n_pad, p.y_scale_pitch = fp8_scale_pitch(g.n);
    p.col_group = p.tile_shift = 0;
    p.stream = stream;
    if (up)
        launch_fp8_shape<256, true>(p, st);
    else if (fp8_tiles_are_wide(g, compute_units()))
        launch_fp8_shape<256, false>(p, st);
    else
        launch_fp8_shape<128, false>(p, st);
}

// The FFN behind the argument checks.  row_token == nullptr: x holds the permuted rows.
static hipError_t launch_ffn_fp8(const moe_desc_t& d, const Sizes& s, const Fp8Workspace& ws, const void* x,
                                 const int32_t* row_token, const int32_t* expert_offset, const moe_fp8_experts_t& w, void* yp,
                                 hipStream_t st) {
    const int hp = fp8_pitch(d.d_hidden);
    const Fp8Gemm up = fp8_gemm(d.n_experts, s.max_rows, d.d_model, hp), down = fp8_gemm(d.n_experts, s.max_rows, hp, d.d_model);
    const bool stream = fp8_weights_stream(3.0 * d.n_experts * up.pitch * up.n_pad);
    const int64_t x_rows = row_token ? d.n_tokens : s.max_rows;
    if (!fp8_ffn_is_few_rows(d, s)) {
        {
            ProfileScope prof(MOE_KERNEL_DISPATCH, st);
            const hipError_t e = launch_quantize_rows(MOE_DTYPE_BF16, x, x_rows, d.d_model, nullptr,
                                                      row_token ? nullptr : expert_offset + d.n_experts, ws.xq, ws.xs, st);
            if (e != hipSuccess) return e;
        }
        {
            ProfileScope prof(MOE_KERNEL_FFN_GATE_UP, st);
            launch_fp8_tiles(up, expert_offset, ws.xq, ws.xs, x_rows, row_token, w.gate, w.gate_scale, w.up, w.up_scale, ws.hidden,
                             ws.hidden_scale, stream, st);
        }
        ProfileScope prof(MOE_KERNEL_FFN_DOWN, st);
        launch_fp8_tiles(down, expert_offset, ws.hidden, ws.hidden_scale, s.max_rows, nullptr, w.down, w.down_scale, nullptr, nullptr, yp, nullptr,
                         stream, st);
        return hipGetLastError();
    }
    {
        ProfileScope prof(MOE_KERNEL_FFN_GATE_UP, st);
        launch_fp8_thin_gate_up(up, expert_offset, x, x_rows, row_token, w, ws.hidden, stream, st);
    }
    ProfileScope prof(MOE_KERNEL_FFN_DOWN, st);
    launch_fp8_thin(down, expert_offset, ws.hidden, nullptr, s.max_rows, nullptr, w.down, w.down_scale, yp, stream, st);
    return hipGetLastError();
}

}  // namespace capmoe

using namespace capmoe;

static int ffn_fp8_impl(const moe_desc_t* desc, const void* x, const int32_t* row_token, const int32_t* expert_offset,
                        const moe_fp8_experts_t* experts, void* yp, const Fp8Workspace& ws, void* stream) {
    return launch_ffn_fp8(*desc, derive(*desc), ws, x, row_token, expert_offset, *experts, yp, (hipStream_t)stream) == hipSuccess
               ? MOE_OK
               : MOE_ERR_HIP;
}

static int ffn_fp8_checked(const moe_desc_t* desc, const void* x, bool gathered, const int32_t* row_token, const int32_t* expert_offset,
                           const moe_fp8_experts_t* experts, void* yp, void* workspace, size_t workspace_bytes, void* stream) {
    const int v = validate_fp8(desc);
    if (v != MOE_OK) return v;
    const Sizes s = derive(*desc);
    if (!expert_offset || !workspace || (s.max_rows > 0 && (!x || !yp || (gathered && !row_token)))) return MOE_ERR_INVALID_ARG;
    if (misaligned16(x) || misaligned16(yp) || ((uintptr_t)workspace & 255) != 0) return MOE_ERR_INVALID_ARG;
    const int w = validate_experts(experts);
    if (w != MOE_OK) return w;
    if (gathered && too_large_to_gather(desc)) return MOE_ERR_UNSUPPORTED;
    const Fp8Workspace ws = ffn_fp8_workspace(*desc, s, workspace);
    if (workspace_bytes < ws.bytes) return MOE_ERR_WORKSPACE_TOO_SMALL;
    if (s.max_rows == 0) return MOE_OK;
    return ffn_fp8_impl(desc, x, row_token, expert_offset, experts, yp, ws, stream);
}

extern "C" {

int moe_fp8_query(int32_t cols, int32_t* pitch, int32_t* scale_pitch) {
    if (cols < 1) return MOE_ERR_INVALID_ARG;
    if (cols > kFp8MaxWidth) return MOE_ERR_UNSUPPORTED;
    if (pitch) *pitch = fp8_pitch(cols);
    if (scale_pitch) *scale_pitch = fp8_scale_pitch(cols);
    return MOE_OK;
}

static int quantize_checks(int dtype, int32_t cols) {
    if ((dtype != MOE_DTYPE_F32 && dtype != MOE_DTYPE_BF16) || cols < 1) return MOE_ERR_INVALID_ARG;
    if (cols > kFp8MaxWidth || cols % (dtype == MOE_DTYPE_BF16 ? 8 : 4) != 0) return MOE_ERR_UNSUPPORTED;
    return MOE_OK;
}

int moe_quantize_rows(int dtype, const void* x, int64_t n_rows, int32_t cols, const int32_t* row_token,
                      const int32_t* row_count, void* q, uint8_t* scale, void* stream) {
    const int v = quantize_checks(dtype, cols);
    if (v != MOE_OK) return v;
    if (n_rows < 0) return MOE_ERR_INVALID_ARG;
    if (n_rows == 0) return MOE_OK;
    if (!x || !q || !scale || misaligned16(x) || misaligned16(q) || misaligned4(scale)) return MOE_ERR_INVALID_ARG;
    if (n_rows >= (int64_t)1 << 31 || n_rows * fp8_blocks(cols) >= (int64_t)1 << 31) return MOE_ERR_UNSUPPORTED;
    return launch_quantize_rows(dtype, x, n_rows, cols, row_token, row_count, q, scale, (hipStream_t)stream) == hipSuccess
               ? MOE_OK
               : MOE_ERR_HIP;
}

int moe_quantize_weights(int dtype, const void* w, int32_t n_experts, int32_t n_out, int32_t n_in, void* q,
                         uint8_t* scale, void* stream) {
    const int v = quantize_checks(dtype, n_in);
    if (v != MOE_OK) return v;
    if (n_experts < 1 || n_out < 1) return MOE_ERR_INVALID_ARG;
    if (n_out > kFp8MaxWidth) return MOE_ERR_UNSUPPORTED;
    if (!w || !q || !scale || misaligned16(w) || misaligned16(q) || misaligned4(scale)) return MOE_ERR_INVALID_ARG;
    if ((int64_t)fp8_blocks(n_out) * fp8_blocks(n_in) >= ((int64_t)1 << 24) / n_experts) return MOE_ERR_UNSUPPORTED;  // blocks of a launch
    return launch_quantize_weights(dtype, w, n_experts, n_out, n_in, q, scale, (hipStream_t)stream) == hipSuccess ? MOE_OK
                                                                                                                   : MOE_ERR_HIP;
}

int moe_gemm_query(const moe_gemm_t* gemm, size_t* workspace_bytes) {
    const int v = validate_gemm(gemm);
    if (v != MOE_OK) return v;
    if (workspace_bytes) *workspace_bytes = 0;
    return MOE_OK;
}

int moe_grouped_gemm_fp8(const moe_gemm_t* gemm, const void* x, const uint8_t* x_scale, const int32_t* row_token,
                         const int32_t* expert_offset, const void* w, const uint8_t* w_scale, void* y, void* workspace,
                         size_t workspace_bytes, void* stream) {
    const int v = validate_gemm(gemm);
    if (v != MOE_OK) return v;
    if (gemm->max_rows == 0) return MOE_OK;
    if (!x || !x_scale || !expert_offset || !w || !w_scale || !y) return MOE_ERR_INVALID_ARG;
    if (misaligned16(x) || misaligned16(w) || misaligned16(y) || misaligned4(x_scale) || misaligned4(w_scale)) return MOE_ERR_INVALID_ARG;
    (void)workspace, (void)workspace_bytes;  // none is needed
    const Fp8Gemm g = fp8_gemm(gemm->n_experts, gemm->max_rows, gemm->n_in, gemm->n_out);
    if (row_token && gemm->src_rows == 0) return MOE_ERR_INVALID_ARG;
    if (row_token && (uint64_t)gemm->src_rows * (uint64_t)g.pitch > kBeyond) return MOE_ERR_UNSUPPORTED;
    hipStream_t st = (hipStream_t)stream;
    const int64_t x_rows = row_token ? gemm->src_rows : gemm->max_rows;
    const bool streamed = fp8_weights_stream((double)g.experts * g.pitch * g.n_pad);
    if (fp8_gemm_is_few_rows(g)) {
        launch_fp8_thin(g, expert_offset, x, x_scale, x_rows, row_token, w, w_scale, y, streamed, st);
    } else {
        launch_fp8_tiles(g, expert_offset, x, x_scale, x_rows, row_token, w, w_scale, nullptr, nullptr, y, nullptr, streamed, st);
    }
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

int moe_query_fp8(const moe_desc_t* desc, size_t* workspace_bytes) {
    const int v = validate_fp8(desc);
    if (v != MOE_OK) return v;
    size_t other = 0;
    const int q = moe_query(desc, nullptr, nullptr, nullptr, &other);
    if (q != MOE_OK) return q;
    const Sizes s = derive(*desc);
    const size_t mine = ffn_fp8_workspace(*desc, s, nullptr).bytes;
    if (workspace_bytes) *workspace_bytes = std::max(mine, other);
    return MOE_OK;
}

int moe_grouped_ffn_fp8(const moe_desc_t* desc, const void* xp, const int32_t* expert_offset,
                        const moe_fp8_experts_t* experts, void* yp, void* workspace, size_t workspace_bytes,
                        void* stream) {
    return ffn_fp8_checked(desc, xp, false, nullptr, expert_offset, experts, yp, workspace, workspace_bytes, stream);
}

int moe_dispatch_ffn_fp8(const moe_desc_t* desc, const void* x, const int32_t* expert_offset, const int32_t* row_token,
                         const moe_fp8_experts_t* experts, void* yp, void* workspace, size_t workspace_bytes,
                         void* stream) {
    return ffn_fp8_checked(desc, x, true, row_token, expert_offset, experts, yp, workspace, workspace_bytes, stream);
}

int moe_layer_forward_fp8(const moe_desc_t* desc, const void* x, const float* w_router, const float* bias,
                          const moe_fp8_experts_t* experts, const uint8_t* token_class, uint32_t seed, float* logits,
                          float* scores, int32_t* topk_idx, float* topk_score, int32_t* expert_count,
                          int32_t* seg_count, int32_t* expert_offset, int32_t* row_token, float* row_weight,
                          int32_t* pair_row, void* yp, void* y, void* workspace, size_t workspace_bytes, void* stream) {
    // every check first, so that a refusal leaves nothing enqueued
    const int v = validate_fp8(desc);
    if (v != MOE_OK) return v;
    const Sizes s = derive(*desc);
    if (!expert_count || !seg_count || !expert_offset || !workspace) return MOE_ERR_INVALID_ARG;
    if (((uintptr_t)workspace & 255) != 0) return MOE_ERR_INVALID_ARG;
    if (desc->n_tokens > 0) {
        if (!x || !w_router || !logits || !scores || !topk_idx || !topk_score || !pair_row || !yp || !y || !row_weight)
            return MOE_ERR_INVALID_ARG;
        if (misaligned16(x) || misaligned16(w_router) || misaligned16(yp) || misaligned16(y) || misaligned16(scores) ||
            misaligned16(topk_idx) || misaligned16(pair_row))
            return MOE_ERR_INVALID_ARG;
        if (too_large_to_gather(desc)) return MOE_ERR_UNSUPPORTED;
    }
    if (s.max_rows > 0) {
        if (!row_token) return MOE_ERR_INVALID_ARG;
        const int w = validate_experts(experts);
        if (w != MOE_OK) return w;
    }
    size_t need = 0;
    const int q = moe_query_fp8(desc, &need);
    if (q != MOE_OK) return q;
    if (workspace_bytes < need) return MOE_ERR_WORKSPACE_TOO_SMALL;
    int st = moe_route_topk(desc, x, w_router, bias, 0, logits, scores, topk_idx, topk_score, workspace, workspace_bytes, stream);
    if (st != MOE_OK) return st;
    st = moe_capacity_drop_ranked(desc, scores, topk_idx, token_class, seed, expert_count, seg_count, expert_offset, row_token,
                                  row_weight, pair_row, workspace, workspace_bytes, stream);
    if (st != MOE_OK) return st;
    if (s.max_rows > 0) {
        st = ffn_fp8_impl(desc, x, row_token, expert_offset, experts, yp, ffn_fp8_workspace(*desc, s, workspace), stream);
        if (st != MOE_OK) return st;
    }
    return moe_combine(desc, yp, row_weight, pair_row, y, stream);
}

}  // extern "C"
