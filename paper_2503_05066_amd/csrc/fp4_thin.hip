// Products on 4-bit rows and 4-bit expert weights, grouped by expert.
//
//   y[r,n] = sum over blocks b of 32 k:  2^(xs[r,b] + ws[n,b] - 254) * sum over k in b: x[r,k] w[e,n,k]
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 128 k at once, 64 bytes of a row, and takes a scale byte per row and 32 of
// them from each lane.  Lane l holds piece l >> 4 (16 bytes, one block) of row l & 15.  A slab is 128 bytes of a row: pieces
// l >> 4 and (l >> 4) + 4, so the four scale bytes of two slabs that a lane needs are one word of a group of 16.
#include <algorithm>

#include "ffn_tile.h"
#include "fp4.h"

namespace capmoe {

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(4))) int i32x4;

struct Thin4Args {
    const uint8_t *x, *x_scale;
    const int32_t* gather;
    const uint8_t *w[2], *w_scale[2];
    uint16_t* y;
    const int32_t* expert_offset;
    int experts, pitch, scale_pitch, n, n_pad, col_blocks;
};

__device__ __forceinline__ i32x8 operand(const uint8_t* p) {
    const i32x4 v = *(const i32x4*)p;
    return __builtin_shufflevector(v, v, 0, 1, 2, 3, -1, -1, -1, -1);
}

// A block takes 64 rows of an expert and 64 weight rows (gate and up rows of 32 columns), a wave 16 of the rows.
template <bool SWIGLU>
__global__ __launch_bounds__(256) void fp4_simple_kernel(const Thin4Args p) {
    constexpr int kCols = SWIGLU ? 32 : 64;
    int tile = blockIdx.x / p.col_blocks;
    const int n0 = (blockIdx.x - tile * p.col_blocks) * kCols;
    int e = 0, lo = 0, hi = 0;
    for (;; ++e) {
        if (e >= p.experts) return;
        lo = p.expert_offset[e], hi = p.expert_offset[e + 1];
        const int tiles = (hi - lo + 63) / 64;
        if (tile < tiles) break;
        tile -= tiles;
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lr = lane & 15, lk = lane >> 4;
    const int row = lo + tile * 64 + wave * 16 + lr;
    const int64_t src = p.gather ? p.gather[min(row, hi - 1)] : min(row, hi - 1);
    const uint8_t* x = p.x + src * p.pitch + lk * 16;
    const uint8_t* xs = p.x_scale + src * p.scale_pitch + lk * 4;
    const uint8_t *w[4], *ws[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t at = (int64_t)e * p.n_pad + n0 + (SWIGLU ? i % 2 : i) * 16 + lr;
        w[i] = p.w[SWIGLU ? i / 2 : 0] + at * p.pitch + lk * 16;
        ws[i] = p.w_scale[SWIGLU ? i / 2 : 0] + at * p.scale_pitch + lk * 4;
    }
    f32x4 acc[4] = {};
    for (int k = 0; k < p.pitch; k += 128) {
        const int at = k / 256 * 16, sh = k & 128 ? 16 : 0;  // of the scales: two bytes a slab
        const int sx = (int)(*(const uint32_t*)(xs + at) >> sh);
        int sw[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) sw[i] = (int)(*(const uint32_t*)(ws[i] + at) >> sh);
        const i32x8 x0 = operand(x + k), x1 = operand(x + k + 64);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            acc[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(w[i] + k), x0, acc[i], 4, 4, 0, sw[i], 0, sx);
            acc[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(w[i] + k + 64), x1, acc[i], 4, 4, 1, sw[i], 1, sx);
        }
    }
    if (row >= hi) return;
#pragma unroll
    for (int i = 0; i < (SWIGLU ? 2 : 4); ++i) {
        const int col = n0 + i * 16 + 4 * lk;
        f32x4 o = acc[i];
        if (SWIGLU) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                o[k] = o[k] * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(o[k] * -1.4426950408889634f)) * acc[i + 2][k];
        }
        if (col < p.n) *(uint2*)(p.y + (int64_t)row * p.n + col) = make_uint2(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]));
    }
}

void launch_fp4_thin(const Fp4Gemm& g, const int32_t* expert_offset, const void* x, const uint8_t* x_scale, int64_t x_rows,
                        const int32_t* gather, const void* w, const uint8_t* w_scale, const void* w_up, const uint8_t* up_scale,
                        void* y, hipStream_t st) {
    Thin4Args a;
    a.x = (const uint8_t*)x, a.x_scale = x_scale, a.gather = gather;
    a.w[0] = (const uint8_t*)w, a.w[1] = (const uint8_t*)w_up, a.w_scale[0] = w_scale, a.w_scale[1] = up_scale;
    a.y = (uint16_t*)y, a.expert_offset = expert_offset;
    a.experts = g.experts, a.pitch = g.pitch, a.scale_pitch = g.scale_pitch, a.n = g.n, a.n_pad = g.n_pad;
    const int cols = w_up ? 32 : 64;
    a.col_blocks = (g.n + cols - 1) / cols;
    const int64_t tiles = g.max_rows / 64 + std::min<int64_t>(g.max_rows, g.experts);
    auto kern = w_up ? fp4_simple_kernel<true> : fp4_simple_kernel<false>;
    hipLaunchKernelGGL(kern, dim3((unsigned)(tiles * a.col_blocks)), dim3(256), 0, st, a);
}

}  // namespace capmoe
