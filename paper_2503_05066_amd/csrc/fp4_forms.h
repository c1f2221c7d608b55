// Sizes of the 4-bit format and the rules by which a call on 4-bit experts takes its kernels and their shapes (host code).
#pragma once

#include "fp8_forms.h"

namespace capmoe {

constexpr int kFp4Block = 32;    // values of a row that share a scale
constexpr int kFp4Slab = 256;    // columns of 128 bytes of a row
constexpr int kFp4Group = 512;   // columns of 16 scale bytes

__host__ __device__ inline int fp4_slabs(int cols) { return (cols + kFp4Slab - 1) / kFp4Slab; }
__host__ __device__ inline int fp4_pitch(int cols) { return fp4_slabs(cols) * (kFp4Slab / 2); }
__host__ __device__ inline int fp4_groups(int cols) { return (cols + kFp4Group - 1) / kFp4Group; }
__host__ __device__ inline int fp4_scale_pitch(int cols) { return fp4_groups(cols) * (kFp4Group / kFp4Block); }

// One product on 4-bit weights as the kernels take it.
struct Fp4Gemm {
    int experts;
    int64_t max_rows;
    int k;            // columns of the activations as they are
    int pitch;        // bytes of a 4-bit row
    int scale_pitch;
    int n;            // output columns
    int n_pad;        // weight rows of an expert
};
inline Fp4Gemm fp4_gemm(int experts, int64_t max_rows, int k, int n) {
    return Fp4Gemm{experts, max_rows, k, fp4_pitch(k), fp4_scale_pitch(k), n, fp8_pitch(n)};
}

// Which kernels an FFN or a product takes: those for few rows (fp4_thin.hip) or on high row tiles.
inline bool fp4_ffn_is_few_rows(const moe_desc_t& d, const Sizes& s) {
    const bool few = fp8_few_weights(3.0 * d.n_experts * fp4_pitch(d.d_model) * fp8_pitch(d.d_hidden));
    const int64_t most = std::min<int64_t>((int64_t)s.n_blocks * s.cap, d.n_tokens);  // rows of an expert
    return most <= (few ? 32 : 16) || (most <= kFp8MostPasses * 16 && s.max_rows <= (few ? 16ll : 4ll) * d.n_experts);
}
inline bool fp4_gemm_is_few_rows(const Fp4Gemm& g) {
    const bool few = fp8_few_weights((double)g.experts * g.pitch * g.n_pad);
    return g.max_rows <= (few ? 64 : 32) || (g.max_rows <= kFp8MostPasses * 32 && g.max_rows <= (few ? 32ll : 8ll) * g.experts);
}

// Which width a product on high tiles takes, 256 or 128 columns.
inline bool fp4_tiles_are_wide(const Fp4Gemm& g, int cus) {
    const int64_t tiles = g.max_rows / kFfnTileM + std::min<int64_t>(g.max_rows, g.experts);
    return g.n_pad % 256 == 0 && 4 * tiles * (g.n_pad / 256) > 3 * cus;
}

}  // namespace capmoe
