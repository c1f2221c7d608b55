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

}  // namespace capmoe
