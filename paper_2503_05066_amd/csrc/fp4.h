// Internal declarations of the 4-bit experts (see include/capmoe.h for the format): e2m1 values, a power-of-two scale for each
// 32 of a row.
#pragma once

#include "fp4_forms.h"
#include "quantize.h"

namespace capmoe {

// ---------------------------------------------------------------------------------------------
// quantising on the device
// ---------------------------------------------------------------------------------------------
constexpr uint32_t kFp4NoNumber = 255;  // the scale byte of a block that holds a NaN or an infinity

// The scale byte of a block whose largest magnitude has these fp32 bits: the smallest b >= 0 with
// amax <= 6 * 2^(b - 127) = 1.5 * 2^(b - 125), read off amax's exponent and whether its fraction exceeds 0.5.
__device__ __forceinline__ uint32_t fp4_scale_byte(uint32_t amax_bits) {
    if (amax_bits >= 0x7f800000u) return kFp4NoNumber;
    const int b = (int)(amax_bits >> 23) - 2 + ((amax_bits & 0x7fffffu) > 0x400000u ? 1 : 0);
    return b > 0 ? (uint32_t)b : 0u;
}

// fp32 bits of the largest magnitude of a lane's eight values, whether they are finite or not
template <bool BF16>
__device__ __forceinline__ uint32_t amax_of_8(const Eight<BF16>& e) {
    if constexpr (BF16) {
        u16x2 m = {0, 0};
#pragma unroll
        for (int w = 0; w < 4; ++w) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, e.v[w] & 0x7fff7fffu));
        return (uint32_t)max(m[0], m[1]) << 16;
    } else {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, e.v[i] & 0x7fffffffu);
        return top;
    }
}

// Eight values divided by 2^(byte - 127) and rounded to e2m1, the first in the lowest four bits; one instruction per pair.
template <bool BF16>
__device__ __forceinline__ uint32_t to_e2m1(const Eight<BF16>& e, uint32_t byte) {
    if (byte == kFp4NoNumber) return 0;
    const float scale = __uint_as_float(byte << 23);  // the instructions read the exponent
    uint32_t q = 0;
    if constexpr (BF16) {
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(fp8_bf16x2, e.v[0]), scale, 0);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(fp8_bf16x2, e.v[1]), scale, 1);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(fp8_bf16x2, e.v[2]), scale, 2);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(fp8_bf16x2, e.v[3]), scale, 3);
    } else {
        auto f = [&](int i) { return __uint_as_float(e.v[i]); };
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f(0), f(1), scale, 0);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f(2), f(3), scale, 1);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f(4), f(5), scale, 2);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f(6), f(7), scale, 3);
    }
    return q;
}

// the largest of the 4 lanes l & ~3 .. l | 3
__device__ __forceinline__ uint32_t max_of_4(uint32_t m) {
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xb1, 0xf, 0xf, false));  // quad_perm 1 0 3 2
    return max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4e, 0xf, 0xf, false));  // quad_perm 2 3 0 1
}

// v of lane l, l ^ 16, l ^ 32, l ^ 48, or-ed
__device__ __forceinline__ uint32_t or_over_rows_of_16(uint32_t v) {
    const auto a = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = a[0] | a[1];
    const auto b = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return b[0] | b[1];
}

// A wave holds 512 columns of a row, eight a lane, from a column that divides 512: their 4-bit form.  Behind the row's end the
// values are zeros, which is also what the row is filled with.  q, scale: of the group.
template <bool BF16>
__device__ __forceinline__ void write_group_fp4(const Eight<BF16>& e, int lane, int col, int cols_filled, uint8_t* q, uint8_t* scale) {
    const uint32_t byte = fp4_scale_byte(max_of_4(amax_of_8(e)));
    if (col < cols_filled) *(uint32_t*)(q + lane * 4) = to_e2m1(e, byte);
    // block 4 j + g is that of lanes 16 j + 4 g ..: its byte has place 4 g + j, byte j of word g
    const uint32_t word = or_over_rows_of_16(byte << (8 * (lane >> 4)));
    if ((lane & 0x33) == 0) *(uint32_t*)(scale + lane) = word;
}

// ---------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------
hipError_t launch_quantize_rows_fp4(int dtype, const void* x, int64_t n_rows, int cols, const int32_t* row_token,
                                    const int32_t* row_count, void* q, uint8_t* scale, hipStream_t st);
hipError_t launch_quantize_weights_fp4(int dtype, const void* w, int experts, int n_out, int n_in, void* q, uint8_t* scale,
                                       hipStream_t st);
hipError_t launch_dequantize_rows(int bits, int dtype, const void* q, const uint8_t* scale, int64_t n_rows, int cols, void* y,
                                  hipStream_t st);
hipError_t launch_norm_rows(const moe_norm_t& norm, const void* x, const void* residual, const void* weight,
                            const int32_t* row_count, void* sum, void* y, void* q, uint8_t* scale, hipStream_t st);

// Arguments of the kernels for high row tiles (fp4.hip): as those of the 8-bit ones (fp8.h); y: bf16 rows of n columns, with SWIGLU 4-bit
// rows of y_pitch bytes.
struct Fp4Args : Fp8Args {
    int y_pitch;
};
template <int BN, bool SWIGLU>
void launch_fp4_shape(Fp4Args p, hipStream_t st);

// Kernels for tiles of few rows: a product, y bf16, or (up != nullptr) the gate and the up product and y, y_scale = silu(gate) * up in
// 4 bits; g.n is then a multiple of 128.
void launch_fp4_thin(const Fp4Gemm& g, const int32_t* expert_offset, const void* x, const uint8_t* x_scale, int64_t x_rows,
                     const int32_t* gather, const void* w, const uint8_t* w_scale, const void* up, const uint8_t* up_scale, void* y,
                     uint8_t* y_scale, bool stream, hipStream_t st);

}  // namespace capmoe
