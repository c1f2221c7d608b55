// Internal declarations of the 8-bit experts (see include/capmoe.h for the format): e4m3 values, power-of-two scales.
#pragma once

#include "fp8_forms.h"

namespace capmoe {

// ---------------------------------------------------------------------------------------------
// quantising on the device
// ---------------------------------------------------------------------------------------------
typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
typedef __attribute__((ext_vector_type(2))) short s16x2;
typedef __attribute__((ext_vector_type(2))) __bf16 fp8_bf16x2;

// The scale byte of a block whose largest finite magnitude has these fp32 bits: the smallest b >= 0 with
// amax <= 448 * 2^(b - 127) = 1.75 * 2^(b - 119), read off amax's exponent and whether its fraction exceeds 0.75.
__device__ inline uint32_t scale_byte(uint32_t amax_bits) {
    const int b = (int)(amax_bits >> 23) - 8 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return b > 0 ? (uint32_t)b : 0u;
}

// Largest finite magnitude of 2W bf16 values (as the low 15 bits of one).  Values that are not finite are replaced by
// zeros and their places set in `bad` (bit 2w + half): rare, so everything else costs two instructions per pair.
template <int W>
__device__ __forceinline__ uint32_t amax_bf16(uint32_t (&v)[W], uint32_t& bad) {
    static_assert(W <= 16, "a bit per value");
    u16x2 m = {0, 0};
#pragma unroll
    for (int w = 0; w < W; ++w) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, v[w] & 0x7fff7fffu));
    uint32_t top = m[0] > m[1] ? m[0] : m[1];
    bad = 0;
    if (top >= 0x7f80u) {
        top = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const uint32_t lo = v[w] & 0x7fffu, hi = (v[w] >> 16) & 0x7fffu;
            if (lo >= 0x7f80u) {
                bad |= 1u << (2 * w);
                v[w] &= 0xffff0000u;
            } else if (lo > top) {
                top = lo;
            }
            if (hi >= 0x7f80u) {
                bad |= 2u << (2 * w);
                v[w] &= 0x0000ffffu;
            } else if (hi > top) {
                top = hi;
            }
        }
    }
    return top;
}

// The places of `bad` become NaN.
template <int Q>
__device__ __forceinline__ void mark_bad(uint32_t (&q)[Q], uint32_t bad) {
    if (bad) {
#pragma unroll
        for (int i = 0; i < 4 * Q; ++i)
            if (bad & (1u << i)) q[i / 4] = (q[i / 4] & ~(0xffu << (8 * (i % 4)))) | (0x7fu << (8 * (i % 4)));
    }
}

// 2W bf16 values divided by 2^(byte - 127) and rounded to e4m3: one instruction per pair.
template <int W>
__device__ __forceinline__ void to_e4m3(const uint32_t (&v)[W], uint32_t byte, uint32_t (&q)[W / 2]) {
    const float scale = __uint_as_float(byte << 23);  // the instruction reads the exponent
#pragma unroll
    for (int i = 0; i < W / 2; ++i) {
        s16x2 o = {0, 0};
        o = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(o, __builtin_bit_cast(fp8_bf16x2, v[2 * i]), scale, false);
        o = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(o, __builtin_bit_cast(fp8_bf16x2, v[2 * i + 1]), scale, true);
        q[i] = __builtin_bit_cast(uint32_t, o);
    }
}

// The largest of the values of lanes l, l ^ 16, l ^ 32, l ^ 48.
__device__ __forceinline__ uint32_t max_over_rows_of_16(uint32_t m) {
    auto a = __builtin_amdgcn_permlane32_swap(m, m, false, false);
    m = a[0] > a[1] ? a[0] : a[1];
    auto b = __builtin_amdgcn_permlane16_swap(m, m, false, false);
    return b[0] > b[1] ? b[0] : b[1];
}

// ---------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------
hipError_t launch_quantize_rows(int dtype, const void* x, int64_t n_rows, int cols, const int32_t* row_token,
                                const int32_t* row_count, void* q, uint8_t* scale, hipStream_t st);
hipError_t launch_quantize_weights(int dtype, const void* w, int experts, int n_out, int n_in, void* q, uint8_t* scale,
                                   hipStream_t st);

// Arguments of the kernels for high row tiles (fp8.hip).
struct Fp8Args {
    const uint8_t *x, *x_scale;
    int64_t x_rows;                    // rows of x
    const int32_t* gather;
    const uint8_t *w[2], *w_scale[2];  // gate (or the only weights), up
    uint8_t* y;                        // bf16 rows of n columns; with SWIGLU 8-bit rows of n_pad
    uint8_t* y_scale;                  // with SWIGLU
    const int32_t* expert_offset;
    int64_t max_rows;
    int experts;
    int pitch, scale_pitch;            // of x and of a weight row
    int n, n_pad, y_scale_pitch;
    int col_group, tile_shift;
    int stream;                        // the weights' lines need not be kept
};
// One launch over all tiles; the shape: 256 weight rows, gate and up rows of 128 columns or not, or 128.
template <int BN, bool SWIGLU>
void launch_fp8_shape(Fp8Args p, hipStream_t st);

// Kernels for tiles of few rows.  x_scale == nullptr: x is bf16 and is quantised as it is read.
void launch_fp8_thin(const Fp8Gemm& g, const int32_t* expert_offset, const void* x, const uint8_t* x_scale, int64_t x_rows,
                     const int32_t* gather, const void* w, const uint8_t* w_scale, void* y, bool stream, hipStream_t st);
// .. the products of the gate and the up weights, and y = silu(gate) * up; x is bf16
void launch_fp8_thin_gate_up(const Fp8Gemm& g, const int32_t* expert_offset, const void* x, int64_t x_rows, const int32_t* gather,
                             const moe_fp8_experts_t& w, void* y, bool stream, hipStream_t st);

}  // namespace capmoe
