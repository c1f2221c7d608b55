// Activations and expert weights to e2m1 with a power-of-two scale per row and 32 columns, and 4- and 8-bit rows back to values.
//
//   b = smallest b >= 0 with amax <= 6 * 2^(b - 127),  q = e2m1(x / 2^(b - 127))
//
// The division is exact, so there is one rounding, and the bits do not depend on who computes them.  A wave takes 512 columns
// of a row, the 16 scale bytes of a group: every value is read and written once; the bytes bound the kernels.
#include <algorithm>

#include "ffn_tile.h"
#include "fp4.h"

namespace capmoe {

// Where row r of the output comes from: row r, the r-th of a permutation, or a weight row of an expert's `out` whose rows are
// filled up to `pad`.
struct FromRows {
    static constexpr bool kOnce = false;
    static constexpr int kAhead = 1, kMostBlocks = 4096;
    const int32_t* row_token;
    __device__ __forceinline__ int64_t of(uint32_t r) const { return row_token ? row_token[r] : r; }
};
struct FromWeights {
    static constexpr bool kOnce = true;  // read once, at load: lines that need not be kept
    static constexpr int kAhead = 2, kMostBlocks = 65536;
    Divisor pad;
    int out;
    __device__ __forceinline__ int64_t of(uint32_t r) const {  // below 0: a row of zeros
        const uint32_t e = pad.divide(r), n = r - e * pad.d;
        return n < (uint32_t)out ? (int64_t)e * out + n : -1;
    }
};

// A wave requests kAhead groups before it writes the first.  Of rows one, in few blocks, of weights two, in many (us, kAhead and
// blocks 1 4096, 1 16384, 2 4096, 2 65536; rows 13000 x 2048 of 4096 permuted 11.1, 12.0, 11.3, 12.4, 8192 x 4096 14.0, 16.0, 14.3, 14.4; weights
// 65536 x 2048 61, 59, 58, 54, 114688 x 4096 243, 246, 237, 207).
template <bool BF16, class From>
__global__ __launch_bounds__(256) void quantize_fp4_kernel(const void* __restrict__ x, const From from,
                                                           const int32_t* __restrict__ row_count, uint8_t* __restrict__ q,
                                                           uint8_t* __restrict__ scale, int64_t n_rows, int cols, Divisor groups) {
    if (row_count) n_rows = min(n_rows, (int64_t)max(*row_count, 0));
    const uint32_t total = (uint32_t)(n_rows * groups.d);
    const int lane = threadIdx.x & 63, filled = fp4_slabs(cols) * kFp4Slab;
    constexpr int kAhead = From::kAhead;
    for (uint32_t b0 = (blockIdx.x * 4 + (threadIdx.x >> 6)) * kAhead; b0 < total; b0 += gridDim.x * 4 * kAhead) {
        Eight<BF16> e[kAhead];
        uint32_t r[kAhead], g[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const uint32_t b = min(b0 + u, total - 1);
            r[u] = groups.divide(b), g[u] = b - r[u] * groups.d;
            const int64_t src = from.of(r[u]);
            const int col = (int)g[u] * kFp4Group + lane * 8;
            e[u].template load<From::kOnce>((const uint8_t*)x + src * cols * (BF16 ? 2 : 4), src >= 0 ? col : cols, cols);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (b0 + u >= total) break;
            write_group_fp4(e[u], lane, (int)g[u] * kFp4Group + lane * 8, filled,
                            q + (int64_t)r[u] * (filled / 2) + g[u] * (kFp4Group / 2), scale + (int64_t)(b0 + u) * 16);
        }
    }
}

template <class From>
static hipError_t launch_quantize_fp4(int dtype, const void* x, const From& from, const int32_t* row_count, int64_t n_rows, int cols,
                                      void* q, uint8_t* scale, hipStream_t st) {
    const Divisor groups((uint32_t)fp4_groups(cols));
    const dim3 grid((unsigned)std::min<int64_t>((n_rows * groups.d + 4 * From::kAhead - 1) / (4 * From::kAhead), From::kMostBlocks));
    auto kern = dtype == MOE_DTYPE_BF16 ? quantize_fp4_kernel<true, From> : quantize_fp4_kernel<false, From>;
    hipLaunchKernelGGL(kern, grid, dim3(256), 0, st, x, from, row_count, (uint8_t*)q, scale, n_rows, cols, groups);
    return hipGetLastError();
}

hipError_t launch_quantize_rows_fp4(int dtype, const void* x, int64_t n_rows, int cols, const int32_t* row_token,
                                    const int32_t* row_count, void* q, uint8_t* scale, hipStream_t st) {
    return launch_quantize_fp4(dtype, x, FromRows{row_token}, row_count, n_rows, cols, q, scale, st);
}

hipError_t launch_quantize_weights_fp4(int dtype, const void* w, int experts, int n_out, int n_in, void* q, uint8_t* scale,
                                       hipStream_t st) {
    const int pad = fp8_pitch(n_out);
    return launch_quantize_fp4(dtype, w, FromWeights{Divisor((uint32_t)pad), n_out}, nullptr, (int64_t)experts * pad, n_in, q, scale, st);
}

// A wave takes 512 columns of a row, eight a lane.
template <int BITS, bool BF16, bool ONCE>
__global__ __launch_bounds__(256) void dequantize_rows_kernel(const uint8_t* __restrict__ q, const uint8_t* __restrict__ scale,
                                                              void* __restrict__ y, int64_t n_rows, int cols, Divisor groups) {
    const uint32_t total = (uint32_t)(n_rows * groups.d);
    const int lane = threadIdx.x & 63;
    for (uint32_t b = blockIdx.x * 4 + (threadIdx.x >> 6); b < total; b += gridDim.x * 4) {
        const uint32_t r = groups.divide(b), g = b - r * groups.d;
        const int col = (int)g * kFp4Group + lane * 8;
        if (col >= cols) continue;
        float v[8];
        uint32_t byte;
        if constexpr (BITS == 4) {
            const uint32_t w = *(const uint32_t*)(q + (int64_t)r * fp4_pitch(cols) + col / 2);
            byte = scale[(int64_t)b * 16 + 4 * ((lane >> 2) & 3) + (lane >> 4)];
            typedef __attribute__((ext_vector_type(2))) float f32x2;
            const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0), c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1);
            const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2), f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3);
            v[0] = a[0], v[1] = a[1], v[2] = c[0], v[3] = c[1], v[4] = d[0], v[5] = d[1], v[6] = f[0], v[7] = f[1];
        } else {
            const uint2 w = *(const uint2*)(q + (int64_t)r * fp8_pitch(cols) + col);
            byte = scale[(int64_t)r * fp8_scale_pitch(cols) + col / kFp8Block];
            typedef __attribute__((ext_vector_type(2))) float f32x2;
            const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.x, false), c = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.x, true);
            const f32x2 d = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.y, false), f = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.y, true);
            v[0] = a[0], v[1] = a[1], v[2] = c[0], v[3] = c[1], v[4] = d[0], v[5] = d[1], v[6] = f[0], v[7] = f[1];
        }
        // 2^(byte - 127); 255 is not a number, and neither is anything times it
        const float scaled = __uint_as_float(byte == 0 ? 0x00400000u : (byte == 255 ? 0x7fc00000u : byte << 23));
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= scaled;
        if constexpr (BF16) {
            const uint4 o = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
            store16<ONCE>((uint16_t*)y + (int64_t)r * cols + col, o);
        } else {
            auto bits = [&](int i) { return __float_as_uint(v[i]); };
            float* out = (float*)y + (int64_t)r * cols + col;
            store16<ONCE>(out, make_uint4(bits(0), bits(1), bits(2), bits(3)));
            if (col + 4 < cols) store16<ONCE>(out + 4, make_uint4(bits(4), bits(5), bits(6), bits(7)));
        }
    }
}

hipError_t launch_dequantize_rows(int bits, int dtype, const void* q, const uint8_t* scale, int64_t n_rows, int cols, void* y,
                                  hipStream_t st) {
    const Divisor groups((uint32_t)fp4_groups(cols));
    const dim3 grid((unsigned)std::min<int64_t>((n_rows * groups.d + 3) / 4, 16384));
    // Values that the L2s do not hold are written past them (64 experts of 1024 x 2048, quantised and back: 121 us, 105).
    const bool bf16 = dtype == MOE_DTYPE_BF16, once = (double)n_rows * cols * (bf16 ? 2 : 4) > kL2Bytes;
    auto kern = bits == 4 ? (bf16 ? (once ? dequantize_rows_kernel<4, true, true> : dequantize_rows_kernel<4, true, false>)
                                  : (once ? dequantize_rows_kernel<4, false, true> : dequantize_rows_kernel<4, false, false>))
                          : (bf16 ? (once ? dequantize_rows_kernel<8, true, true> : dequantize_rows_kernel<8, true, false>)
                                  : (once ? dequantize_rows_kernel<8, false, true> : dequantize_rows_kernel<8, false, false>));
    hipLaunchKernelGGL(kern, grid, dim3(256), 0, st, (const uint8_t*)q, scale, y, n_rows, cols, groups);
    return hipGetLastError();
}

}  // namespace capmoe
