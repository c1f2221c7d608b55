// Activations and expert weights to e4m3 with power-of-two scales per 128 values of a row, or per 128 x 128 block.
//
//   b = smallest b >= 0 with amax <= 448 * 2^(b - 127),  q = e4m3(x / 2^(b - 127))
//
// The division is exact, so there is one rounding, and the bits do not depend on who computes them.  Both kernels read
// every value once and write it once; the bytes bound them.
#include <algorithm>

#include "fp8.h"

namespace capmoe {

// n / d for n < 2^31 by a multiplication: with 2^(s - 1) < d <= 2^s and m = ceil(2^(31 + s) / d), floor(n * m / 2^(31 + s)).
struct Divisor {
    uint32_t d, m;
    int s;
    explicit Divisor(uint32_t d_) : d(d_), s(0) {
        while ((1u << s) < d) ++s;
        m = (uint32_t)((((uint64_t)1 << (31 + s)) + d - 1) / d);
    }
    __device__ __forceinline__ uint32_t divide(uint32_t n) const { return (uint32_t)(((uint64_t)n * m) >> (31 + s)); }
};

// Eight values of a lane, of a row that begins at x and has `cols` of them, from column col; zeros behind the row's end.
template <bool BF16>
struct Eight {
    uint32_t v[BF16 ? 4 : 8];
    __device__ __forceinline__ void load(const void* row, int col, int cols) {
        if (BF16) {
            uint4 p = make_uint4(0, 0, 0, 0);
            if (col < cols) p = *(const uint4*)((const uint16_t*)row + col);
            v[0] = p.x, v[1] = p.y, v[2] = p.z, v[3] = p.w;
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint4 p = make_uint4(0, 0, 0, 0);
                if (col + 4 * h < cols) p = *(const uint4*)((const float*)row + col + 4 * h);
                v[(4 * h) % (BF16 ? 4 : 8)] = p.x, v[(4 * h + 1) % (BF16 ? 4 : 8)] = p.y;
                v[(4 * h + 2) % (BF16 ? 4 : 8)] = p.z, v[(4 * h + 3) % (BF16 ? 4 : 8)] = p.w;
            }
        }
    }
    // fp32 bits of the largest finite magnitude; values that are not finite become zeros, noted in bad
    __device__ __forceinline__ uint32_t amax(uint32_t& bad) {
        if constexpr (BF16) {
            return amax_bf16(v, bad) << 16;
        } else {
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, v[i] & 0x7fffffffu);
            bad = 0;
            if (top >= 0x7f800000u) {
                top = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t a = v[i] & 0x7fffffffu;
                    if (a >= 0x7f800000u)
                        bad |= 1u << i, v[i] = 0;
                    else
                        top = max(top, a);
                }
            }
            return top;
        }
    }
    __device__ __forceinline__ uint2 quantized(uint32_t byte, uint32_t bad) const {
        uint32_t q[2];
        if constexpr (BF16) {
            to_e4m3(v, byte, q);
        } else {
            const float inverse = __uint_as_float((254u - byte) << 23);  // byte <= 247: a normal number
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                int o = __builtin_amdgcn_cvt_pk_fp8_f32(__uint_as_float(v[4 * i]) * inverse, __uint_as_float(v[4 * i + 1]) * inverse, 0, false);
                q[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(__uint_as_float(v[4 * i + 2]) * inverse,
                                                                 __uint_as_float(v[4 * i + 3]) * inverse, o, true);
            }
        }
        mark_bad(q, bad);
        return make_uint2(q[0], q[1]);
    }
};

// the largest of the 16 lanes l & ~15 .. l | 15
__device__ __forceinline__ uint32_t max_of_16(uint32_t m) {
#pragma unroll
    for (int off = 1; off < 16; off <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, off, kWave));
    return m;
}

// Sixteen lanes take a block of a row, eight values each; consecutive groups take consecutive blocks.
template <bool BF16>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const void* __restrict__ x, const int32_t* __restrict__ row_token,
                                                            const int32_t* __restrict__ row_count, uint8_t* __restrict__ q,
                                                            uint8_t* __restrict__ scale, int64_t n_rows, int cols, int scale_pitch,
                                                            Divisor blocks) {
    if (row_count) n_rows = min(n_rows, (int64_t)max(*row_count, 0));
    const uint32_t total = (uint32_t)(n_rows * blocks.d);
    const int lane = threadIdx.x & 15;
    for (uint32_t b = blockIdx.x * 16 + (threadIdx.x >> 4); b < total; b += gridDim.x * 16) {
        const uint32_t r = blocks.divide(b), kb = b - r * blocks.d;
        const int64_t src = row_token ? row_token[r] : r;
        const int col = (int)kb * kFp8Block + lane * 8;
        Eight<BF16> e;
        e.load((const uint8_t*)x + src * cols * (BF16 ? 2 : 4), col, cols);
        uint32_t bad;
        const uint32_t byte = scale_byte(max_of_16(e.amax(bad)));
        *(uint2*)(q + (int64_t)r * blocks.d * kFp8Block + col) = e.quantized(byte, bad);
        uint8_t* s = scale + (int64_t)r * scale_pitch + kb;
        if (lane == 0)
            *s = (uint8_t)byte;
        else if (kb == blocks.d - 1 && (int)kb + lane < scale_pitch)
            s[lane] = 0;  // the row's fill
    }
}

// A block of 256 threads takes a 128 x 128 block of an expert's weights and keeps it in registers: 16 lanes to a row,
// eight rows a thread.  64 x 1024 x 2048 in bf16 76 us, 5.3 TB/s (a copy of 1 GiB 4.7).
template <bool BF16>
__global__ __launch_bounds__(256) void quantize_weights_kernel(const void* __restrict__ w, uint8_t* __restrict__ q,
                                                               uint8_t* __restrict__ scale, int n_out, int n_in, int n_blocks,
                                                               int scale_pitch, Divisor blocks) {
    __shared__ uint32_t part[4];
    const uint32_t row_block = blocks.divide(blockIdx.x), kb = blockIdx.x - row_block * blocks.d;  // row_block over all experts
    const int e = (int)(row_block / (uint32_t)n_blocks), n0 = (int)(row_block - (uint32_t)e * n_blocks) * kFp8Block;
    const int lane = threadIdx.x & 15, row = threadIdx.x >> 4, col = (int)kb * kFp8Block + lane * 8;
    Eight<BF16> v[8];
    uint32_t bad[8], top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int n = n0 + row + 16 * i;
        v[i].load((const uint8_t*)w + ((int64_t)e * n_out + n) * n_in * (BF16 ? 2 : 4), n < n_out ? col : n_in, n_in);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, v[i].amax(bad[i]));
    top = max_over_rows_of_16(max_of_16(top));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = top;
    __syncthreads();
    const uint32_t byte = scale_byte(max(max(part[0], part[1]), max(part[2], part[3])));
#pragma unroll
    for (int i = 0; i < 8; ++i)
        *(uint2*)(q + ((int64_t)row_block * kFp8Block + row + 16 * i) * blocks.d * kFp8Block + col) = v[i].quantized(byte, bad[i]);
    uint8_t* s = scale + (int64_t)row_block * scale_pitch + kb;
    if (threadIdx.x == 0)
        *s = (uint8_t)byte;
    else if (kb == blocks.d - 1 && (int)(kb + threadIdx.x) < scale_pitch)
        s[threadIdx.x] = 0;
}

hipError_t launch_quantize_rows(int dtype, const void* x, int64_t n_rows, int cols, const int32_t* row_token,
                                const int32_t* row_count, void* q, uint8_t* scale, hipStream_t st) {
    const Divisor blocks((uint32_t)fp8_blocks(cols));
    const int64_t groups = n_rows * blocks.d;
    // (8192 x 4096 bf16: 18.6 us with up to 16384 blocks, 16.3, 6.2 TB/s, with 4096; fp32 29.0 and 30.2; two or four blocks of values
    // requested at once are no faster)
    const dim3 grid((unsigned)std::min<int64_t>((groups + 15) / 16, dtype == MOE_DTYPE_BF16 ? 4096 : 16384));
    auto kern = dtype == MOE_DTYPE_BF16 ? quantize_rows_kernel<true> : quantize_rows_kernel<false>;
    hipLaunchKernelGGL(kern, grid, dim3(256), 0, st, x, row_token, row_count, (uint8_t*)q, scale, n_rows, cols, fp8_scale_pitch(cols),
                       blocks);
    return hipGetLastError();
}

hipError_t launch_quantize_weights(int dtype, const void* w, int experts, int n_out, int n_in, void* q, uint8_t* scale,
                                   hipStream_t st) {
    const Divisor blocks((uint32_t)fp8_blocks(n_in));
    const int n_blocks = fp8_blocks(n_out);
    auto kern = dtype == MOE_DTYPE_BF16 ? quantize_weights_kernel<true> : quantize_weights_kernel<false>;
    hipLaunchKernelGGL(kern, dim3((unsigned)((int64_t)experts * n_blocks * blocks.d)), dim3(256), 0, st, w, (uint8_t*)q, scale, n_out,
                       n_in, n_blocks, fp8_scale_pitch(n_in), blocks);
    return hipGetLastError();
}

}  // namespace capmoe
