// What the kernels share that read rows of activations or weights and write them in 8 or 4 bits.
#pragma once

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

constexpr double kL2Bytes = 32 << 20;  // of the eight XCDs together

// ONCE: the line is not kept in the caches.
template <bool ONCE>
__device__ __forceinline__ uint4 load16(const void* p) {
    if constexpr (ONCE) {
        typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
        const u32x4 v = __builtin_nontemporal_load((const u32x4*)p);
        return make_uint4(v[0], v[1], v[2], v[3]);
    } else {
        return *(const uint4*)p;
    }
}
template <bool ONCE>
__device__ __forceinline__ void store16(void* p, const uint4& v) {
    if constexpr (ONCE) {
        typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
        __builtin_nontemporal_store(u32x4{v.x, v.y, v.z, v.w}, (u32x4*)p);
    } else {
        *(uint4*)p = v;
    }
}

// Eight values of a lane, of a row that begins at x and has `cols` of them, from column col; zeros behind the row's end.
template <bool BF16>
struct Eight {
    uint32_t v[BF16 ? 4 : 8];
    template <bool ONCE = false>
    __device__ __forceinline__ void load(const void* row, int col, int cols) {
        if (BF16) {
            uint4 p = make_uint4(0, 0, 0, 0);
            if (col < cols) p = load16<ONCE>((const uint16_t*)row + col);
            v[0] = p.x, v[1] = p.y, v[2] = p.z, v[3] = p.w;
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint4 p = make_uint4(0, 0, 0, 0);
                if (col + 4 * h < cols) p = load16<ONCE>((const float*)row + col + 4 * h);
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

}  // namespace capmoe
