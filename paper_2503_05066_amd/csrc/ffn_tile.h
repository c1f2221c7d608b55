// What the kernels of the expert products on high row tiles share (ffn.hip: bf16, fp8.hip: 8 bits): the block tile, an item of
// work, the accumulators, single words of LDS and of memory, waits.
//
// Lengths along K count 16-bit units, whatever the elements are: a K slab is 64 units, 128 bytes of a row.
#pragma once

#include <type_traits>
#include <utility>

#include "common.h"
#include "schedule.h"

namespace capmoe {

// two floats -> two bf16 (round to nearest even) in one word, lo in the low half: the hardware conversion
typedef __attribute__((ext_vector_type(2))) float f32x2_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
__device__ inline uint32_t pack_bf16x2(float lo, float hi) {
    const f32x2_t v = {lo, hi};
    const bf16x2_t b = __builtin_convertvector(v, bf16x2_t);
    return *(const uint32_t*)&b;
}

typedef __attribute__((address_space(3))) void* lptr_t;

// s_waitcnt immediate for "at most n vector-memory operations outstanding, LDS/scalar counter
// at zero" (gfx9 encoding: vmcnt in bits 3:0 and 15:14, expcnt 6:4 left at 7, lgkmcnt 11:8).
__host__ __device__ constexpr int waitcnt_vm(int n) { return (n & 15) | (7 << 4) | ((n >> 4) << 14); }

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;

constexpr int kRsrcFlags = 0x00020000;  // raw buffer of 32-bit words, no swizzle (gfx9 descriptor word 3)
constexpr int kDeviceScope = 16;        // cache policy bit sc1 of the buffer instructions

// f(0), f(1), .. f(N - 1) with compile-time arguments
template <class F, int... Is>
__device__ __forceinline__ void each_of(std::integer_sequence<int, Is...>, F&& f) {
    (f(std::integral_constant<int, Is>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void each(F&& f) {
    each_of(std::make_integer_sequence<int, N>{}, f);
}

// The accumulators have fixed places (see ffn.hip): fragment F in a[4F .. 4F+3].
template <int F>
__device__ __forceinline__ void acc_zero() {
    asm volatile(
        "v_accvgpr_write_b32 a[%0], 0\n\tv_accvgpr_write_b32 a[%1], 0\n\t"
        "v_accvgpr_write_b32 a[%2], 0\n\tv_accvgpr_write_b32 a[%3], 0" ::"n"(4 * F), "n"(4 * F + 1), "n"(4 * F + 2), "n"(4 * F + 3));
}
template <int F>
__device__ __forceinline__ f32x4 acc_read() {
    f32x4 c;
    asm volatile("v_accvgpr_read_b32 %0, a[%1]" : "=v"(c[0]) : "n"(4 * F));
    asm volatile("v_accvgpr_read_b32 %0, a[%1]" : "=v"(c[1]) : "n"(4 * F + 1));
    asm volatile("v_accvgpr_read_b32 %0, a[%1]" : "=v"(c[2]) : "n"(4 * F + 2));
    asm volatile("v_accvgpr_read_b32 %0, a[%1]" : "=v"(c[3]) : "n"(4 * F + 3));
    return c;
}

// The block tile: 256 activation rows x BN weight rows over 64-wide K slabs, 2 x 2 waves.
//
// LDS rows are 128 bytes (64 bf16).  They are filled by direct global->LDS loads: one wave-wide load writes
// 1 KB of consecutive LDS (64 lanes x 16 bytes = 8 rows), and each lane chooses WHICH 16-byte piece of its
// row it fetches, so that piece kc of row r lands at position kc ^ ((r >> 1) & 7): with the 64 LDS banks of
// this chip, the 16 lanes that a 16-byte read serves per cycle then fall into 16 different bank groups, for
// the fill as well as for the operand reads.  Lane l reads row (l & 15), piece (l >> 4) of a k-step and ends
// with output columns 4*(l >> 4) .. +3 of activation row (l & 15) of each 16 x 16 sub-tile.
//
// The waves of a column take the 16-row activation sub-tiles in turn, so that a partly filled tile keeps all four waves
// multiplying: its time follows its rows in steps of 32.  (With halves of a tile instead, 128 x 2048 x 768 with 129 to 200
// rows on most experts 638 -> 618 us a layer, 60 x 2048 x 1408 with at most 127 227 -> 224.)
//
// SWIGLU: weight rows [0,BN/2) of the tile come from W_gate, [BN/2,BN) from W_up, for the same BN/2 hidden
// columns; a wave holds matching gate and up columns and applies silu(g)*u itself.
template <int BN_, bool SWIGLU_>
struct Shape {
    static constexpr int BM = kFfnTileM, BN = BN_, NW = 4, BK = 64;
    static constexpr bool SWIGLU = SWIGLU_;
    static constexpr int kThreads = 64 * NW;
    static constexpr int kNCols = SWIGLU ? BN / 2 : BN;  // output columns of a block
    static constexpr int TM = BM / 2 / 16, TN = BN / 2 / 16;
    static constexpr int A_LOADS = BM / 8 / NW, B_LOADS = BN / 8 / NW;  // wave-wide loads of eight 128-byte rows per slab
    static constexpr int A_SLOT = BM * 128, B_SLOT = BN * 128, B_BASE = 2 * A_SLOT;
    static constexpr int kLdsBytes = 2 * A_SLOT + 3 * B_SLOT;
    // Slabs in LDS for a tile of `live` x 32 rows: up to five of these, activations and weights of a slab lie side by side in a
    // ring of three slots, up to two in a ring of four; above, two slots of activations and three of weights.
    static constexpr int kRingLive = 5;
    static __host__ __device__ constexpr int ring(int live) { return live <= 2 ? 4 : (live <= kRingLive ? 3 : 2); }
    static __host__ __device__ constexpr int a_stride(int live) { return live <= kRingLive ? live * 4096 + B_SLOT : A_SLOT; }
    static __host__ __device__ constexpr int b_stride(int live) { return live <= kRingLive ? live * 4096 + B_SLOT : B_SLOT; }
    static __host__ __device__ constexpr int b_base(int live) { return live <= kRingLive ? live * 4096 : B_BASE; }
    static_assert(4 * (2 * 4096 + B_SLOT) <= kLdsBytes && 3 * (kRingLive * 4096 + B_SLOT) <= kLdsBytes, "rings");
    static constexpr int TNO = SWIGLU ? TN / 2 : TN;  // 16-column output sub-tiles of a wave
    static constexpr int fragment(int i, int j) { return i * TM + j; }  // of weight sub-tile i, activation sub-tile j
    static_assert(TNO % 2 == 0 && B_LOADS % 2 == 0, "sub-tiles leave in pairs; a load must not straddle two tensors");
};

// Which part of the product a block does next (uniform over the block).
struct WorkItem {
    int valid;
    int e, row0, rows, n0;  // output rows [row0, row0 + rows) of expert e, output columns from n0
    int first, slabs;       // its K slabs (all of them unless the item is cut along K)
    int turn;               // the slab of these that the walk begins with (it wraps around)
    int once;               // the weights are fetched with the non-temporal policy
    int slices, slice;      // units of an item that is cut along K (1: not cut)
    int unit, stride;       // where this unit's partial tile lies: unit of slice 0, units between slices
    int ticket;             // index of the item's ticket
    int short_unit;         // its partial tiles are in the region of the short items
};

// a read-only word that is the same for the whole wave, through the scalar cache (written by earlier kernels only)
__device__ __forceinline__ int scalar_word(const int32_t* p, int i) {
    return ((const __attribute__((address_space(4))) int32_t*)(uintptr_t)p)[i];
}

// A word of LDS for another wave or from one.  (Through a generic pointer it would be a FLAT access, which waits for the
// vector-memory counter as well: the whole round trip and all younger requests, with nothing else on the SIMD to run.)
typedef __attribute__((address_space(3))) volatile int* lds_int_t;
__device__ __forceinline__ lds_int_t lds_word(uint8_t* smem, int at) { return (lds_int_t)(smem + at); }

// Waits until at most n memory operations of this wave are outstanding (the instruction takes a constant).
__device__ __forceinline__ void wait_for_all_but(int n) {
    switch (n) {
#define CAPMOE_WAIT(k) \
    case k: __builtin_amdgcn_s_waitcnt(waitcnt_vm(k)); break;
#define CAPMOE_WAIT8(k) \
    CAPMOE_WAIT(k) CAPMOE_WAIT(k + 1) CAPMOE_WAIT(k + 2) CAPMOE_WAIT(k + 3) CAPMOE_WAIT(k + 4) CAPMOE_WAIT(k + 5) \
    CAPMOE_WAIT(k + 6) CAPMOE_WAIT(k + 7)
        CAPMOE_WAIT8(0) CAPMOE_WAIT8(8) CAPMOE_WAIT8(16) CAPMOE_WAIT8(24) CAPMOE_WAIT8(32) CAPMOE_WAIT8(40) CAPMOE_WAIT8(48)
        CAPMOE_WAIT8(56)
#undef CAPMOE_WAIT8
#undef CAPMOE_WAIT
        default: __builtin_amdgcn_s_waitcnt(waitcnt_vm(0)); break;
    }
}

}  // namespace capmoe
