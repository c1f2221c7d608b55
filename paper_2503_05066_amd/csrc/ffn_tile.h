// What the kernels of the expert products on high row tiles share (ffn.hip: bf16, fp8.hip: 8 bits): the block tile and its LDS
// layout, the requests that fill it, the order of the work, and what becomes of the accumulators.
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

// What a wave needs to request its pieces of a K slab: one buffer descriptor per operand tensor (the
// block's activation rows, its weight rows, and for SwiGLU tiles the up-projection rows) and one 32-bit
// byte offset per wave-wide load.  The loads are MUBUF loads with an LDS destination: unlike the global
// (FLAT-encoded) form, the compiler does not count them against the LDS counter, so the operand reads of the
// matrix loop keep fine-grained waits; the K advance goes into the scalar offset.
// Each descriptor opens the block's own window of a tensor (its activation rows, its weight rows), so
// 32-bit byte offsets suffice whatever the tensor size; with a gather list the window is the whole
// unpermuted input, whose size the host checks.
template <class S>
struct Fills {
    __amdgpu_buffer_rsrc_t a, b0, b1;
    uint32_t va[S::A_LOADS], vb[S::B_LOADS];
    int first, slabs, turn;
    uint8_t* smem;
    int wv;

    __device__ __forceinline__ void weights_of_lane(int lane, int K) {  // the same for every item
#pragma unroll
        for (int i = 0; i < S::B_LOADS; ++i) {
            const int r = (wv + S::NW * i) * 8 + lane / 8, kc = (lane % 8) ^ ((r >> 1) & 7);
            const int rb = S::SWIGLU && r >= S::BN / 2 ? r - S::BN / 2 : r;  // the up-projection rows of the same hidden columns
            vb[i] = ((uint32_t)rb * (uint32_t)K + kc * 8) * 2u;
        }
    }
    __device__ __forceinline__ void aim(const WorkItem& w, const uint16_t* A, const uint16_t* B0, const uint16_t* B1,
                                        const int32_t* gather, int lane, int K, int Nout) {
        a = __builtin_amdgcn_make_buffer_rsrc((void*)(gather ? A : A + (size_t)w.row0 * K), 0, -1, kRsrcFlags);
        b0 = __builtin_amdgcn_make_buffer_rsrc((void*)(B0 + ((size_t)w.e * Nout + w.n0) * K), 0, -1, kRsrcFlags);
        b1 = S::SWIGLU ? __builtin_amdgcn_make_buffer_rsrc((void*)(B1 + ((size_t)w.e * Nout + w.n0) * K), 0, -1, kRsrcFlags) : b0;
        first = w.first;
        slabs = w.slabs;
        turn = w.turn;
        uint32_t row[S::A_LOADS];
#pragma unroll
        for (int i = 0; i < S::A_LOADS; ++i) {
            const int r = (wv + S::NW * i) * 8 + lane / 8;
            const int rr = r < w.rows ? r : w.rows - 1;  // rows past the expert's end repeat its last row
            row[i] = gather ? (uint32_t)gather[w.row0 + rr] : (uint32_t)rr;
        }
#pragma unroll
        for (int i = 0; i < S::A_LOADS; ++i) {
            const int r = (wv + S::NW * i) * 8 + lane / 8, kc = (lane % 8) ^ ((r >> 1) & 7);
            va[i] = (row[i] * (uint32_t)K + kc * 8) * 2u;
        }
    }
    __device__ __forceinline__ uint32_t k_bytes(int kt) const {
        kt += turn;
        kt = kt < slabs ? kt : kt - slabs;
        return (uint32_t)(kt + first) * (S::BK * 2);
    }
    // load i of slab kt's activations / weights into the slot that begins at byte `slot` of LDS
    __device__ __forceinline__ void one_a(int i, int kt, int slot) const {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(a, (lptr_t)(smem + slot + (wv + S::NW * i) * 1024), 16, va[i], k_bytes(kt), 0, 0);
    }
    __device__ __forceinline__ void one_b(int i, int kt, int slot, bool once) const {
        // i and once are compile-time constants after unrolling
        uint8_t* dst = smem + slot + (wv + S::NW * i) * 1024;
        const __amdgpu_buffer_rsrc_t r = S::SWIGLU && i >= S::B_LOADS / 2 ? b1 : b0;
        if (once)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lptr_t)dst, 16, vb[i], k_bytes(kt), 0, 2);  // bit 1: non-temporal
        else
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lptr_t)dst, 16, vb[i], k_bytes(kt), 0, 0);
    }
    // The first slabs of an item, as many as its loop keeps in LDS.  Returns how many requests are younger than those of the
    // first slab.
    __device__ __forceinline__ int start(int live, bool once) const {
        const int n = min(S::ring(live), slabs);
        for (int kt = 0; kt < n; ++kt) {
            const int sa = kt * S::a_stride(live), sb = S::b_base(live) + kt * S::b_stride(live);
            if (once) {
#pragma unroll
                for (int i = 0; i < S::B_LOADS; ++i) one_b(i, kt, sb, true);
            } else {
#pragma unroll
                for (int i = 0; i < S::B_LOADS; ++i) one_b(i, kt, sb, false);
            }
#pragma unroll
            for (int i = 0; i < S::A_LOADS; ++i)
                if (i < live) one_a(i, kt, sa);
            __builtin_amdgcn_sched_barrier(0);  // their order is what the waits count
        }
        return (n - 1) * (S::B_LOADS + live);
    }
};

// a read-only word that is the same for the whole wave, through the scalar cache (written by earlier kernels only)
__device__ __forceinline__ int scalar_word(const int32_t* p, int i) {
    return ((const __attribute__((address_space(4))) int32_t*)(uintptr_t)p)[i];
}

// A word of LDS for another wave or from one.  (Through a generic pointer it would be a FLAT access, which waits for the
// vector-memory counter as well: the whole round trip and all younger requests, with nothing else on the SIMD to run.)
typedef __attribute__((address_space(3))) volatile int* lds_int_t;
__device__ __forceinline__ lds_int_t lds_word(uint8_t* smem, int at) { return (lds_int_t)(smem + at); }

// Decode a block's position in a list of `total` = tiles x column blocks work items, ordered
// [column group][row tile][column in group].
__device__ inline void decode_item(int logical, int nt, int col_group, int& tile, int& nb) {
    const int per_group = nt * col_group;
    const int cg = logical / per_group, rem = logical - cg * per_group;
    tile = rem / col_group;
    nb = cg * col_group + (rem - tile * col_group);
}

// The order of the work.  Every XCD (block id mod 8) gets a contiguous eighth of it, so that blocks that run together on an
// XCD share row and weight tiles in its L2, and its blocks take the next position of that eighth as they get free.
//
// split_hdr[4] set (see the tile schedule: a long launch that is never cut along K): the blocks walk the list
// that holds both kinds expert by expert, so the short tiles of an expert run next to its big tiles and their
// weight streaming overlaps matrix work.
//
// Otherwise the two lists one after the other: the XCD's eighth of the big items, then its eighth of the short
// ones (longest first; ordered by height instead, with an eighth of every height for each XCD, the items that stream weights
// no longer ran beside those that multiply: 279 -> 297 and 419 -> 456 us).  The last split_hdr[0] big items of an XCD's
// share run as split_hdr[1] units each; the units follow the XCD's whole items, slice by slice, so that the units that run
// together read the same K range of the tiles they share.  A GEMM too short in K to be cut there runs the few big items left
// over after the XCD's last full round (split_hdr[6]) as kFfnRowPieces quarters of their rows each: twice the compute-unit
// time, on compute units that would have idled, in half the item's time.
//
// The last split_hdr[5] items of the order (of the joint list, or of the short items) are not dealt out in eighths: whichever
// XCD has a compute unit free takes the next one, so that an XCD that runs a few per cent slower than the others
// (they differ) does not end the launch alone.
template <class S>
struct WorkOrder {
    const TileListArgs& L;
    int slabs, Nout, group_big, group_short, xcd;
    bool stream;
    bool joint;
    int nt_big, nt_short;        // row tiles (joint: all of them in nt_big)
    int base_big, base_short;    // first item of this XCD's eighth
    int whole, pieces, whole_s, units, units_s;  // positions of each kind, in this order
    int cut, cut_here, slices, cut_s, cut_s_here, slices_s;
    int fixed, pool;             // joint, short items: those dealt out in eighths, those shared at the end
    int few_big;                 // less than a round of big items

    __device__ __forceinline__ WorkOrder(const TileListArgs& lists, const int32_t* hdr, int K, int Nout_, int gb, int gs, bool stream_)
        : L(lists), slabs(K / S::BK), Nout(Nout_), group_big(gb), group_short(gs), xcd(blockIdx.x & 7), stream(stream_) {
        const int ncol = Nout / S::kNCols;
        // everything at once: a block that starts waits for one fetch, not for one after the other
        int h[7];
#pragma unroll
        for (int i = 0; i < 7; ++i) h[i] = scalar_word(hdr, i);
        const int n_all = scalar_word(L.u_count, 0), n_big = scalar_word(L.b_count, 0), n_short = scalar_word(L.s_count, 0);
        joint = h[4];
        pool = h[5];
        pieces = whole_s = units = units_s = 0;
        cut = cut_here = cut_s = cut_s_here = 0;
        slices = slices_s = 1;
        nt_short = base_short = fixed = few_big = 0;
        if (joint) {
            nt_big = n_all;
            fixed = nt_big * ncol - pool;
            const int chunk = (fixed + 7) >> 3;
            base_big = xcd * chunk;
            whole = max(0, min(chunk, fixed - base_big));
        } else {
            nt_big = n_big, nt_short = n_short;
            cut = h[0], slices = h[1];
            cut_s = h[2], slices_s = h[3];
            const int in_rows = h[6];
            const int total_b = nt_big * ncol, total_s = nt_short * ncol;
            fixed = total_s - pool;
            const int chunk_b = (total_b + 7) >> 3, chunk_s = (fixed + 7) >> 3;
            few_big = chunk_b <= kFfnSplitUnits / 8;
            base_big = xcd * chunk_b, base_short = xcd * chunk_s;
            const int mine = max(0, min(chunk_b, total_b - base_big)), mine_s = max(0, min(chunk_s, fixed - base_short));
            whole = min(mine, chunk_b - cut - in_rows);
            whole_s = min(mine_s, chunk_s - cut_s);
            pieces = in_rows > 0 ? (mine - whole) * kFfnRowPieces : 0;
            cut_here = cut > 0 ? mine - whole : 0, cut_s_here = mine_s - whole_s;
            units = cut_here * slices, units_s = cut_s_here * slices_s;
        }
    }
    __device__ __forceinline__ int positions() const { return whole + pieces + whole_s + units + units_s; }

    // position p of this XCD's share, or item p - kPoolItem of the shared end of the order
    static constexpr int kPoolItem = 1 << 30;
    __device__ __forceinline__ WorkItem at(int p) const {
        WorkItem w;
        w.valid = 0;
        int logical, rows_word, tile, nb, quarter = -1, alone;
        w.slices = 1, w.slice = w.unit = w.stride = w.ticket = w.short_unit = 0;
        bool is_short = false;  // of the list of short tiles
        if (p >= kPoolItem) {
            if (p - kPoolItem >= pool) return w;
            logical = fixed + p - kPoolItem;
            is_short = !joint;
        } else if (p < whole) {
            logical = base_big + p;
        } else if ((p -= whole) < pieces) {
            logical = base_big + whole + p / kFfnRowPieces;
            quarter = p % kFfnRowPieces;
        } else if ((p -= pieces) < whole_s) {
            logical = base_short + p;
            is_short = true;
        } else if ((p -= whole_s) < units) {
            w.slices = slices, w.stride = cut;
            w.slice = p / cut_here;
            const int idx = p - w.slice * cut_here;
            logical = base_big + whole + idx;
            w.unit = w.ticket = xcd * (kFfnSplitUnits / 8) + idx;
        } else if ((p -= units) < units_s) {
            w.slices = slices_s, w.stride = cut_s;
            w.slice = p / cut_s_here;
            const int idx = p - w.slice * cut_s_here;
            logical = base_short + whole_s + idx;
            w.unit = xcd * (kFfnSplitUnits / 8) + idx;
            w.ticket = kFfnSplitUnits + w.unit;
            is_short = true, w.short_unit = 1;
        } else {
            return w;
        }
        if (is_short)
            decode_item(logical, nt_short, group_short, tile, nb);
        else
            decode_item(logical, nt_big, group_big, tile, nb);
        // uniform, also where the divisions ran on the vector unit
        tile = __builtin_amdgcn_readfirstlane(tile), nb = __builtin_amdgcn_readfirstlane(nb);
        w.valid = 1;
        w.n0 = nb * S::kNCols;
        w.e = scalar_word(is_short ? L.s_expert : (joint ? L.u_expert : L.b_expert), tile);
        w.row0 = scalar_word(is_short ? L.s_row0 : (joint ? L.u_row0 : L.b_row0), tile);
        rows_word = scalar_word(is_short ? L.s_rows : (joint ? L.u_rows : L.b_rows), tile);
        w.rows = rows_word & kTileRowsMask;
        alone = stream && (rows_word & kAloneTileFlag);
        if (is_short)
            // with less than a round of big items those of the same expert run beside it and read the same weights (314 tokens,
            // all at 8 experts x 3840 x 640: 169 -> 155 us)
            w.once = stream && (alone || !few_big || w.slices > 1);
        else
            w.once = w.slices > 1 ? 0 : (quarter >= 0 ? stream : alone);
        if (quarter >= 0) {  // a big tile has more than 64 rows: no quarter is empty
            const int from = quarter * w.rows / kFfnRowPieces, to = (quarter + 1) * w.rows / kFfnRowPieces;
            w.row0 += from;
            w.rows = to - from;
        }
        w.first = 0;
        w.slabs = slabs;
        if (w.slices > 1) {  // (a division is forty instructions, and nothing runs beside a launch's first look-up)
            w.first = w.slice * slabs / w.slices;
            w.slabs = (w.slice + 1) * slabs / w.slices - w.first;
        }
        // The start of the walk depends on the output columns alone and only moves where the expert has a single tile: in a
        // GEMM that is not cut along K a row's sums run in the same order whatever other experts share the launch.  (Which
        // items are cut follows from the tiles of all experts.)
        w.turn = alone && w.once ? (int)((long long)w.n0 * w.slabs / Nout) : 0;
        return w;
    }
};

// Writes sub-tile row j (16 rows of this wave) of a block's output tile: a lane holds 4 consecutive columns of a row in each
// sub-tile; the lanes exchange halves between two sub-tiles (v_permlane16_swap), hold 16 bytes each, and a wave's store writes
// 64 consecutive bytes of 16 rows.  Nothing passes through LDS, which by then receives the next item's first slabs.  Rows past
// the tile's end lie past the end of the descriptor's window and are not written: the number of stores is the same for all.
template <class S>
struct TileWriter {
    __amdgpu_buffer_rsrc_t c;
    uint32_t at;      // byte offset of this lane's first column in row 0
    uint32_t pitch;   // bytes of a row
    __device__ __forceinline__ TileWriter(uint16_t* C, const WorkItem& w, int Nout, int wm, int wn, int lane) {
        c = __builtin_amdgcn_make_buffer_rsrc((void*)(C + (size_t)w.row0 * Nout + w.n0), 0,
                                              ((w.rows - 1) * Nout + S::kNCols) * 2, kRsrcFlags);
        const int lr = lane & 15, lk = lane >> 4;
        pitch = (uint32_t)Nout * 2u;
        at = (uint32_t)(wm * 16 + lr) * pitch + (uint32_t)(wn * (S::kNCols / 2) + (lk & 1) * 16 + (lk >> 1) * 8) * 2u;
    }
    template <class Frag>
    __device__ __forceinline__ void rows(int j, Frag&& frag) const {  // frag(i): sub-tile i's values, i a compile-time argument
        each<S::TNO / 2>([&](auto pair_c) {
            constexpr int i = 2 * decltype(pair_c)::value;
            uint32_t half[2][2];
            each<2>([&](auto s_c) {
                constexpr int s = decltype(s_c)::value;
                const f32x4 g = frag(std::integral_constant<int, i + s>{});
                float o[4];
                if constexpr (S::SWIGLU) {
                    const f32x4 u = frag(std::integral_constant<int, i + s + S::TNO>{});
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        o[v] = g[v] * u[v] * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g[v] * -1.4426950408889634f));
                } else {
#pragma unroll
                    for (int v = 0; v < 4; ++v) o[v] = g[v];
                }
                half[s][0] = pack_bf16x2(o[0], o[1]);
                half[s][1] = pack_bf16x2(o[2], o[3]);
            });
            const auto lo = __builtin_amdgcn_permlane16_swap(half[0][0], half[1][0], false, false);
            const auto hi = __builtin_amdgcn_permlane16_swap(half[0][1], half[1][1], false, false);
            const u32x4 out = {lo[0], hi[0], lo[1], hi[1]};
            __builtin_amdgcn_raw_buffer_store_b128(out, c, at + (uint32_t)(j * 32) * pitch + i * 32, 0, 0);
        });
    }
};

// An item cut along K: partial tiles through the workspace; of the waves that hold the same part of the item's units, the last
// one to finish adds them and writes the output.
// The units of an item may run on different XCDs, whose L2 caches do not see each other's lines.  A fence
// that writes back and invalidates a whole L2 per unit costs more than the cut saves, so the partial tiles
// are stored and loaded with device-scope cache policy instead (written through to memory, read around
// caches that may be stale), each store is acknowledged before the ticket is taken, and the ticket is a
// device-scope atomic (a byte of it for each of the four waves).
template <class S>
__device__ __forceinline__ void finish_unit(const WorkItem& w, const TileWriter<S>& out,
                                            float* split_partial, int32_t* split_counter, int wv, int lane, int live) {
    constexpr int TN = S::TN, TM = S::TM;
    // a unit's partial tile is stored in register order (fragment, lane): whole 1 KB lines per wave store
    const size_t unit_floats = (size_t)(w.short_unit ? kFfnTileSmall : S::BM) * S::BN;
    float* item = split_partial + (w.short_unit ? (size_t)kFfnSplitUnits * kFfnTileM * 256 : 0) + (size_t)w.unit * unit_floats;
    // (a short item has two live sub-tiles at most: its fragments are packed)
    const int height = w.short_unit ? kFfnTileSmall / 32 : TM;
    const uint32_t at = (uint32_t)((wv * TN * height * 64 + lane) * 16);  // + fragment * 1024 bytes
    {
        const __amdgpu_buffer_rsrc_t mine = __builtin_amdgcn_make_buffer_rsrc(
            (void*)(item + (size_t)(w.slice * w.stride) * unit_floats), 0, -1, kRsrcFlags);
        each<TM>([&](auto j_c) {
            constexpr int j = decltype(j_c)::value;
            if (j < live)
                each<TN>([&](auto i_c) {
                    constexpr int i = decltype(i_c)::value;
                    const f32x4 v = acc_read<S::fragment(i, j)>();
                    __builtin_amdgcn_raw_buffer_store_b128(*(const u32x4*)&v, mine, at + (j * TN + i) * 1024, 0, kDeviceScope);
                });
        });
    }
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));  // every store of this lane has been acknowledged
    int order = 0;
    if (lane == 0) order = __hip_atomic_fetch_add(split_counter + w.ticket, 1 << (8 * wv), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    order = (__builtin_amdgcn_readfirstlane(order) >> (8 * wv)) & 255;
    if (order != w.slices - 1) return;  // another unit of this item finishes later and does the sum
    const __amdgpu_buffer_rsrc_t all = __builtin_amdgcn_make_buffer_rsrc((void*)item, 0, -1, kRsrcFlags);
    const uint32_t unit_bytes = (uint32_t)(w.stride * unit_floats * 4);
#pragma unroll 1
    for (int j = 0; j < live; ++j) {
        f32x4 sum[TN];
#pragma unroll
        for (int i = 0; i < TN; ++i) sum[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
        for (int s0 = 0; s0 < w.slices; s0 += 4) {  // slice order, whichever unit does it: the same sum every run
            // four slices in flight at a time: a load that goes around the caches takes microseconds
            u32x4 q[4][TN];
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < TN; ++i)
                    q[t][i] = __builtin_amdgcn_raw_buffer_load_b128(
                        all, at + (j * TN + i) * 1024, (uint32_t)(s0 + t < w.slices ? s0 + t : s0) * unit_bytes, kDeviceScope);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if (s0 + t < w.slices) {
#pragma unroll
                    for (int i = 0; i < TN; ++i) sum[i] += *(const f32x4*)&q[t][i];
                }
        }
        out.rows(j, [&](auto i_c) { return sum[decltype(i_c)::value]; });
    }
}

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

// Tickets of the blocks of an XCD lie in the last of its split units' tickets, that of the shared end in the last ticket of
// the short items: at most kFfnSplitUnits / 8 - 1 items of an XCD are cut (what is left after full rounds).
constexpr int kXcdTicket = kFfnSplitUnits / 8 - 1, kPoolTicket = kFfnSplitUnits + kFfnSplitUnits / 8 - 1;

// The three tile lists of a workspace as the kernels take them; joint == false leaves the joint list unwritten
// (the fp32 kernels walk the list of big tiles only).
inline TileListArgs tile_list_args(const FfnWorkspace& ws, bool joint) {
    return TileListArgs{ws.big.expert, ws.big.row0,  ws.big.rows,      ws.big.count,       ws.small.expert,
                        ws.small.row0, ws.small.rows, ws.small.count,   ws.big.max_tiles,   ws.small.max_tiles,
                        ws.all.expert, ws.all.row0,  ws.all.rows,      ws.all.count,       joint ? ws.all.max_tiles : 0};
}

inline int column_group(int nb_total) {
    for (int g = 4; g > 1; --g)
        if (nb_total % g == 0) return g;
    return 1;
}

}  // namespace capmoe
