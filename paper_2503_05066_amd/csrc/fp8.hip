// Products on 8-bit rows and 8-bit expert weights, grouped by expert, on high row tiles (fp8_thin.hip has the few-row ones).
//
//   y[r,n] = sum over blocks b of 128 k:  2^(xs[r,b] + ws[e,n/128,b] - 254) * sum over k in b: x[r,k] w[e,n,k]
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 128 k at once and applies a power of two for each 32 k of each row of both
// operands, so the scales cost the vector unit nothing but their distribution, and the sums stay in the accumulation
// registers (a scale of any fp32 value would take one fused multiply-add per output and block, half of the matrix time).
// Registers alone sustain 4.17 PFLOP/s of it on random operands (without scales 4.26; 32x32x64 3.83).
//
// Tiles, LDS layout, requests and the order of the work are those of the bf16 kernel (ffn_tile.h): a row's slab is 128
// bytes there, 64 k, and here, 128 k, so a slab moves the same bytes in the same time and multiplies twice as much.
// Lane l takes pieces l >> 4 and (l >> 4) + 4 (16 bytes each) of row l & 15 of both operands, which numbers the k of a
// slab alike in both.
#include <algorithm>

#include "ffn_tile.h"
#include "fp8.h"

namespace capmoe {

typedef __attribute__((ext_vector_type(8))) int i32x8;

template <int F>
__device__ __forceinline__ void acc_mfma8(const i32x8& w, const i32x8& x, uint32_t w_scale, uint32_t x_scale) {
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 a[%0:%1], %2, %3, a[%0:%1], %4, %5 op_sel_hi:[0,0,0]" ::"n"(4 * F),
                 "n"(4 * F + 3), "v"(w), "v"(x), "v"(w_scale), "v"(x_scale));
}

// The tile of the bf16 kernel with room for an exchange between waves: up to 2 x 32 rows keep one slab less in flight.
template <int BN_, bool SWIGLU_>
struct Shape8 : Shape<BN_, SWIGLU_> {
    using Base = Shape<BN_, SWIGLU_>;
    static __host__ __device__ constexpr int ring(int live) { return live <= 1 ? 4 : (live <= Base::kRingLive ? 3 : 2); }
    // the last 4 KB of LDS: of low tiles no slot reaches there, of high ones only the third slot of weights, which is
    // first requested in the loop
    static constexpr int kExchange = 160 * 1024 - 4096;
    static_assert(4 * (4096 + Base::B_SLOT) <= kExchange && 3 * (Base::kRingLive * 4096 + Base::B_SLOT) <= kExchange, "exchange");
    static constexpr int kLdsBytes = 160 * 1024;
};

// What a wave needs to request its pieces of a K slab (see Fills in ffn_tile.h) and the scales.
template <class S>
struct Fills8 {
    __amdgpu_buffer_rsrc_t a, b0, b1, sa, sb0, sb1;
    uint32_t va[S::A_LOADS], vb;  // of the weights the rows of load i lie 32 * i rows further
    uint32_t vsa[2];              // scales: of the rows of sub-tiles 0..3 and 4..7, a quarter of the wave each
    int first, slabs, turn;
    uint32_t row_step;            // bytes of 32 weight rows
    uint8_t* smem;
    int wv;

    __device__ __forceinline__ void weights_of_lane(int lane, int pitch) {  // the same for every item
        const int r = wv * 8 + lane / 8, kc = (lane % 8) ^ ((r >> 1) & 7);
        vb = (uint32_t)r * (uint32_t)pitch + kc * 16;
        row_step = 32u * (uint32_t)pitch;
    }
    __device__ __forceinline__ void aim(const WorkItem& w, const Fp8Args& p, int lane, int wm, int wn) {
        const int32_t* gather = p.gather;
        a = __builtin_amdgcn_make_buffer_rsrc((void*)(gather ? p.x : p.x + (size_t)w.row0 * p.pitch), 0, -1, kRsrcFlags);
        sa = __builtin_amdgcn_make_buffer_rsrc((void*)(gather ? p.x_scale : p.x_scale + (size_t)w.row0 * p.scale_pitch), 0, -1, kRsrcFlags);
        const size_t n_at = (size_t)w.e * p.n_pad + w.n0;
        b0 = __builtin_amdgcn_make_buffer_rsrc((void*)(p.w[0] + n_at * p.pitch), 0, -1, kRsrcFlags);
        b1 = S::SWIGLU ? __builtin_amdgcn_make_buffer_rsrc((void*)(p.w[1] + n_at * p.pitch), 0, -1, kRsrcFlags) : b0;
        // a wave's weight rows lie in one block of 128 (with SWIGLU in one of either tensor)
        const size_t s_at = (n_at / kFp8Block + (S::SWIGLU || S::BN == 128 ? 0 : wn)) * p.scale_pitch;
        sb0 = __builtin_amdgcn_make_buffer_rsrc((void*)(p.w_scale[0] + s_at), 0, -1, kRsrcFlags);
        sb1 = S::SWIGLU ? __builtin_amdgcn_make_buffer_rsrc((void*)(p.w_scale[1] + s_at), 0, -1, kRsrcFlags) : sb0;
        first = w.first;
        slabs = w.slabs;
        turn = w.turn;
        uint32_t row[S::A_LOADS], srow[2];
#pragma unroll
        for (int i = 0; i < S::A_LOADS; ++i) {
            const int r = (wv + S::NW * i) * 8 + lane / 8;
            const int rr = r < w.rows ? r : w.rows - 1;  // rows past the expert's end repeat its last row
            row[i] = gather ? (uint32_t)gather[w.row0 + rr] : (uint32_t)rr;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = (4 * h + (lane >> 4)) * 32 + wm * 16 + (lane & 15);
            const int rr = r < w.rows ? r : w.rows - 1;
            srow[h] = gather ? (uint32_t)gather[w.row0 + rr] : (uint32_t)rr;
        }
#pragma unroll
        for (int i = 0; i < S::A_LOADS; ++i) {
            const int r = (wv + S::NW * i) * 8 + lane / 8, kc = (lane % 8) ^ ((r >> 1) & 7);
            va[i] = row[i] * (uint32_t)p.pitch + kc * 16;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) vsa[h] = srow[h] * (uint32_t)p.scale_pitch;
    }
    __device__ __forceinline__ int slab_at(int kt) const {
        kt += turn;
        return (kt < slabs ? kt : kt - slabs) + first;
    }
    __device__ __forceinline__ void one_a(int i, uint32_t k, int slot) const {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(a, (lptr_t)(smem + slot + (wv + S::NW * i) * 1024), 16, va[i], k, 0, 0);
    }
    __device__ __forceinline__ void one_b(int i, uint32_t k, int slot, bool once) const {
        // i and once are compile-time constants after unrolling
        uint8_t* dst = smem + slot + (wv + S::NW * i) * 1024;
        const bool second = S::SWIGLU && i >= S::B_LOADS / 2;
        const __amdgpu_buffer_rsrc_t r = second ? b1 : b0;
        const uint32_t at = k + (uint32_t)(second ? i - S::B_LOADS / 2 : i) * row_step;
        if (once)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lptr_t)dst, 16, vb, at, 0, 2);  // bit 1: non-temporal
        else
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lptr_t)dst, 16, vb, at, 0, 0);
    }
    // The first slabs of an item, as many as its loop keeps whole in LDS.  Returns how many requests are younger than those
    // of the first slab.
    __device__ __forceinline__ int start(int live, bool once) const {
        const int n = min(S::ring(live), slabs);
        for (int kt = 0; kt < n; ++kt) {
            const int sa_ = kt * S::a_stride(live), sb_ = S::b_base(live) + kt * S::b_stride(live);
            const uint32_t k = (uint32_t)slab_at(kt) * 128u;
            if (once) {
#pragma unroll
                for (int i = 0; i < S::B_LOADS; ++i) one_b(i, k, sb_, true);
            } else {
#pragma unroll
                for (int i = 0; i < S::B_LOADS; ++i) one_b(i, k, sb_, false);
            }
#pragma unroll
            for (int i = 0; i < S::A_LOADS; ++i)
                if (i < live) one_a(i, k, sa_);
            __builtin_amdgcn_sched_barrier(0);  // their order is what the waits count
        }
        return (n - 1) * (S::B_LOADS + live);
    }
};

// The scales of four slabs (a dword of scale bytes) at a time: those in use and the next ones, requested four slabs ahead.
template <class S>
struct Scales8 {
    uint32_t raw[2], raw_w[2];    // next: of 64 rows each, a row per lane; of the weights, the same in all lanes
    uint32_t w[2];                // in use
    __device__ __forceinline__ void request(const Fills8<S>& f, int slab, int live) {
        const uint32_t at = (uint32_t)(slab >> 2) * 4u;
        raw[0] = __builtin_amdgcn_raw_buffer_load_b32(f.sa, f.vsa[0], at, 0);
        if (live > 4) raw[1] = __builtin_amdgcn_raw_buffer_load_b32(f.sa, f.vsa[1], at, 0);
        raw_w[0] = __builtin_amdgcn_raw_buffer_load_b32(f.sb0, 0, at, 0);
        if (S::SWIGLU) raw_w[1] = __builtin_amdgcn_raw_buffer_load_b32(f.sb1, 0, at, 0);
    }
    // the slab after the last one that shares its dword with `slab`
    static __device__ __forceinline__ int following(const Fills8<S>& f, int slab) {
        const int next = (slab | 3) + 1;
        return next < f.first + f.slabs ? next : f.first;
    }
};
// v holds a value per lane of four groups of 16: out[g] gets group g's in all four groups
__device__ __forceinline__ void spread(uint32_t v, uint32_t (&out)[4]) {
    const auto half = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    const auto lo = __builtin_amdgcn_permlane16_swap(half[0], half[0], false, false);
    const auto hi = __builtin_amdgcn_permlane16_swap(half[1], half[1], false, false);
    out[0] = lo[0], out[1] = lo[1], out[2] = hi[0], out[3] = hi[1];
}

// K loop of a wave.  LIVE = number of 16-row activation sub-tiles per wave that are fetched and multiplied.
//
// A slab is one matrix instruction per pair of sub-tiles, and its operands (a wave's 128 rows of either side) take 64 registers
// each.  Two sets of both do not fit, so tiles with LIVE above 2 walk a slab in four parts, halves of the activations (A0, A1)
// by halves of the weights (B0, B1), in turn
//     A0 B0 | A1 B0 | A1 B1 | A0 B1      then      A1 B0 | A0 B0 | A0 B1 | A1 B1
// where every half is read anew as soon as its second part is done: B0 of the next slab in the third part, the next slab's
// first half of A in the fourth, the other half of A in the slab's own first part, B1 in its first two.  So a slab leaves LDS
// in the middle of its instructions:
//     parts 1, 2 | barrier kt (slab kt+1 landed, slab kt no longer read) | parts 3, 4 and the requests
// Tiles with fewer rows hold two sets of operands; they read slab kt+1 while they multiply slab kt, behind a barrier that
// lies after the first quarter of its instructions.
// The slots of slab kt are free from barrier kt on: high tiles request the activations of slab kt+2 (two slots) and the weights
// of slab kt+3 (three), low ones all of slab kt+R (see ring).  Requests complete in order: at barrier kt the weights of slab
// kt+2 (the slabs kt+2 .. kt+R-1) may still fly.
template <class S, bool ONCE>
struct MatrixLoop8 {
    const Fills8<S>& fills;
    Scales8<S>& scales;
    int a_lane, b_lane;  // byte offset, inside a slot, of this lane's first piece of the wave's first row

    static __device__ __forceinline__ constexpr int b_tile(int i) {
        return S::SWIGLU ? ((i / (S::TN / 2)) * (S::BN / 2) + (i % (S::TN / 2)) * 16) * 128 : i * 16 * 128;
    }
    // where a slab's operands of this lane lie in LDS: the first and, four pieces further, the second half of a row's 128 bytes
    struct From {
        const uint8_t *lo, *hi;
        __device__ __forceinline__ From(const uint8_t* slot, int lane_at) : lo(slot + lane_at), hi(slot + (lane_at ^ 64)) {}
        __device__ __forceinline__ void fetch(i32x8& to, int at) const {
            const u32x4 a = *(const u32x4*)(lo + at), b = *(const u32x4*)(hi + at);
            to = __builtin_bit_cast(i32x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    };

    // PHASE, draw, before_last: as in ffn.hip
    template <int LIVE, int PHASE, class D, class F>
    __device__ __forceinline__ void run(D&& draw, F&& before_last) {
        constexpr int TN = S::TN, B_LOADS = S::B_LOADS, NM = TN * LIVE;
        constexpr int R = S::ring(LIVE);
        constexpr bool RING = LIVE <= S::kRingLive, PARTS = LIVE > 2;
        constexpr int SETS = PARTS ? 1 : 2;
        constexpr int PER = B_LOADS + LIVE;      // requests per slab
        constexpr int TAIL = RING ? R : 3;       // slabs at the end that run without some of the requests
        constexpr int A_STRIDE = S::a_stride(LIVE), B_STRIDE = S::b_stride(LIVE), B_BASE = S::b_base(LIVE);
        constexpr int SA = RING ? R : 2, SB = RING ? R : 3;
        constexpr int QB = PARTS ? NM / 2 : (NM / 4 > 0 ? NM / 4 : 1);  // instructions ahead of the barrier
        constexpr int TH = TN / 2, H0 = (LIVE + 1) / 2;
        // instruction q of a slab with parity SET: its activation and weight sub-tile, and how many rows of instructions (of
        // consecutive q on one activation sub-tile) come before it
        struct At {
            int j, i, row, first;
        };
        auto walk = [](int set, int q) constexpr {
            if (!PARTS) return At{q / TN, q % TN, q / TN, q % TN == 0};
            const int half[2] = {H0, LIVE - H0}, f = set, n_f = half[f], n_g = half[f ^ 1];
            const int r = q / TH, i = q % TH;  // row of instructions
            const int part = r < n_f ? 0 : (r < LIVE ? 1 : (r < LIVE + n_g ? 2 : 3));
            const int in = r - (part == 0 ? 0 : (part == 1 ? n_f : (part == 2 ? LIVE : LIVE + n_g)));
            const int h = part == 0 || part == 3 ? f : f ^ 1;
            return At{(h == 0 ? 0 : H0) + in, (part < 2 ? 0 : TH) + i, r, i == 0};
        };
        constexpr int ROWS = PARTS ? 2 * LIVE : LIVE;  // rows of instructions
        // operand reads of a slab, in order, and where: item r of `count` between instructions lo and hi
        auto spread_at = [](int r, int count, int lo, int hi) constexpr { return lo + r * (hi - lo) / count; };
        auto before = [spread_at](int q, int count, int lo, int hi) constexpr {  // items that lie ahead of q
            int n = 0;
            while (n < count && spread_at(n, count, lo, hi) < q) ++n;
            return n;
        };
        uint8_t* const smem = fills.smem;
        const int KT = fills.slabs;
        int a_lane = this->a_lane, b_lane = this->b_lane;
        asm volatile("" : "+v"(a_lane), "+v"(b_lane));  // the first operand reads stay here, not ahead of all instances
        i32x8 xa[SETS][LIVE], wb[SETS][TN];
        uint32_t dist[8];  // scale dwords of the sub-tiles' rows

        auto take_scales = [&](int slab) {  // the next four slabs' scales come into use
            uint32_t d4[4];
            spread(scales.raw[0], d4);
#pragma unroll
            for (int j = 0; j < 4; ++j) dist[j] = d4[j];
            if (LIVE > 4) {
                spread(scales.raw[1], d4);
#pragma unroll
                for (int j = 0; j < 4; ++j) dist[4 + j] = d4[j];
            }
            scales.w[0] = scales.raw_w[0];
            if (S::SWIGLU) scales.w[1] = scales.raw_w[1];
            scales.request(fills, Scales8<S>::following(fills, slab), LIVE);
        };
        // item r of what is read ahead of a slab's first instruction (PARTS: its first half of A and B0) or, LATE, in its
        // first parts (the other half of A and B1), in the order of use
        auto read_item = [&](auto set_c, auto late_c, auto r_c, const From& a, const From& b) {
            constexpr int set = decltype(set_c)::value, r = decltype(r_c)::value;
            constexpr bool late = decltype(late_c)::value;
            constexpr int s = PARTS ? 0 : set;
            if constexpr (!PARTS) {
                if constexpr (r == 0)
                    a.fetch(xa[s][0], 0);
                else if constexpr (r <= TN)
                    b.fetch(wb[s][r - 1], b_tile(r - 1));
                else
                    a.fetch(xa[s][r - TN], (r - TN) * 2 * 16 * 128);
            } else {
                constexpr int h = late ? set ^ 1 : set, from = h == 0 ? 0 : H0, n = h == 0 ? H0 : LIVE - H0;
                if constexpr (late ? r < n : r >= TH) {
                    constexpr int j = from + (late ? r : r - TH);
                    a.fetch(xa[0][j], j * 2 * 16 * 128);
                } else {
                    constexpr int i = late ? TH + r - n : r;
                    b.fetch(wb[0][i], b_tile(i));
                }
            }
        };
        auto first_items = [](int set) constexpr { return PARTS ? TH + (set == 0 ? H0 : LIVE - H0) : TN + LIVE; };
        auto late_items = [](int set) constexpr { return PARTS ? TH + (set == 0 ? LIVE - H0 : H0) : 0; };
        auto slot_a = [&](int slot) { return From(smem + slot * A_STRIDE, a_lane); };
        auto slot_b = [&](int slot) { return From(smem + B_BASE + slot * B_STRIDE, b_lane); };
        auto read_first = [&](auto set_c) {
            const From a = slot_a(0), b = slot_b(0);
            each<first_items(decltype(set_c)::value)>([&](auto r_c) { read_item(set_c, std::false_type{}, r_c, a, b); });
        };
        int kt = 0, sa = 0, sb = 0;
        // One slab.  T < 0: all requests are made; otherwise TAIL - T slabs are left, this one included.
        auto slab = [&](auto set_c, auto tail_c) {
            constexpr int SET = decltype(set_c)::value, T = decltype(tail_c)::value;
            constexpr bool MORE = T < TAIL - 1;
            constexpr bool FILL_A = T < 0 || (!RING && T == 0), FILL_B = T < 0;
            constexpr int YOUNGER = T < 0 ? (RING ? (R - 2) * PER : B_LOADS)
                                          : (RING ? (R - 2 - T > 0 ? (R - 2 - T) * PER : 0) : (T == 0 ? B_LOADS : 0));
            constexpr int NEXT_SET = SET ^ 1, N_FIRST = first_items(NEXT_SET), N_LATE = late_items(SET);
            constexpr int FIRST_HI = PARTS ? NM - TH : NM;
            constexpr int FILLS = FILL_B ? PER : (FILL_A ? LIVE : 0);
            const int at = fills.slab_at(kt);
            const int sa1 = sa == SA - 1 ? 0 : sa + 1, sb1 = sb == SB - 1 ? 0 : sb + 1;
            const uint32_t ka = (uint32_t)fills.slab_at(kt + (RING ? R : 2)) * 128u, kb = (uint32_t)fills.slab_at(kt + (RING ? R : 3)) * 128u;
            const From a0 = slot_a(sa), b0 = slot_b(sb), a1 = slot_a(sa1), b1 = slot_b(sb1);
            if (kt > 0 && ((at & 3) == 0 || at == fills.first)) take_scales(at);
            // the slab's scale byte of each dword, by statements that lie two instructions ahead of its use (see accumulators.py)
            const uint32_t sh = (uint32_t)(at & 3) * 8u;
            uint32_t sw[2], sx[2];
            auto shift = [&](uint32_t& to, uint32_t from) {
                asm volatile("v_lshrrev_b32 %0, %1, %2" : "=v"(to) : "s"(sh), "v"(from));
            };
            shift(sx[0], dist[walk(SET, 0).j]);
            shift(sw[0], scales.w[0]);
            if (S::SWIGLU) shift(sw[1], scales.w[1]);
            asm volatile("s_nop 1");
            __builtin_amdgcn_sched_barrier(0);
            each<NM>([&](auto q_c) {
                constexpr int q = decltype(q_c)::value;
                constexpr At now = walk(SET, q);
                if constexpr (q == QB) {
                    // slab kt+1 has landed for this wave (younger requests may still fly), this wave's operand reads of
                    // slab kt have returned (the LDS counter is part of the wait)
                    __builtin_amdgcn_s_waitcnt(waitcnt_vm(YOUNGER));
                    __builtin_amdgcn_s_barrier();
                    __builtin_amdgcn_sched_barrier(0);
                }
                // reads behind the barrier: of the next slab; ahead of it: the rest of this one
                if constexpr (q < QB && N_LATE > 0) {
                    constexpr int lo = before(q, N_LATE, 0, QB - 6), hi = before(q + 1, N_LATE, 0, QB - 6);
                    each<hi - lo>([&](auto r) {
                        read_item(set_c, std::true_type{}, std::integral_constant<int, lo + decltype(r)::value>{}, a0, b0);
                    });
                }
                if constexpr (MORE && q >= QB) {
                    // PARTS: B0 over all of it, an activation sub-tile behind its row of part 3
                    constexpr int N_B = PARTS ? TH : N_FIRST, N_A = N_FIRST - N_B;
                    constexpr int lo = before(q, N_B, QB, FIRST_HI), hi = before(q + 1, N_B, QB, FIRST_HI);
                    each<hi - lo>([&](auto r) {
                        read_item(std::integral_constant<int, NEXT_SET>{}, std::false_type{},
                                  std::integral_constant<int, lo + decltype(r)::value>{}, a1, b1);
                    });
                    if constexpr (N_A > 0 && q > QB && (q - QB) % TH == 0 && (q - QB) / TH <= N_A)
                        read_item(std::integral_constant<int, NEXT_SET>{}, std::false_type{},
                                  std::integral_constant<int, N_B + (q - QB) / TH - 1>{}, a1, b1);
                }
                if constexpr (FILLS > 0 && q >= QB) {
                    auto pos = [](int f) constexpr { return QB + (4 * f + PHASE) * (NM - QB) / (4 * PER); };
                    auto ahead = [pos](int to) constexpr {
                        int n = 0;
                        while (n < FILLS && pos(n) < to) ++n;
                        return n;
                    };
                    constexpr int lo = ahead(q), hi = ahead(q + 1);
                    each<hi - lo>([&](auto r) {
                        constexpr int f = lo + decltype(r)::value;
                        if constexpr (f < LIVE)
                            fills.one_a(f, ka, sa * A_STRIDE);
                        else
                            fills.one_b(f - LIVE, kb, B_BASE + sb * B_STRIDE, ONCE);
                    });
                }
                if constexpr (now.first && now.row + 1 < ROWS) {  // the next row's scales
                    constexpr int ahead = q + (PARTS ? TH : TN);
                    shift(sx[(now.row + 1) & 1], dist[walk(SET, ahead).j]);
                }
                constexpr int s = PARTS ? 0 : SET;
                acc_mfma8<S::fragment(now.i, now.j)>(wb[s][now.i], xa[s][now.j], sw[S::SWIGLU ? now.i / TH : 0], sx[now.row & 1]);
                __builtin_amdgcn_sched_barrier(0);
            });
        };
        auto advance = [&]() {
            ++kt;
            sa = sa == SA - 1 ? 0 : sa + 1;
            sb = sb == SB - 1 ? 0 : sb + 1;
        };
        using zero = std::integral_constant<int, 0>;
        using one = std::integral_constant<int, 1>;
        using steady = std::integral_constant<int, -1>;
        take_scales(fills.slab_at(0));
        int left = KT - TAIL;  // slabs with all requests
        const int skip = left < 0 ? -left : 0;
        if ((left > 0 ? left : skip) & 1)
            read_first(one{});
        else
            read_first(zero{});
        if (!RING && KT > 2) {  // the third slot of weights
            const uint32_t k = (uint32_t)fills.slab_at(2) * 128u;
#pragma unroll
            for (int f = 0; f < B_LOADS; ++f) fills.one_b(f, k, B_BASE + 2 * B_STRIDE, ONCE);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (left > 0 && (left & 1)) {
            slab(one{}, steady{});
            advance();
            --left;
        }
        for (; left > 0; left -= 2) {
            slab(zero{}, steady{});
            advance();
            slab(one{}, steady{});
            advance();
        }
        draw();
        each<TAIL>([&](auto t_c) {
            constexpr int t = decltype(t_c)::value;
            if (t < skip) return;
            // the slot of the slab before is read no more; a product of one slab has the second slot free
            if (t == TAIL - 1) before_last((kt == 0 ? 1 : (sa == 0 ? SA - 1 : sa - 1)) * A_STRIDE);
            __builtin_amdgcn_sched_barrier(0);
            slab(std::integral_constant<int, t & 1>{}, t_c);
            advance();
        });
        // the last matrix instructions retire before anything else reads the accumulators
        asm volatile("s_nop 15\n\ts_nop 15");
    }
};

// Writes sub-tile row j of a block's bf16 output (see TileWriter in ffn_tile.h); columns at or behind n are not written.
template <class S>
struct ColumnWriter {
    __amdgpu_buffer_rsrc_t c;
    uint32_t at, pitch;
    int col, n;
    __device__ __forceinline__ ColumnWriter(const Fp8Args& p, const WorkItem& w, int wm, int wn, int lane) {
        const int lr = lane & 15, lk = lane >> 4;
        n = p.n;
        pitch = (uint32_t)p.n * 2u;
        c = __builtin_amdgcn_make_buffer_rsrc((void*)(p.y + ((size_t)w.row0 * p.n + w.n0) * 2), 0,
                                              (int)((uint32_t)(w.rows - 1) * pitch + (uint32_t)min(S::kNCols, p.n - w.n0) * 2u), kRsrcFlags);
        const int in = wn * (S::kNCols / 2) + (lk & 1) * 16 + (lk >> 1) * 8;
        col = w.n0 + in;
        at = (uint32_t)(wm * 16 + lr) * pitch + (uint32_t)in * 2u;
    }
    template <class Frag>
    __device__ __forceinline__ void rows(int j, Frag&& frag) const {
        each<S::TNO / 2>([&](auto pair_c) {
            constexpr int i = 2 * decltype(pair_c)::value;
            uint32_t half[2][2];
            each<2>([&](auto s_c) {
                constexpr int s = decltype(s_c)::value;
                const f32x4 g = frag(std::integral_constant<int, i + s>{});
                half[s][0] = pack_bf16x2(g[0], g[1]);
                half[s][1] = pack_bf16x2(g[2], g[3]);
            });
            const auto lo = __builtin_amdgcn_permlane16_swap(half[0][0], half[1][0], false, false);
            const auto hi = __builtin_amdgcn_permlane16_swap(half[0][1], half[1][1], false, false);
            const u32x4 out = {lo[0], hi[0], lo[1], hi[1]};
            __builtin_amdgcn_raw_buffer_store_b128(out, c, col + i * 16 < n ? at + (uint32_t)(j * 32) * pitch + i * 32 : kBeyond, 0, 0);
        });
    }
};

// The hidden activation of a block: silu(gate) * up rounded to bf16, then the 128 columns of each row quantised.  Two waves
// hold halves of a row and exchange the largest magnitudes of theirs through LDS.
template <class S>
__device__ __forceinline__ int write_hidden(const Fp8Args& p, const WorkItem& w, int wm, int wn, int lane, int live, uint8_t* smem) {
    constexpr int TM = S::TM;
    const int lr = lane & 15, lk = lane >> 4;
    uint32_t v[TM][8], bad[TM], top[TM];
    each<TM>([&](auto j_c) {
        constexpr int j = decltype(j_c)::value;
        if (j < live) {
            each<4>([&](auto i_c) {
                constexpr int i = decltype(i_c)::value;
                const f32x4 g = acc_read<S::fragment(i, j)>(), u = acc_read<S::fragment(i + 4, j)>();
                float o[4];
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    o[k] = g[k] * u[k] * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g[k] * -1.4426950408889634f));
                v[j][2 * i] = pack_bf16x2(o[0], o[1]);
                v[j][2 * i + 1] = pack_bf16x2(o[2], o[3]);
            });
            top[j] = max_over_rows_of_16(amax_bf16(v[j], bad[j]));
            if (lk == 0) *lds_word(smem, S::kExchange + (wn * S::BM + j * 32 + wm * 16 + lr) * 4) = (int)top[j];
        }
    });
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(63));  // the LDS counter alone
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    const __amdgpu_buffer_rsrc_t c = __builtin_amdgcn_make_buffer_rsrc((void*)(p.y + (size_t)w.row0 * p.n_pad + w.n0), 0,
                                                                       (w.rows - 1) * p.n_pad + S::kNCols, kRsrcFlags);
    const __amdgpu_buffer_rsrc_t cs = __builtin_amdgcn_make_buffer_rsrc(
        (void*)(p.y_scale + (size_t)w.row0 * p.y_scale_pitch + w.n0 / kFp8Block), 0, (w.rows - 1) * p.y_scale_pitch + 1, kRsrcFlags);
    each<TM>([&](auto j_c) {
        constexpr int j = decltype(j_c)::value;
        if (j < live) {
            const int row = j * 32 + wm * 16 + lr;
            const uint32_t other = (uint32_t)*lds_word(smem, S::kExchange + ((wn ^ 1) * S::BM + row) * 4);
            const uint32_t byte = scale_byte(max(top[j], other) << 16);
            uint32_t q[4];
            to_e4m3(v[j], byte, q);
            mark_bad(q, bad[j]);
            // lane group g gets the four dwords of sub-tile g
            const auto a = __builtin_amdgcn_permlane32_swap(q[0], q[2], false, false);
            const auto b = __builtin_amdgcn_permlane32_swap(q[1], q[3], false, false);
            const auto lo = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
            const auto hi = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
            const u32x4 out = {lo[0], lo[1], hi[0], hi[1]};
            __builtin_amdgcn_raw_buffer_store_b128(out, c, (uint32_t)(row * p.n_pad + wn * 64 + lk * 16), 0, 0);
            __builtin_amdgcn_raw_buffer_store_b8((uint8_t)byte, cs, lk == 0 && wn == 0 ? (uint32_t)(row * p.y_scale_pitch) : kBeyond, 0, 0);
        }
    });
    return 2 * live;
}

// One block per compute unit for the whole launch (see ffn.hip).
template <class S>
__global__ __launch_bounds__(S::kThreads) void fp8_gemm_kernel(const Fp8Args p) {
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    if constexpr (S::TN * S::TM == 64)
        asm volatile("" ::: "a255");  // the kernel has all accumulation registers
    else
        asm volatile("" ::: "a127");
    static_assert(S::TN * S::TM == 64 || S::TN * S::TM == 32, "accumulators");
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wv >> 1, wn = wv & 1;
    int per_xcd = gridDim.x >> 3;
    asm volatile("" : "+s"(per_xcd));  // kept, not fetched again with every ticket
    const WorkOrder<S> order(p.L, p.hdr, p.pitch / 2, p.n_pad, p.col_group_big, p.col_group_small, p.stream);
    int place = blockIdx.x >> 3;
    if (order.pool > 0 && place >= order.positions()) {  // nothing left of the XCD's share: it starts in the shared end
        if (wv == 0) {
            int n = 0;
            if (lane == 0)
                n = WorkOrder<S>::kPoolItem +
                    __hip_atomic_fetch_add(p.counter + kPoolTicket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            n = __builtin_amdgcn_readfirstlane(n);
            if (lane < S::NW) *lds_word(smem, lane * 1024) = n;  // a copy per wave, in the quarter that only it overwrites
        }
        __syncthreads();
        place = __builtin_amdgcn_readfirstlane(*lds_word(smem, wv * 1024));
    }
    WorkItem cur = order.at(place);
    if (!cur.valid) return;
    const bool more = order.pool > 0 || order.positions() > per_xcd;  // whether a block may find another item
    const int lr = lane & 15, lk = lane >> 4;
    const int piece0 = (lk ^ ((lr >> 1) & 7)) << 4;
    const int a_lane = (wm * 16 + lr) * 128 + piece0;
    const int b_lane = ((S::SWIGLU ? wn * (S::BN / 4) : wn * (S::BN / 2)) + lr) * 128 + piece0;

    Fills8<S> fills;
    Scales8<S> scales;
    fills.smem = smem;
    fills.wv = wv;
    fills.weights_of_lane(lane, p.pitch);
    fills.aim(cur, p, lane, wm, wn);
    scales.request(fills, fills.slab_at(0), (cur.rows + 31) >> 5);
    __builtin_amdgcn_sched_barrier(0);
    int younger = fills.start((cur.rows + 31) >> 5, cur.once);
    for (;;) {
        const int live = (cur.rows + 31) >> 5;
        each<S::TM>([&](auto j_c) {
            if (decltype(j_c)::value < live)
                each<S::TN>([](auto i_c) { acc_zero<S::fragment(decltype(i_c)::value, decltype(j_c)::value)>(); });
        });
        __builtin_amdgcn_sched_barrier(0);
        wait_for_all_but(younger);
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        // The block's next position.  (The offset of zero is one that the compiler takes for a value per lane: see ffn.hip.)
        int next = __builtin_nondeterministic_value(0), none = 0, handed = 0;
        asm volatile("" : "+v"(none));
        auto draw = [&]() {
            if (more && tid == 0)
                next = __hip_atomic_fetch_add(p.counter + (blockIdx.x & 7) * (kFfnSplitUnits / 8) + kXcdTicket + none, 1,
                                              __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        };
        auto hand_over = [&](int at) {
            handed = at + wv * 1024;
            if (more && wv == 0) {
                int n = 0;
                if (lane == 0) {
                    n = next + per_xcd;
                    if (order.pool > 0 && n >= order.positions())
                        n = WorkOrder<S>::kPoolItem +
                            __hip_atomic_fetch_add(p.counter + kPoolTicket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                }
                n = __builtin_amdgcn_readfirstlane(n);
                if (lane < S::NW) *lds_word(smem, at + lane * 1024) = n;
            }
        };
        auto loop = [&](auto once_c) {
            MatrixLoop8<S, decltype(once_c)::value> m{fills, scales, a_lane, b_lane};
            switch (live) {
                case 8:
                    switch (wv) {
                        case 0: m.template run<8, 0>(draw, hand_over); break;
                        case 1: m.template run<8, 1>(draw, hand_over); break;
                        case 2: m.template run<8, 2>(draw, hand_over); break;
                        default: m.template run<8, 3>(draw, hand_over); break;
                    }
                    break;
                case 7: m.template run<7, 0>(draw, hand_over); break;
                case 6: m.template run<6, 0>(draw, hand_over); break;
                case 5: m.template run<5, 0>(draw, hand_over); break;
                case 4: m.template run<4, 0>(draw, hand_over); break;
                case 3: m.template run<3, 0>(draw, hand_over); break;
                case 2: m.template run<2, 0>(draw, hand_over); break;
                default: m.template run<1, 0>(draw, hand_over); break;
            }
        };
        if (cur.once)
            loop(std::true_type{});
        else
            loop(std::false_type{});
        WorkItem nxt;
        nxt.valid = 0;
        if (more) nxt = order.at(__builtin_amdgcn_readfirstlane(*lds_word(smem, handed)));
        younger = 0;
        if (nxt.valid) {
            fills.aim(nxt, p, lane, wm, wn);
            scales.request(fills, fills.slab_at(0), (nxt.rows + 31) >> 5);
            __builtin_amdgcn_sched_barrier(0);
            younger = fills.start((nxt.rows + 31) >> 5, nxt.once);
        }
        if constexpr (S::SWIGLU) {
            younger += write_hidden<S>(p, cur, wm, wn, lane, live, smem);
        } else {
            const ColumnWriter<S> out(p, cur, wm, wn, lane);
            each<S::TM>([&](auto j_c) {
                constexpr int j = decltype(j_c)::value;
                if (j < live) out.rows(j, [&](auto i_c) { return acc_read<S::fragment(decltype(i_c)::value, j)>(); });
            });
            younger += live * (S::TNO / 2);
        }
        if (!nxt.valid) return;
        cur = nxt;
    }
}

template <int BN, bool SWIGLU>
void launch_fp8_shape(Fp8Args p, const FfnWorkspace& ws, hipStream_t st) {
    using S = Shape8<BN, SWIGLU>;
    auto kern = fp8_gemm_kernel<S>;
    static std::atomic<uint64_t> configured{0};
    once_per_device(configured, [&] {
        (void)hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, S::kLdsBytes);
    });
    const int nb = p.n_pad / S::kNCols;
    // a block per compute unit, the same number on every XCD; fewer where the plan cannot hold as many items (one that runs
    // as row pieces is four)
    const int per_xcd = std::max(1, compute_units() / 8);
    const long long items = (long long)kFfnRowPieces * nb * ((long long)ws.big.max_tiles + ws.small.max_tiles);
    const int grid = 8 * (int)std::min<long long>(per_xcd, (items + 7) / 8);
    p.col_group_big = column_group(nb);
    p.col_group_small = p.stream ? nb : column_group(nb);
    hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(S::kThreads), S::kLdsBytes, st, p);
}

// The build compiles this file once for each shape (each takes as long as all other files together).
#if CAPMOE_FP8_SHAPE == 0
template void launch_fp8_shape<256, true>(Fp8Args, const FfnWorkspace&, hipStream_t);
#elif CAPMOE_FP8_SHAPE == 1
template void launch_fp8_shape<256, false>(Fp8Args, const FfnWorkspace&, hipStream_t);
#else
template void launch_fp8_shape<128, false>(Fp8Args, const FfnWorkspace&, hipStream_t);
#endif

}  // namespace capmoe
