// Products on 4-bit rows and 4-bit expert weights, grouped by expert, on high row tiles (fp4_thin.hip has the few-row ones).
//
//   y[r,n] = sum over blocks b of 32 k:  2^(xs[r,b] + ws[e,n,b] - 254) * sum over k in b: x[r,k] w[e,n,k]
//
// v_mfma_scale_f32_16x16x128_f8f6f4 takes 128 k of e2m1 at once, 64 bytes of a row, and a scale byte from every lane for its
// 32 k, so the scales cost the vector unit nothing.  Registers alone sustain 5.6 PFLOP/s of it on random operands (8 bits: 4.3).
//
// Tiles, LDS layout of the rows, requests, the parts of a slab and the order of the work are those of the 8-bit kernel (fp8.hip): a row's
// slab is 128 bytes, here 256 k and two matrix instructions per pair of sub-tiles.  Lane l takes pieces l >> 4 and
// (l >> 4) + 4 (16 bytes, one block of 32 k each) of row l & 15 of both operands, one for either instruction.
//
// What differs is the scales: a byte per row and 32 k of both operands, 8 KB for two slabs of a tile, which lie in groups of 16 bytes
// per row (512 k) such that the four bytes of a lane are one word.  They come through LDS as the rows do: 16 bytes of a row at a time, one
// request per wave and slab (the rows' scales in even slabs, the weights' in odd ones), in three slots.  A lane reads the two bytes
// of a slab for a sub-tile with the sub-tile itself.
#include <algorithm>

#include "fp4.h"
#include "narrow_tile.h"

namespace capmoe {

// M: which of a slab's two instructions; its scales are byte M of the words
template <int F, int M>
__device__ __forceinline__ void acc_mfma4(const u32x4& w, const u32x4& x, uint32_t w_scale, uint32_t x_scale) {
    if constexpr (M == 0)
        asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 a[%0:%1], %2, %3, a[%0:%1], %4, %5 op_sel:[0,0,0] op_sel_hi:[0,0,0] cbsz:4 blgp:4" ::"n"(
                         4 * F),
                     "n"(4 * F + 3), "v"(w), "v"(x), "v"(w_scale), "v"(x_scale));
    else
        asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 a[%0:%1], %2, %3, a[%0:%1], %4, %5 op_sel:[1,1,0] op_sel_hi:[0,0,0] cbsz:4 blgp:4" ::"n"(
                         4 * F),
                     "n"(4 * F + 3), "v"(w), "v"(x), "v"(w_scale), "v"(x_scale));
}

// The tile of the 8-bit kernel, its slabs in a ring of units in LDS (halves of a slab for tiles with LIVE above 2), behind
// them three slots of scales.
template <int BN_, bool SWIGLU_>
struct Shape4 : Shape<BN_, SWIGLU_> {
    using Base = Shape<BN_, SWIGLU_>;
    static constexpr int kScaleSlot = 8192, kScaleSlots = 3;  // of two slabs: 256 rows, 256 weight rows
    static constexpr int kLdsBytes = 160 * 1024;
    static constexpr int kScales = kLdsBytes - kScaleSlots * kScaleSlot;
    static constexpr int TH = Base::TN / 2;
    static_assert(Base::A_LOADS == 8, "a request per sub-tile pair");
    static constexpr int kHalfLoads = Base::B_LOADS / 2;  // a wave's requests for half of a slab's weights
    static __host__ __device__ constexpr bool parts(int live) { return live > 2; }
    static __host__ __device__ constexpr int half0(int live) { return (live + 1) / 2; }  // sub-tile pairs in the first half
    static __host__ __device__ constexpr int a_bytes(int live) { return (parts(live) ? half0(live) : live) * 4096; }
    static __host__ __device__ constexpr int unit(int live) { return a_bytes(live) + (parts(live) ? Base::B_SLOT / 2 : Base::B_SLOT); }
    static __host__ __device__ constexpr int units(int live) {  // in the ring
        const int n = kScales / unit(live), most = parts(live) ? 6 : kTail;
        return n < most ? n : most;
    }
    // Slabs at the end of an item that run without some of the requests.  The scales of slab kt + 4 or what lies beside them are
    // requested in slab kt, so these slabs request none.
    static constexpr int kTail = 3;
    // (the bounds that the scales' requests ask for, see MatrixLoop4)
    static_assert(units(8) >= 4 && units(3) <= 6 && units(1) == kTail && units(2) == kTail, "ring");
    // which half of the activations the first slab of an item begins with: such that the tail always begins with the first
    static __host__ __device__ constexpr int parity(int slabs) {
        const int left = slabs - kTail;
        return (left > 0 ? left : -left) & 1;
    }
};

// What a wave needs to request its pieces of a K slab (see Fills in ffn_tile.h) and the scales.
template <class S>
struct Fills4 {
    __amdgpu_buffer_rsrc_t a, b0, b1, sa, sb;
    typedef __attribute__((ext_vector_type(8))) unsigned int u32x8;  // (of an array the compiler would keep a copy in memory)
    u32x8 va;           // per sub-tile pair
    uint32_t vb;        // of the weights the rows of load i lie 32 * i rows further
    uint32_t vsa, vsb;  // scales: a row per lane, 64 rows per wave
    int slabs, turn;
    uint32_t row_step;  // bytes of 32 weight rows
    uint8_t* smem;
    int wv;

    __device__ __forceinline__ void weights_of_lane(int lane, int pitch, int scale_pitch) {  // the same for every item
        const int r = wv * 8 + lane / 8, kc = (lane % 8) ^ ((r >> 1) & 7);
        vb = (uint32_t)r * (uint32_t)pitch + kc * 16;
        row_step = 32u * (uint32_t)pitch;
        // with SWIGLU waves 0 and 1 take gate rows, 2 and 3 up rows; of 128 weight rows, waves 2 and 3 take them once more
        vsb = (uint32_t)((wv * 64 + lane) & (S::SWIGLU || S::BN == 128 ? 127 : 255)) * (uint32_t)scale_pitch;
    }
    __device__ __forceinline__ void aim(const WorkItem& w, const Fp4Args& p, int lane) {
        const int32_t* gather = p.gather;
        const int64_t x0 = gather ? 0 : w.row0;
        a = __builtin_amdgcn_make_buffer_rsrc((void*)(p.x + x0 * p.pitch), 0,
                                              (int)(uint32_t)min((p.x_rows - x0) * p.pitch, (int64_t)kBeyond), kRsrcFlags);
        sa = __builtin_amdgcn_make_buffer_rsrc((void*)(p.x_scale + x0 * p.scale_pitch), 0,
                                               (int)(uint32_t)min((p.x_rows - x0) * p.scale_pitch, (int64_t)kBeyond), kRsrcFlags);
        const size_t n_at = (size_t)w.e * p.n_pad + w.n0;
        // No bound: the kNCols rows of a tile are all there (n_pad is a multiple of that; see fp8.hip)
        b0 = __builtin_amdgcn_make_buffer_rsrc((void*)(p.w[0] + n_at * p.pitch), 0, -1, kRsrcFlags);
        b1 = S::SWIGLU ? __builtin_amdgcn_make_buffer_rsrc((void*)(p.w[1] + n_at * p.pitch), 0, -1, kRsrcFlags) : b0;
        const uint8_t* scale = S::SWIGLU && wv >= 2 ? p.w_scale[1] : p.w_scale[0];
        sb = __builtin_amdgcn_make_buffer_rsrc((void*)(scale + n_at * p.scale_pitch), 0, S::kNCols * p.scale_pitch, kRsrcFlags);
        slabs = __builtin_amdgcn_readfirstlane(w.slabs);
        // two slabs share a group of scales: the walk does not part them
        turn = __builtin_amdgcn_readfirstlane(slabs & 1 ? 0 : w.turn & ~1);
        uint32_t row[S::A_LOADS], srow;
#pragma unroll
        for (int i = 0; i < S::A_LOADS; ++i) {
            const int r = (wv + S::NW * i) * 8 + lane / 8;
            const int rr = r < w.rows ? r : w.rows - 1;  // rows past the expert's end repeat its last row
            row[i] = gather ? (uint32_t)gather[w.row0 + rr] : (uint32_t)rr;
        }
        {
            const int r = wv * 64 + lane, rr = r < w.rows ? r : w.rows - 1;
            srow = gather ? (uint32_t)gather[w.row0 + rr] : (uint32_t)rr;
        }
#pragma unroll
        for (int i = 0; i < S::A_LOADS; ++i) {
            const int r = (wv + S::NW * i) * 8 + lane / 8, kc = (lane % 8) ^ ((r >> 1) & 7);
            va[i] = row[i] * (uint32_t)p.pitch + kc * 16;
        }
        vsa = srow * (uint32_t)p.scale_pitch;
    }
    __device__ __forceinline__ int slab_at(int kt) const {
        kt += turn;
        return kt < slabs ? kt : kt - slabs;
    }
    // sub-tile pair j of the activations at k bytes of their rows, to byte `to` of LDS
    __device__ __forceinline__ void one_a(int j, uint32_t k, int to) const {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(a, (lptr_t)(smem + to + wv * 1024), 16, va[j], k, 0, 0);
    }
    // request i of half h of the weights
    __device__ __forceinline__ void one_b(int h, int i, uint32_t k, int to, bool once) const {
        // i and once are compile-time constants after unrolling
        constexpr int kPer = S::TH / 2;  // 32-row steps of one wave column's half
        uint8_t* dst = smem + to + (wv + S::NW * i) * 1024;
        const __amdgpu_buffer_rsrc_t r = S::SWIGLU && h ? b1 : b0;
        const uint32_t at = k + (uint32_t)(S::SWIGLU ? i : i / kPer * (S::BN / 64) + h * kPer + i % kPer) * row_step;
        if (once)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lptr_t)dst, 16, vb, at, 0, 2);  // bit 1: non-temporal
        else
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lptr_t)dst, 16, vb, at, 0, 0);
    }
    // Scale request i: of the group of slabs i & ~1 and one further, of the rows (i even) or the weights, to that part of a slot.
    // (Of a group behind the last, bytes that nobody reads.)
    __device__ __forceinline__ void one_scale(int i, int slot) const {
        const uint32_t at = (uint32_t)(slab_at(i & ~1) >> 1) * 16u;
        uint8_t* dst = smem + S::kScales + slot * S::kScaleSlot + wv * 1024;
        if (i & 1)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(sb, (lptr_t)(dst + 4096), 16, vsb, at, 0, 0);
        else
            __builtin_amdgcn_raw_ptr_buffer_load_lds(sa, (lptr_t)dst, 16, vsa, at, 0, 0);
    }
    // The first units of an item and the scales of its first four slabs, in the order in which a loop before it would have requested them
    // (see MatrixLoop4).  Returns how many requests are younger than those of the first unit.
    __device__ __forceinline__ int start(int live, bool once) const {
        const bool parts = S::parts(live);
        const int nu = S::units(live), h0 = S::half0(live), parity = S::parity(slabs);
        const int n = min(nu, parts ? 2 * slabs : slabs);
        one_scale(0, 0);
        one_scale(1, 0);
        int younger = 0, scale = 2;
        for (int u = 0; u < n; ++u) {
            // request i lies ahead of unit nu + 2 (i - 4), or nu + i - 4
            while (scale < 4 && (parts ? nu + 2 * (scale - 4) : nu + scale - 4) <= u) {
                one_scale(scale, 1);
                ++scale;
                if (u > 0) ++younger;
            }
            const int s = parts ? u >> 1 : u, late = parts ? u & 1 : 0, h = late ^ ((s + parity) & 1), to = u * S::unit(live);
            const uint32_t k = (uint32_t)slab_at(s) * (uint32_t)kSlabBytes;
            int count = 0;
#pragma unroll
            for (int hb = 0; hb < 2; ++hb) {
                if (parts && hb != late) continue;
                const int base = to + S::a_bytes(live) + (parts ? 0 : hb * (S::Base::B_SLOT / 2));
                if (once) {
#pragma unroll
                    for (int i = 0; i < S::kHalfLoads; ++i) one_b(hb, i, k, base, true);
                } else {
#pragma unroll
                    for (int i = 0; i < S::kHalfLoads; ++i) one_b(hb, i, k, base, false);
                }
                count += S::kHalfLoads;
            }
            const int lo = parts && h ? h0 : 0, hi = parts && !h ? h0 : live;
#pragma unroll
            for (int j = 0; j < S::A_LOADS; ++j)
                if (j >= lo && j < hi) one_a(j, k, to + (j - lo) * 4096);
            count += hi - lo;
            if (u > 0) younger += count;
            __builtin_amdgcn_sched_barrier(0);  // their order is what the waits count
        }
        return younger;
    }
};

// K loop of a wave.  LIVE = number of 16-row activation sub-tiles per wave that are fetched and multiplied.  How a slab is walked in
// parts, read and requested stands at MatrixLoop8 (fp8.hip).  The scales add one request per wave and slab: slab kt makes request
// i = kt + 4 (see one_scale) ahead of its first unit's, which is unit 2 kt + NU of half slabs, or kt + NU of slabs.  So
//   - a group's two requests (i = 2 g, 2 g + 1) have landed when unit 4 g of half slabs, or 2 g of slabs, has: the first of the group's
//     first slab, behind whose barrier the waves begin to read the group (2 (2 g - 3) + NU <= 4 g and 2 g - 3 + NU <= 2 g hold for the rings);
//   - the slot (g mod 3) was read for the last time in slab 2 g - 5, and the first request for it is made behind a barrier of slab 2 g - 4.
// The waits count the requests that are younger than the unit they wait for, and with them those for scales ahead of younger units.
template <class S, bool ONCE>
struct MatrixLoop4 {
    const Fills4<S>& fills;
    int a_lane, b_lane;    // byte offset, inside a unit's activations and half of weights, of this lane's first piece
    int sa_lane, sb_lane;  // .. inside a slot, of this lane's word of scales

    // where a unit's operands of this lane lie in LDS: the first and, four pieces further, the second half of a row's 128 bytes, and the
    // scales of either
    struct From {
        const uint8_t *lo, *hi, *scales;
        __device__ __forceinline__ From(const uint8_t* base, int lane_at, const uint8_t* scales_)
            : lo(base + lane_at), hi(base + (lane_at ^ 64)), scales(scales_) {}
        __device__ __forceinline__ void fetch(u32x4 (&to)[2], uint32_t& scale, int at, int row) const {
            to[0] = *(const u32x4*)(lo + at), to[1] = *(const u32x4*)(hi + at);
            scale = *(const uint16_t*)(scales + row * 16);
        }
    };
    static __host__ __device__ constexpr int weight_row(int i) { return S::SWIGLU ? i / S::TH * 128 + i % S::TH * 16 : i * 16; }

    // PHASE (0..3): where in a step this wave places its requests: the waves leave every barrier together (see ffn.hip)
    template <int LIVE, int PHASE>
    __device__ __forceinline__ void run() {
        constexpr int TN = S::TN, TH = S::TH, NM = TN * LIVE, HALF_LOADS = S::kHalfLoads;
        constexpr bool PARTS = S::parts(LIVE);
        constexpr int SETS = PARTS ? 1 : 2, STEPS = PARTS ? 2 : 1;  // units per slab
        constexpr int NU = S::units(LIVE), UNIT = S::unit(LIVE), A_BYTES = S::a_bytes(LIVE), TAIL = S::kTail, H0 = S::half0(LIVE);
        // pair q of a slab that begins with half `set` of the activations
        struct At {
            int j, i;
        };
        auto walk = [](int set, int q) constexpr {
            if (!PARTS) return At{q / TN, q % TN};
            const int half[2] = {H0, LIVE - H0}, f = set, n_f = half[f], n_g = half[f ^ 1];
            const int r = q / TH, i = q % TH;
            const int part = r < n_f ? 0 : (r < LIVE ? 1 : (r < LIVE + n_g ? 2 : 3));
            const int in = r - (part == 0 ? 0 : (part == 1 ? n_f : (part == 2 ? LIVE : LIVE + n_g)));
            const int h = part == 0 || part == 3 ? f : f ^ 1;
            return At{(h == 0 ? 0 : H0) + in, (part < 2 ? 0 : TH) + i};
        };
        // unit k (0: the one a slab with parity set begins with): its half of the activations, requests
        auto half_of = [](int set, int k) constexpr { return (k & 1) ^ ((set + k / 2) & 1); };
        auto loads_a = [half_of](int set, int k) constexpr { return !PARTS ? LIVE : (half_of(set, k) == 0 ? H0 : LIVE - H0); };
        auto loads = [loads_a](int set, int k) constexpr { return loads_a(set, k) + (PARTS ? HALF_LOADS : 2 * HALF_LOADS); };
        uint8_t* const smem = fills.smem;
        const int KT = fills.slabs;
        int a_lane = this->a_lane, b_lane = this->b_lane;
        asm volatile("" : "+v"(a_lane), "+v"(b_lane));  // the first operand reads stay here, not ahead of all instances
        u32x4 xa[SETS][LIVE][2], wb[SETS][TN][2];
        uint32_t sx[SETS][LIVE], sw[SETS][TN];  // scale bytes of a slab's two instructions

        // Operand read r of unit k of a slab with parity set: its weights, then its activations, in the order of use (without
        // parts: an activation, the weights, the other activations).
        auto weights_first = [](int k) constexpr { return PARTS ? k % 2 == 0 : false; };
        auto read_item = [&](auto set_c, auto k_c, auto r_c, const From& a, const From& b) {
            constexpr int set = decltype(set_c)::value, k = decltype(k_c)::value, r = decltype(r_c)::value;
            if constexpr (!PARTS) {
                constexpr int s = set ^ (k & 1);
                if constexpr (r == 0 || r > TN)
                    a.fetch(xa[s][r == 0 ? 0 : r - TN], sx[s][r == 0 ? 0 : r - TN], (r == 0 ? 0 : r - TN) * 4096, (r == 0 ? 0 : r - TN) * 32);
                else
                    b.fetch(wb[s][r - 1], sw[s][r - 1], (r - 1) / TH * (S::Base::B_SLOT / 2) + (r - 1) % TH * 2048, weight_row(r - 1));
            } else {
                constexpr int h = half_of(set, k), n = loads_a(set, k), from = h == 0 ? 0 : H0;
                constexpr int ra = weights_first(k) ? r - TH : r, rb = weights_first(k) ? r : r - n;
                if constexpr (ra >= 0 && ra < n)
                    a.fetch(xa[0][from + ra], sx[0][from + ra], ra * 4096, (from + ra) * 32);
                else
                    b.fetch(wb[0][k % 2 * TH + rb], sw[0][k % 2 * TH + rb], rb * 2048, weight_row(k % 2 * TH + rb));
            }
        };
        auto items = [loads_a](int set, int k) constexpr { return loads_a(set, k) + (PARTS ? TH : TN); };
        // where read r of the unit that is read in step `st` lies among the step's instructions (counted from its barrier)
        constexpr int LEN = 2 * NM / STEPS;                                   // instructions of a step
        constexpr int QB = PARTS ? 2 : (LEN / 4 > 0 ? LEN / 4 / 2 * 2 : 2);   // of these, ahead of the barrier
        auto read_at = [loads_a](int set, int st, int r) constexpr {
            if (!PARTS) return QB + r * (LEN - QB) / (LIVE + TN);
            if (st == 0) return QB + r * (LEN - QB - 8) / (loads_a(set, 1) + TH);  // activations, then weights
            // weights over all of it, an activation sub-tile behind its row of the third part
            return r < TH ? QB + r * (LEN - QB - 8) / TH : (r - TH + 1) * 2 * TH;
        };
        int kt = 0, slot = 0;               // of the unit that is read
        int scale_slot = 0, fill_scale = 2;  // of the scales that are read, and requested
        auto up = [](int s) { return s == NU - 1 ? 0 : s + 1; };
        auto up_scale = [](int s) { return s == S::kScaleSlots - 1 ? 0 : s + 1; };
        // One slab.  T < 0: all requests are made; otherwise TAIL - T slabs are left, this one included.
        auto slab = [&](auto set_c, auto tail_c) __attribute__((always_inline)) {
            constexpr int SET = decltype(set_c)::value, T = decltype(tail_c)::value;
            constexpr int L = T < 0 ? 1 << 20 : TAIL - T;
            each<STEPS>([&](auto st_c) {
                constexpr int ST = decltype(st_c)::value;
                constexpr int K = ST + 1;                                     // the unit that is read in this step
                constexpr bool MORE = ST + 1 < STEPS || L > 1;                // there is one
                constexpr int KF = ST + NU;                                   // the unit that is requested
                constexpr bool FILL = KF < STEPS * (L < 1000 ? L : 1000);
                constexpr int LEFT = STEPS * (L < 1000 ? L : 1000) - 1 - K;   // units behind the one that is read
                constexpr int FLY = LEFT < NU - 2 ? (LEFT > 0 ? LEFT : 0) : NU - 2;
                auto younger = [loads]() constexpr {
                    int n = 0;
                    for (int k = K + 1; k <= K + FLY; ++k) {
                        n += loads(SET, k);
                        // a request for scales lies ahead of the unit, made in a slab that makes them
                        const bool ahead = !PARTS || (k - NU) % 2 == 0;
                        if (ahead && k <= (PARTS ? 2 * L - 8 : L - 4) + NU) ++n;
                    }
                    return n;
                };
                constexpr int YOUNGER = younger();
                static_assert(YOUNGER < 64, "vmcnt");
                const int fill_slot = slot;  // the unit that was read before
                slot = up(slot);
                const int at = kt + K / STEPS;  // the slab whose unit that is
                if constexpr (K == STEPS) scale_slot = at & 1 ? scale_slot : up_scale(scale_slot);
                const uint8_t* const scales = smem + S::kScales + scale_slot * S::kScaleSlot + (at & 1) * 2;
                const From a(smem + slot * UNIT, a_lane, scales + sa_lane), b(smem + slot * UNIT + A_BYTES, b_lane, scales + sb_lane);
                const uint32_t kf = (uint32_t)fills.slab_at(kt + KF / STEPS) * (uint32_t)kSlabBytes;
                each<LEN>([&](auto n_c) {
                    constexpr int n = decltype(n_c)::value;
                    // two pairs at a time, the first instruction of either, then the second: an instruction does not wait for the one before
                    constexpr int q = ST * (LEN / 2) + n / 4 * 2 + n % 2, m = n / 2 % 2;
                    constexpr At now = walk(SET, q);
                    if constexpr (n == QB) {
                        // the unit has landed for this wave (younger requests may still fly), this wave's operand reads of the
                        // one before have returned (the LDS counter is part of the wait)
                        __builtin_amdgcn_s_waitcnt(waitcnt_vm(YOUNGER));
                        __builtin_amdgcn_s_barrier();
                        __builtin_amdgcn_sched_barrier(0);
                        if constexpr (ST == 0 && T < 0) {
                            fills.one_scale(kt + 4, fill_scale);
                            fill_scale = kt & 1 ? up_scale(fill_scale) : fill_scale;
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    }
                    if constexpr (MORE && n >= QB) {
                        each_at<0, items(SET, K), n>([read_at](int r) constexpr { return read_at(SET, ST, r); },
                                                     [&](auto r_c) { read_item(set_c, std::integral_constant<int, K>{}, r_c, a, b); });
                    }
                    if constexpr (FILL && n >= QB) {
                        constexpr int N = loads(SET, KF), NA = loads_a(SET, KF), H = half_of(SET, KF);
                        each_at<0, N, n>([](int f) constexpr { return QB + (4 * f + PHASE) * (LEN - QB) / (4 * N); }, [&](auto f_c) {
                            constexpr int f = decltype(f_c)::value;
                            if constexpr (f < NA)
                                fills.one_a((PARTS && H ? H0 : 0) + f, kf, fill_slot * UNIT + f * 4096);
                            else
                                fills.one_b(PARTS ? KF % 2 : (f - NA) / HALF_LOADS, (f - NA) % HALF_LOADS, kf,
                                            fill_slot * UNIT + A_BYTES + (PARTS ? 0 : (f - NA) / HALF_LOADS * (S::Base::B_SLOT / 2)), ONCE);
                        });
                    }
                    constexpr int s = PARTS ? 0 : SET;
                    acc_mfma4<S::fragment(now.i, now.j), m>(wb[s][now.i][m], xa[s][now.j][m], sw[s][now.i], sx[s][now.j]);
                    __builtin_amdgcn_sched_barrier(0);
                });
            });
            ++kt;
        };
        using zero = std::integral_constant<int, 0>;
        using one = std::integral_constant<int, 1>;
        using steady = std::integral_constant<int, -1>;
        auto begin = [&](auto set_c) {
            constexpr int set = decltype(set_c)::value;
            const uint8_t* const scales = smem + S::kScales;
            const From a(smem, a_lane, scales + sa_lane), b(smem + A_BYTES, b_lane, scales + sb_lane);
            each<items(set, 0)>([&](auto r_c) { read_item(set_c, zero{}, r_c, a, b); });
        };
        int left = KT - TAIL;  // slabs with all requests
        const int skip = left < 0 ? -left : 0;
        if (S::parity(KT))
            begin(one{});
        else
            begin(zero{});
        __builtin_amdgcn_sched_barrier(0);
        if (left > 0 && (left & 1)) {
            slab(one{}, steady{});
            --left;
        }
        for (; left > 0; left -= 2) {
            slab(zero{}, steady{});
            slab(one{}, steady{});
        }
        each<TAIL>([&](auto t_c) {
            constexpr int t = decltype(t_c)::value;
            if (t < skip) return;
            slab(std::integral_constant<int, t & 1>{}, t_c);
        });
        // the last matrix instructions retire before anything else reads the accumulators
        asm volatile("s_nop 15\n\ts_nop 15");
    }
};

// The hidden activation of a block: silu(gate) * up rounded to bf16, then each 32 columns of a row quantised: two sub-tiles of a wave.
template <class S>
__device__ __forceinline__ int write_hidden(const Fp4Args& p, const WorkItem& w, int wm, int wn, int lane, int live) {
    asm volatile("" : "+v"(lane));  // (see ColumnWriter)
    const int lr = lane & 15, lk = lane >> 4;
    const __amdgpu_buffer_rsrc_t c = __builtin_amdgcn_make_buffer_rsrc((void*)(p.y + (size_t)w.row0 * p.y_pitch + w.n0 / 2), 0,
                                                                       (w.rows - 1) * p.y_pitch + S::kNCols / 2, kRsrcFlags);
    // the tile's four blocks lie in places 4 g + column / 128 of a group; an odd last tile also writes the next four, which no tile has
    const int group = w.n0 / kFp4Group, in = w.n0 % kFp4Group / 128;
    const __amdgpu_buffer_rsrc_t cs = __builtin_amdgcn_make_buffer_rsrc((void*)(p.y_scale + (size_t)w.row0 * p.y_scale_pitch + group * 16), 0,
                                                                        (w.rows - 1) * p.y_scale_pitch + 16, kRsrcFlags);
    const bool fill = w.n0 + S::kNCols == p.n_pad && (in & 1) == 0;
    const uint32_t scale_at = lk < 2 || fill ? (uint32_t)(4 * (2 * wn + (lk & 1)) + in + (lk >> 1)) : kBeyond;
    each<S::TM>([&](auto j_c) {
        constexpr int j = decltype(j_c)::value;
        if (j < live) {
            uint32_t q[2], byte[2];
            each<2>([&](auto b_c) {
                constexpr int b = decltype(b_c)::value;
                Eight<true> v;
                each<2>([&](auto i_c) {
                    constexpr int i = 2 * b + decltype(i_c)::value;
                    const f32x4 g = acc_read<S::fragment(i, j)>(), u = acc_read<S::fragment(i + 4, j)>();
                    float o[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        o[k] = g[k] * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g[k] * -1.4426950408889634f)) * u[k];
                    v.v[2 * (i & 1)] = pack_bf16x2(o[0], o[1]);
                    v.v[2 * (i & 1) + 1] = pack_bf16x2(o[2], o[3]);
                });
                byte[b] = fp4_scale_byte(max_over_rows_of_16(amax_of_8(v)));
                q[b] = to_e2m1(v, byte[b]);  // four codes of either sub-tile
            });
            // lane group g gets the sixteen codes of sub-tile g: four of each group
            const auto a = __builtin_amdgcn_permlane32_swap(q[0], q[1], false, false);
            const uint32_t lo = __builtin_amdgcn_perm(a[1], a[0], 0x05040100), hi = __builtin_amdgcn_perm(a[1], a[0], 0x07060302);
            const auto d = __builtin_amdgcn_permlane16_swap(lo, hi, false, false);
            typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;
            const u32x2 out = {__builtin_amdgcn_perm(d[1], d[0], 0x05040100), __builtin_amdgcn_perm(d[1], d[0], 0x07060302)};
            const int row = j * 32 + wm * 16 + lr;
            __builtin_amdgcn_raw_buffer_store_b64(out, c, (uint32_t)(row * p.y_pitch + wn * 32 + lk * 8), 0, 0);
            const uint32_t mine = lk == 0 ? byte[0] : (lk == 1 ? byte[1] : 0u);
            __builtin_amdgcn_raw_buffer_store_b8((uint8_t)mine, cs, scale_at == kBeyond ? kBeyond : scale_at + (uint32_t)(row * p.y_scale_pitch), 0, 0);
        }
    });
    return 2 * live;
}

// One block per compute unit for the whole launch (see ffn.hip).
template <class S>
__global__ __launch_bounds__(S::kThreads) void fp4_gemm_kernel(const Fp4Args p) {
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    if constexpr (S::TN * S::TM == 64)
        asm volatile("" ::: "a255");  // the kernel has all accumulation registers
    else
        asm volatile("" ::: "a127");
    static_assert(S::TN * S::TM == 64 || S::TN * S::TM == 32, "accumulators");
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wv >> 1, wn = wv & 1;
    const int per_xcd = gridDim.x >> 3, xcd = blockIdx.x & 7;
    const TileOrder<S> order(p, lane, smem + wv * (kMaxExperts * 4));
    const int turn = blockIdx.x >> 3;
    int round = 0;
    WorkItem cur = order.next(xcd, round, turn, per_xcd);
    if (!cur.valid) return;
    __syncthreads();  // the waves' scratch
    const int lr = lane & 15, lk = lane >> 4;
    const int piece0 = (lk ^ ((lr >> 1) & 7)) << 4;
    const int a_lane = (wm * 16 + lr) * 128 + piece0;
    const int b_lane = (wn * S::TH * 16 + lr) * 128 + piece0;
    const int sa_lane = (wm * 16 + lr) * 16 + lk * 4;
    const int sb_lane = 4096 + (wn * (S::SWIGLU ? 64 : S::BN / 2) + lr) * 16 + lk * 4;

    Fills4<S> fills;
    fills.smem = smem;
    fills.wv = wv;
    fills.weights_of_lane(lane, p.pitch, p.scale_pitch);
    fills.aim(cur, p, lane);
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
        auto loop = [&](auto once_c) __attribute__((always_inline)) {
            MatrixLoop4<S, decltype(once_c)::value> m{fills, a_lane, b_lane, sa_lane, sb_lane};
            switch (live) {
                case 8:
                    switch (wv) {
                        case 0: m.template run<8, 0>(); break;
                        case 1: m.template run<8, 1>(); break;
                        case 2: m.template run<8, 2>(); break;
                        default: m.template run<8, 3>(); break;
                    }
                    break;
                case 7: m.template run<7, 0>(); break;
                case 6: m.template run<6, 0>(); break;
                case 5: m.template run<5, 0>(); break;
                case 4: m.template run<4, 0>(); break;
                case 3: m.template run<3, 0>(); break;
                case 2: m.template run<2, 0>(); break;
                default: m.template run<1, 0>(); break;
            }
        };
        if (cur.once)
            loop(std::true_type{});
        else
            loop(std::false_type{});
        const WorkItem nxt = order.next(xcd, round, turn, per_xcd);
        younger = 0;
        if (nxt.valid) {
            fills.aim(nxt, p, lane);
            __builtin_amdgcn_sched_barrier(0);
            younger = fills.start((nxt.rows + 31) >> 5, nxt.once);
        }
        if constexpr (S::SWIGLU) {
            younger += write_hidden<S>(p, cur, wm, wn, lane, live);
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
void launch_fp4_shape(Fp4Args p, hipStream_t st) {
    using S = Shape4<BN, SWIGLU>;
    auto kern = fp4_gemm_kernel<S>;
    static std::atomic<uint64_t> configured{0};
    once_per_device(configured, [&] {
        (void)hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, S::kLdsBytes);
    });
    const int nb = p.n_pad / S::kNCols;
    p.tile_shift = fp4_tile_shift(p.max_rows, nb, compute_units());
    // a block per compute unit, the same number on every XCD (which of them get items is known on the device only)
    const int grid = 8 * std::max(1, compute_units() / 8);
    p.col_group = nb % 4 == 0 ? 4 : (nb % 3 == 0 ? 3 : (nb % 2 == 0 ? 2 : 1));
    hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(S::kThreads), S::kLdsBytes, st, p);
}

// The build compiles this file once for each shape.
#if CAPMOE_FP4_SHAPE == 0
template void launch_fp4_shape<256, true>(Fp4Args, hipStream_t);
#elif CAPMOE_FP4_SHAPE == 1
template void launch_fp4_shape<256, false>(Fp4Args, hipStream_t);
#else
template void launch_fp4_shape<128, false>(Fp4Args, hipStream_t);
#endif

}  // namespace capmoe
