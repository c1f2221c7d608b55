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

#include "fp8.h"
#include "narrow_tile.h"

namespace capmoe {

typedef __attribute__((ext_vector_type(8))) int i32x8;

// BYTE: which byte of the scale words
template <int F, int BYTE>
__device__ __forceinline__ void acc_mfma8(const i32x8& w, const i32x8& x, uint32_t w_scale, uint32_t x_scale) {
    if constexpr (BYTE == 0)
        asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 a[%0:%1], %2, %3, a[%0:%1], %4, %5 op_sel:[0,0,0] op_sel_hi:[0,0,0]" ::"n"(4 * F),
                     "n"(4 * F + 3), "v"(w), "v"(x), "v"(w_scale), "v"(x_scale));
    else
        asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 a[%0:%1], %2, %3, a[%0:%1], %4, %5 op_sel:[1,1,0] op_sel_hi:[0,0,0]" ::"n"(4 * F),
                     "n"(4 * F + 3), "v"(w), "v"(x), "v"(w_scale), "v"(x_scale));
}

// The tile of the bf16 kernel, and how its slabs lie in LDS: in a ring of units.  A unit holds half of a slab's activation
// rows and half of its weight rows (tiles with LIVE above 2), or a slab.  Of activation sub-tile pair j (32 rows) and of 32
// weight rows 4 KB each; half h of the weights is the h-th half of either wave column's sub-tiles (with SWIGLU: gate, up).
template <int BN_, bool SWIGLU_>
struct Shape8 : Shape<BN_, SWIGLU_> {
    using Base = Shape<BN_, SWIGLU_>;
    static constexpr int kLdsBytes = 160 * 1024;
    // the last 4 KB: an exchange between waves at the end of an item, while the next item's first units arrive elsewhere
    static constexpr int kExchange = kLdsBytes - 4096;
    static constexpr int TH = Base::TN / 2;
    static_assert(Base::A_LOADS == 8, "a request per sub-tile pair");
    static constexpr int kHalfLoads = Base::B_LOADS / 2;  // a wave's requests for half of a slab's weights
    static __host__ __device__ constexpr bool parts(int live) { return live > 2; }
    static __host__ __device__ constexpr int half0(int live) { return (live + 1) / 2; }  // sub-tile pairs in the first half
    static __host__ __device__ constexpr int a_bytes(int live) { return (parts(live) ? half0(live) : live) * 4096; }
    static __host__ __device__ constexpr int unit(int live) { return a_bytes(live) + (parts(live) ? Base::B_SLOT / 2 : Base::B_SLOT); }
    static __host__ __device__ constexpr int units(int live) {  // in the ring
        const int n = (parts(live) ? kLdsBytes : kExchange) / unit(live), most = parts(live) ? 6 : 4;
        return n < most ? n : most;
    }
    // of these, how many are requested before the exchange is over
    static __host__ __device__ constexpr int early(int live) { return units(live) * unit(live) <= kExchange ? units(live) : units(live) - 1; }
    static_assert(units(8) >= 5 && units(1) >= 3 && units(2) >= 3 && early(8) * unit(8) <= kExchange, "ring");
    // slabs at the end of an item that run without some of the requests
    static __host__ __device__ constexpr int tail(int live) { return parts(live) ? 3 : units(live); }
    // which half of the activations the first slab of an item begins with: such that the tail always begins with the first
    static __host__ __device__ constexpr int parity(int live, int slabs) {
        const int left = slabs - tail(live);
        return (left > 0 ? left : -left) & 1;
    }
};

// What a wave needs to request its pieces of a K slab (see Fills in ffn_tile.h) and the scales.
template <class S>
struct Fills8 {
    __amdgpu_buffer_rsrc_t a, b0, b1, sa, sb0, sb1;
    typedef __attribute__((ext_vector_type(8))) unsigned int u32x8;  // (of an array the compiler would keep a copy in memory)
    u32x8 va;                     // per sub-tile pair
    uint32_t vb;                  // of the weights the rows of load i lie 32 * i rows further
    uint32_t vsa[2];              // scales: of the rows of sub-tiles 0..3 and 4..7, a quarter of the wave each
    int slabs, turn;
    uint32_t row_step;            // bytes of 32 weight rows
    int64_t scale_at;             // of the wave's weights' scales
    uint8_t* smem;
    int wv;

    __device__ __forceinline__ void weights_of_lane(int lane, int pitch) {  // the same for every item
        const int r = wv * 8 + lane / 8, kc = (lane % 8) ^ ((r >> 1) & 7);
        vb = (uint32_t)r * (uint32_t)pitch + kc * 16;
        row_step = 32u * (uint32_t)pitch;
    }
    __device__ __forceinline__ void aim(const WorkItem& w, const Fp8Args& p, int lane, int wm, int wn) {
        const int32_t* gather = p.gather;
        const int64_t x0 = gather ? 0 : w.row0;
        a = __builtin_amdgcn_make_buffer_rsrc((void*)(p.x + x0 * p.pitch), 0,
                                              (int)(uint32_t)min((p.x_rows - x0) * p.pitch, (int64_t)kBeyond), kRsrcFlags);
        sa = __builtin_amdgcn_make_buffer_rsrc((void*)(p.x_scale + x0 * p.scale_pitch), 0,
                                               (int)(uint32_t)min((p.x_rows - x0) * p.scale_pitch, (int64_t)kBeyond), kRsrcFlags);
        const size_t n_at = (size_t)w.e * p.n_pad + w.n0;
        // No bound: the kNCols rows of a tile are all there (n_pad is a multiple of that), and its requests end with row 31 + 32 * 7
        // of 256, or 31 + 32 * 3 of 128.  With one the FFN of 4096 tokens on 64 x 2048 x 1024 takes 1 % more (171.9 -> 174.2 us).
        b0 = __builtin_amdgcn_make_buffer_rsrc((void*)(p.w[0] + n_at * p.pitch), 0, -1, kRsrcFlags);
        b1 = S::SWIGLU ? __builtin_amdgcn_make_buffer_rsrc((void*)(p.w[1] + n_at * p.pitch), 0, -1, kRsrcFlags) : b0;
        // a wave's weight rows lie in one block of 128 (with SWIGLU in one of either tensor)
        scale_at = (n_at / kFp8Block + (S::SWIGLU || S::BN == 128 ? 0 : wn)) * p.scale_pitch;
        sb0 = __builtin_amdgcn_make_buffer_rsrc((void*)(p.w_scale[0] + scale_at), 0, p.scale_pitch, kRsrcFlags);
        sb1 = S::SWIGLU ? __builtin_amdgcn_make_buffer_rsrc((void*)(p.w_scale[1] + scale_at), 0, p.scale_pitch, kRsrcFlags) : sb0;
        slabs = __builtin_amdgcn_readfirstlane(w.slabs);
        turn = __builtin_amdgcn_readfirstlane(w.turn);
        // the pairs of slabs that share a request for scales (see Scales8) neither wrap around, so that slabs - turn + parity is
        // even, nor begin an item in two words
        turn = (turn & ~3) + (S::tail((w.rows + 31) >> 5) & min(turn, 1));
        turn = __builtin_amdgcn_readfirstlane(turn < slabs ? turn : 0);
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
    // The first units of an item, as many as may be requested while the item before is written.  Returns how many requests are
    // younger than those of the first.
    __device__ __forceinline__ int start(int live, bool once) const {
        const bool parts = S::parts(live);
        const int h0 = S::half0(live), parity = S::parity(live, slabs);
        const int n = min(S::early(live), parts ? 2 * slabs : slabs);
        int younger = 0;
        for (int u = 0; u < n; ++u) {
            const int s = parts ? u >> 1 : u, late = parts ? u & 1 : 0, h = late ^ ((s + parity) & 1), to = u * S::unit(live);
            const uint32_t k = (uint32_t)slab_at(s) * 128u;
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

// The scales of two slabs at a time, one that begins with either half of the activations (see MatrixLoop8).  Their bytes lie in
// two words.  They are requested while the two slabs before are multiplied, whether those shared the words or not, and become
// one word at the end of these: no request for a register is in flight around the loop, nor across the start of an item, where
// the compiler, which cannot know how many requests are younger, would wait for all of them (once every four slabs, before).
// An item's first words come through LDS, like its first units.
template <class S>
struct Scales8 {
    typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;
    u32x2 raw[2], raw_w[2];    // of 64 rows each, a row per lane; of the weights, the same in all lanes
    uint32_t word[2], word_w[2];  // of the next two slabs, in the lowest bytes
    static constexpr int kFirst = S::kExchange + 2048;  // [wave][64-row part][lane]

    // an item's first words
    __device__ __forceinline__ void begin(const Fills8<S>& f) {
        const int at = f.slab_at(0) & ~3;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(f.sa, (lptr_t)(f.smem + kFirst + f.wv * 512 + h * 256), 4, f.vsa[h], at, 0, 0);
    }
    // .. once they are in LDS
    __device__ __forceinline__ void take_first(const Fills8<S>& f, const Fp8Args& p, int64_t w_at, int lane) {
        const int slab = f.slab_at(0), sh = (slab & 3) * 8;
#pragma unroll
        for (int h = 0; h < 2; ++h) word[h] = (uint32_t)*lds_word(f.smem, kFirst + f.wv * 512 + h * 256 + lane * 4) >> sh;
        word_w[0] = (uint32_t)scalar_word((const int32_t*)(p.w_scale[0] + w_at), slab >> 2) >> sh;
        if (S::SWIGLU) word_w[1] = (uint32_t)scalar_word((const int32_t*)(p.w_scale[1] + w_at), slab >> 2) >> sh;
    }
    __device__ __forceinline__ void request(const Fills8<S>& f, int slab) {
        const uint32_t at = (uint32_t)(slab >> 2) * 4u;
        raw[0] = __builtin_amdgcn_raw_buffer_load_b64(f.sa, f.vsa[0], at, 0);
        raw[1] = __builtin_amdgcn_raw_buffer_load_b64(f.sa, f.vsa[1], at, 0);
        raw_w[0] = __builtin_amdgcn_raw_buffer_load_b64(f.sb0, 0, at, 0);
        if (S::SWIGLU) raw_w[1] = __builtin_amdgcn_raw_buffer_load_b64(f.sb1, 0, at, 0);
    }
    __device__ __forceinline__ void take(int slab) {  // the slab that was asked for
        const uint32_t sh = (uint32_t)slab & 3u;
#pragma unroll
        for (int h = 0; h < 2; ++h) word[h] = __builtin_amdgcn_alignbyte(raw[h][1], raw[h][0], sh);
#pragma unroll
        for (int u = 0; u < (S::SWIGLU ? 2 : 1); ++u) word_w[u] = __builtin_amdgcn_alignbyte(raw_w[u][1], raw_w[u][0], sh);
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
// where every half is read anew as soon as its second part is done: the slab's other half of A and B1 in its first two parts,
// B0 and the first half of A of the next slab in the last two.  Either pair is a unit of the ring (see Shape8), which
// therefore stays in LDS for half a slab only:
//     barrier (unit v landed, unit v-1 no longer read) | two parts, operand reads of unit v, requests for unit v-1 + ring
// With five units of 32 KB a request has four half slabs to land in.  With slabs as units (two slots for the activations,
// three for the weights, one barrier a slab) it had two to four: 403 us for 7496 rows of 8 x 14336 x 4096, where requests
// that always hit the L2 took 318.
// Tiles with fewer rows hold two sets of operands and read slab kt+1 while they multiply slab kt, behind a barrier that lies
// after the first quarter of its instructions; their units are slabs.
// Requests complete in order, so the waits count the requests of the units that may still fly.
template <class S, bool ONCE>
struct MatrixLoop8 {
    const Fills8<S>& fills;
    Scales8<S>& scales;
    int a_lane, b_lane;  // byte offset, inside a unit's activations and half of weights, of this lane's first piece

    // where a unit's operands of this lane lie in LDS: the first and, four pieces further, the second half of a row's 128 bytes
    struct From {
        const uint8_t *lo, *hi;
        __device__ __forceinline__ From(const uint8_t* base, int lane_at) : lo(base + lane_at), hi(base + (lane_at ^ 64)) {}
        __device__ __forceinline__ void fetch(i32x8& to, int at) const {
            const u32x4 a = *(const u32x4*)(lo + at), b = *(const u32x4*)(hi + at);
            to = __builtin_bit_cast(i32x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    };

    // PHASE (0..3): where in a step this wave places its requests: the waves leave every barrier together (see ffn.hip)
    template <int LIVE, int PHASE>
    __device__ __forceinline__ void run() {
        constexpr int TN = S::TN, TH = S::TH, NM = TN * LIVE, HALF_LOADS = S::kHalfLoads;
        constexpr bool PARTS = S::parts(LIVE);
        constexpr int SETS = PARTS ? 1 : 2, STEPS = PARTS ? 2 : 1;  // units per slab
        constexpr int NU = S::units(LIVE), UNIT = S::unit(LIVE), A_BYTES = S::a_bytes(LIVE), TAIL = S::tail(LIVE), H0 = S::half0(LIVE);
        // instruction q of a slab that begins with half `set` of the activations
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
        i32x8 xa[SETS][LIVE], wb[SETS][TN];
        uint32_t dist[8], sw[2];  // scale words of the sub-tiles' rows and of the weights

        // the scales of slab kt and the one behind it come into use (second: only the latter begins this pair) and those of the
        // next pair are requested
        auto use_scales = [&](int kt, bool second) {
            const int sh = second ? 8 : 0;
            uint32_t d4[4];
            spread(scales.word[0] << sh, d4);
#pragma unroll
            for (int j = 0; j < 4; ++j) dist[j] = d4[j];
            if (LIVE > 4) {
                spread(scales.word[1] << sh, d4);
#pragma unroll
                for (int j = 0; j < 4; ++j) dist[4 + j] = d4[j];
            }
            sw[0] = scales.word_w[0] << sh;
            if (S::SWIGLU) sw[1] = scales.word_w[1] << sh;
            asm volatile("s_nop 1");  // ahead of the matrix instructions that take them (see accumulators.py)
            __builtin_amdgcn_sched_barrier(0);
            kt += second ? 1 : 2;
            scales.request(fills, fills.slab_at(kt < KT ? kt : 0));
            __builtin_amdgcn_sched_barrier(0);
        };
        // Operand read r of unit k of a slab with parity set: its weights, then its activations, in the order of use (without
        // parts: an activation, the weights, the other activations).
        auto weights_first = [](int k) constexpr { return PARTS ? k % 2 == 0 : false; };
        auto read_item = [&](auto set_c, auto k_c, auto r_c, const From& a, const From& b) {
            constexpr int set = decltype(set_c)::value, k = decltype(k_c)::value, r = decltype(r_c)::value;
            if constexpr (!PARTS) {
                constexpr int s = set ^ (k & 1);
                if constexpr (r == 0 || r > TN)
                    a.fetch(xa[s][r == 0 ? 0 : r - TN], (r == 0 ? 0 : r - TN) * 4096);
                else
                    b.fetch(wb[s][r - 1], (r - 1) / TH * (S::Base::B_SLOT / 2) + (r - 1) % TH * 2048);
            } else {
                constexpr int h = half_of(set, k), n = loads_a(set, k), from = h == 0 ? 0 : H0;
                constexpr int ra = weights_first(k) ? r - TH : r, rb = weights_first(k) ? r : r - n;
                if constexpr (ra >= 0 && ra < n)
                    a.fetch(xa[0][from + ra], ra * 4096);
                else
                    b.fetch(wb[0][k % 2 * TH + rb], rb * 2048);
            }
        };
        auto items = [loads_a](int set, int k) constexpr { return loads_a(set, k) + (PARTS ? TH : TN); };
        // where read r of the unit that is read in step `st` lies among the step's instructions (counted from its barrier)
        constexpr int LEN = NM / STEPS;                                // instructions of a step
        constexpr int QB = PARTS ? 1 : (NM / 4 > 0 ? NM / 4 : 1);      // of these, ahead of the barrier
        auto read_at = [loads_a](int set, int st, int r) constexpr {
            if (!PARTS) return QB + r * (LEN - QB) / (LIVE + TN);
            if (st == 0) return QB + r * (LEN - QB - 4) / (loads_a(set, 1) + TH);  // activations, then weights
            // weights over all of it, an activation sub-tile behind its row of the third part
            return r < TH ? QB + r * (LEN - QB - 4) / TH : (r - TH + 1) * TH;
        };
        int kt = 0, slot = 0;  // of the unit that is read
        auto up = [](int s) { return s == NU - 1 ? 0 : s + 1; };
        // One slab.  T < 0: all requests are made; otherwise TAIL - T slabs are left, this one included.
        auto slab = [&](auto set_c, auto tail_c) {
            constexpr int SET = decltype(set_c)::value, T = decltype(tail_c)::value;
            constexpr int L = T < 0 ? 1 << 20 : TAIL - T;
            if constexpr (SET == 0) use_scales(kt, false);
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
                    for (int k = K + 1; k <= K + FLY; ++k) n += loads(SET, k);
                    return n;
                };
                constexpr int YOUNGER = younger();
                static_assert(YOUNGER < 64, "vmcnt");
                const int fill_slot = slot;  // the unit that was read before
                slot = up(slot);
                const From a(smem + slot * UNIT, a_lane), b(smem + slot * UNIT + A_BYTES, b_lane);
                const uint32_t kf = (uint32_t)fills.slab_at(kt + KF / STEPS) * 128u;
                each<LEN>([&](auto q_c) {
                    constexpr int n = decltype(q_c)::value, q = ST * LEN + n;
                    constexpr At now = walk(SET, q);
                    if constexpr (n == QB) {
                        // the unit has landed for this wave (younger requests may still fly), this wave's operand reads of the
                        // one before have returned (the LDS counter is part of the wait)
                        __builtin_amdgcn_s_waitcnt(waitcnt_vm(YOUNGER));
                        __builtin_amdgcn_s_barrier();
                        __builtin_amdgcn_sched_barrier(0);
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
                    acc_mfma8<S::fragment(now.i, now.j), SET>(wb[s][now.i], xa[s][now.j], sw[S::SWIGLU ? now.i / TH : 0], dist[now.j]);
                    __builtin_amdgcn_sched_barrier(0);
                });
            });
            ++kt;
            if constexpr (SET == 1) scales.take(fills.slab_at(kt < KT ? kt : 0));
        };
        using zero = std::integral_constant<int, 0>;
        using one = std::integral_constant<int, 1>;
        using steady = std::integral_constant<int, -1>;
        auto begin = [&](auto set_c) {
            constexpr int set = decltype(set_c)::value;
            if constexpr (set == 1) use_scales(0, true);
            const From a(smem, a_lane), b(smem + A_BYTES, b_lane);
            each<items(set, 0)>([&](auto r_c) { read_item(set_c, zero{}, r_c, a, b); });
            if constexpr (S::early(LIVE) < NU) {  // the ring's last unit, whose place the exchange had
                constexpr int K = NU - 1, H = half_of(set, K), NA = loads_a(set, K);
                static_assert(PARTS, "a unit is half a slab");
                if (K < 2 * KT) {
                    const uint32_t k = (uint32_t)fills.slab_at(K / 2) * 128u;
                    each<NA>([&](auto f) { fills.one_a((H ? H0 : 0) + decltype(f)::value, k, K * UNIT + decltype(f)::value * 4096); });
                    each<HALF_LOADS>([&](auto f) { fills.one_b(K % 2, decltype(f)::value, k, K * UNIT + A_BYTES, ONCE); });
                }
            }
        };
        int left = KT - TAIL;  // slabs with all requests
        const int skip = left < 0 ? -left : 0;
        if (S::parity(LIVE, KT))
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

// The hidden activation of a block: silu(gate) * up rounded to bf16, then the 128 columns of each row quantised.  Two waves
// hold halves of a row and exchange the largest magnitudes of theirs through LDS.
template <class S>
__device__ __forceinline__ int write_hidden(const Fp8Args& p, const WorkItem& w, int wm, int wn, int lane, int live, uint8_t* smem) {
    constexpr int TM = S::TM;
    asm volatile("" : "+v"(lane));  // (see ColumnWriter)
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
                    o[k] = g[k] * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g[k] * -1.4426950408889634f)) * u[k];
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

    Fills8<S> fills;
    Scales8<S> scales;
    fills.smem = smem;
    fills.wv = wv;
    fills.weights_of_lane(lane, p.pitch);
    fills.aim(cur, p, lane, wm, wn);
    scales.begin(fills);
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
        __builtin_amdgcn_sched_barrier(0);
        scales.take_first(fills, p, fills.scale_at, lane);
        __builtin_amdgcn_s_waitcnt(waitcnt_vm(63));  // read ahead of the barrier: the ring's last unit may go there
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        auto loop = [&](auto once_c) {
            MatrixLoop8<S, decltype(once_c)::value> m{fills, scales, a_lane, b_lane};
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
            fills.aim(nxt, p, lane, wm, wn);
            scales.begin(fills);
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
void launch_fp8_shape(Fp8Args p, hipStream_t st) {
    using S = Shape8<BN, SWIGLU>;
    auto kern = fp8_gemm_kernel<S>;
    static std::atomic<uint64_t> configured{0};
    once_per_device(configured, [&] {
        (void)hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, S::kLdsBytes);
    });
    const int nb = p.n_pad / S::kNCols;
    p.tile_shift = fp8_tile_shift(p.max_rows, p.experts, nb, compute_units());
    // a block per compute unit, the same number on every XCD (which of them get items is known on the device only)
    const int grid = 8 * std::max(1, compute_units() / 8);
    p.col_group = nb % 4 == 0 ? 4 : (nb % 3 == 0 ? 3 : (nb % 2 == 0 ? 2 : 1));
    hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(S::kThreads), S::kLdsBytes, st, p);
}

// The build compiles this file once for each shape (each takes as long as all other files together).
#if CAPMOE_FP8_SHAPE == 0
template void launch_fp8_shape<256, true>(Fp8Args, hipStream_t);
#elif CAPMOE_FP8_SHAPE == 1
template void launch_fp8_shape<256, false>(Fp8Args, hipStream_t);
#else
template void launch_fp8_shape<128, false>(Fp8Args, hipStream_t);
#endif

}  // namespace capmoe
