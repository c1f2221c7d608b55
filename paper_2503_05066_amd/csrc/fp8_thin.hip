// Products on 8-bit expert weights for experts of few rows (fp8.hip has the others): decoding steps and any batch with a
// small capacity.
//
// The work is streaming weights.  A wave has 32 weight rows: 32 output columns, or the gate and up rows of 16 hidden
// columns.  The four waves of a block take different rows or parts of K (see fp8_thin_split) and share nothing until the end: each
// keeps a ring of its own in LDS, filled by direct loads, waits for its own slabs only and needs no barrier (as the bf16 kernel,
// ffn_thin.hip).  Two blocks share a compute unit.
//
// bf16 activations are quantised as they leave LDS: every block does it for itself, for up to 16 rows of a
// slab beside 4 KB of weights, which take longer to arrive; kernels of their own for it, one ahead of either product,
// would cost their launches.  Nor is there a tile schedule: a block finds its expert in the offsets.
#include <algorithm>

#include "fp8.h"
#include "narrow_tile.h"

namespace capmoe {

typedef __attribute__((ext_vector_type(8))) int i32x8;

constexpr int kThin8WeightRows = 32;         // weight rows of a wave
constexpr int kThin8Waves = 4;               // waves of a block
constexpr int kThin8RingBytes = 20 * 1024;   // LDS of a wave

struct Thin8Args {
    const void* x;
    const uint8_t* x_scale;
    int64_t x_rows;       // rows of x (its window); permuted rows: those of the plan at most
    const int32_t* gather;
    const int32_t* expert_offset;
    const uint8_t* w[2];  // gate (or the only weights), up
    const uint8_t* w_scale[2];
    uint16_t* y;
    int experts, k, pitch, n, n_pad, scale_pitch, col_blocks;
    int split;            // waves that share a row of weights, each with a part of K: 4, 2 or 1
};

// One pass: up to NR rows of an expert times a block's weight rows, of which those of its first wave begin at n0.
// QUANT: x is bf16.  ONCE: the weights' lines need not be kept.
template <int NR, bool SWIGLU, bool QUANT, bool ONCE>
struct Thin8 {
    static constexpr int TM = (NR + 15) / 16;
    static constexpr int kCols = SWIGLU ? kThin8WeightRows / 2 : kThin8WeightRows;
    // wave-wide loads of a slab of 128 k: eight weight rows, four bf16 rows or eight 8-bit rows each, and the latter's scales
    static constexpr int kW = kThin8WeightRows / 8, kX = QUANT ? NR / 4 : NR / 8, kS = QUANT ? 0 : 1;
    static constexpr int kLoads = kW + kX + kS;
    static constexpr int kSlot = (kW + kX) * 1024 + kS * 256;
    static constexpr int kRing = kThin8RingBytes / kSlot;  // slabs in flight
    static_assert(kRing >= 2 && kRing * kLoads < 64 && NR % 4 == 0 && (QUANT || NR % 8 == 0), "ring");
    static_assert(2 * TM * 64 * 16 <= kThin8RingBytes, "partial sums");

    static __device__ __forceinline__ void run(const Thin8Args& p, int e, int row0, int rows, int n0, uint8_t* smem) {
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));  // what follows from it is computed here, not for all shapes at the block's start
        const int lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int lr = lane & 15, lk = lane >> 4;
        n0 += wv / p.split * kCols;  // below n_pad: a block's columns divide 128
        const int slabs_all = p.pitch / kFp8Block;
        const int part = wv & (p.split - 1);  // of K
        const int first = part * slabs_all / p.split, n = (part + 1) * slabs_all / p.split - first;
        // column blocks start their walks at different slabs: in step they would all read at the same offset of a
        // power-of-two pitch, i.e. from a few memory channels (see ffn.hip)
        const int turn = (int)((int64_t)n0 * n / p.n_pad);
        auto slab_at = [&](int s) {
            s += turn;
            return first + (s < n ? s : s - n);
        };
        uint8_t* const ring = smem + wv * kThin8RingBytes;

        // ---- rows of the activations first: through a plan their numbers take a fetch of their own ----
        // load i of bf16 rows: rows 4i .. 4i+3, lane l the piece (l % 16) ^ row of row l / 16; of 8-bit rows: rows 8i .. 8i+7,
        // lane l the piece (l % 8) ^ ((row >> 1) & 7) of row l / 8
        uint32_t x_row[kX], s_row = 0;
#pragma unroll
        for (int i = 0; i < kX; ++i) {
            const int r = min(QUANT ? 4 * i + (lane >> 4) : 8 * i + (lane >> 3), rows - 1);  // rows past the end repeat the last one
            x_row[i] = p.gather ? (uint32_t)p.gather[row0 + r] : (uint32_t)r;
        }
        if (!QUANT) {
            const int r = min(lane, rows - 1);
            s_row = p.gather ? (uint32_t)p.gather[row0 + r] : (uint32_t)r;
        }

        // ---- the weights' requests ----
        const int64_t w_at = (int64_t)e * p.n_pad + n0;
        const __amdgpu_buffer_rsrc_t r0 =
            __builtin_amdgcn_make_buffer_rsrc((void*)(p.w[0] + w_at * p.pitch), 0, kCols * p.pitch, kRsrcFlags);
        const __amdgpu_buffer_rsrc_t r1 =
            SWIGLU ? __builtin_amdgcn_make_buffer_rsrc((void*)(p.w[1] + w_at * p.pitch), 0, kCols * p.pitch, kRsrcFlags) : r0;
        const int32_t* scale0 = (const int32_t*)(p.w_scale[0] + w_at / kFp8Block * p.scale_pitch);
        const int32_t* scale1 = SWIGLU ? (const int32_t*)(p.w_scale[1] + w_at / kFp8Block * p.scale_pitch) : scale0;
        uint32_t w_off[SWIGLU ? 2 : 4];  // of the loads of one tensor
#pragma unroll
        for (int i = 0; i < (SWIGLU ? 2 : 4); ++i) {
            const int r = 8 * i + (lane >> 3);
            w_off[i] = (uint32_t)(r * p.pitch) + (((lane & 7) ^ ((r >> 1) & 7)) << 4);
        }
        auto request_w = [&](int s) {
            uint8_t* dst = ring + s % kRing * kSlot;
            const uint32_t k_bytes = (uint32_t)slab_at(s) * kFp8Block;
#pragma unroll
            for (int i = 0; i < kW; ++i) {
                const __amdgpu_buffer_rsrc_t r = SWIGLU && i >= 2 ? r1 : r0;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lptr_t)(dst + i * 1024), 16, w_off[SWIGLU ? i % 2 : i], k_bytes, 0, ONCE ? 2 : 0);
            }
        };
        const int ahead = min(kRing, n);
        for (int u = 0; u < ahead; ++u) request_w(u);

        // ---- the activations' ----
        const int64_t x_pitch = QUANT ? (int64_t)p.k * 2 : p.pitch;
        const int64_t x0 = p.gather ? 0 : row0;
        const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc(
            (void*)((const uint8_t*)p.x + x0 * x_pitch), 0, (int)(uint32_t)min((p.x_rows - x0) * x_pitch, (int64_t)kBeyond), kRsrcFlags);
        const __amdgpu_buffer_rsrc_t rxs =
            QUANT ? rx
                  : __builtin_amdgcn_make_buffer_rsrc((void*)(p.x_scale + x0 * p.scale_pitch), 0,
                                                      (int)(uint32_t)min((p.x_rows - x0) * p.scale_pitch, (int64_t)kBeyond), kRsrcFlags);
        uint32_t x_off[kX];
#pragma unroll
        for (int i = 0; i < kX; ++i) {
            const int r = QUANT ? 4 * i + (lane >> 4) : 8 * i + (lane >> 3);
            const int piece = QUANT ? (lane & 15) ^ (r & 15) : (lane & 7) ^ ((r >> 1) & 7);
            x_off[i] = x_row[i] * (uint32_t)x_pitch + (piece << 4);
        }
        s_row *= (uint32_t)p.scale_pitch;
        auto request_x = [&](int s) {
            uint8_t* dst = ring + s % kRing * kSlot + kW * 1024;
            const int at = slab_at(s);
            if (QUANT) {
                // pieces behind the row's end (the last slab of a k that is no multiple of 128) are read as zeros: from
                // behind the window
                const uint32_t k_bytes = (uint32_t)at * (2 * kFp8Block);
                const int left = p.k - at * kFp8Block;
#pragma unroll
                for (int i = 0; i < kX; ++i) {
                    const int piece = (lane & 15) ^ ((4 * i + (lane >> 4)) & 15);
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (lptr_t)(dst + i * 1024), 16, piece * 8 < left ? x_off[i] + k_bytes : kBeyond, 0, 0, 0);
                }
            } else {
#pragma unroll
                for (int i = 0; i < kX; ++i)
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (lptr_t)(dst + i * 1024), 16, x_off[i], (uint32_t)at * kFp8Block, 0, 0);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rxs, (lptr_t)(dst + kX * 1024), 4, s_row, (uint32_t)at & ~3u, 0, 0);
            }
        };
        for (int u = 0; u < ahead; ++u) request_x(u);
        __builtin_amdgcn_sched_barrier(0);

        f32x4 acc[2][TM];
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int m = 0; m < TM; ++m) acc[q][m] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int w_piece = lr * 128 + ((lk ^ ((lr >> 1) & 7)) << 4);  // this lane's first operand piece of a sub-tile
        auto fetch = [&](const uint8_t* at) {
            const u32x4 lo = *(const u32x4*)(at + w_piece), hi = *(const u32x4*)(at + (w_piece ^ 64));
            return __builtin_bit_cast(i32x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        };
        int scale_word[2] = {scalar_word(scale0, slab_at(0) >> 2), SWIGLU ? scalar_word(scale1, slab_at(0) >> 2) : 0};
        auto multiply = [&](int s) {
            const uint8_t* slot = ring + s % kRing * kSlot;
            const int at = slab_at(s), sh = (at & 3) * 8;
            const int ws[2] = {scale_word[0] >> sh, SWIGLU ? scale_word[1] >> sh : scale_word[0] >> sh};
            i32x8 w[2], x[TM];
            uint32_t byte[TM];
#pragma unroll
            for (int q = 0; q < 2; ++q) w[q] = fetch(slot + q * 16 * 128);
            if constexpr (QUANT) {
                // rows past those that are fetched repeat them: their columns are not stored
                const uint8_t* xs = slot + kW * 1024 + (lr % NR) * 256;
                uint32_t v[16];
#pragma unroll
                for (int h = 0; h < 4; ++h) {  // pieces 2 lk, 2 lk + 1, and eight further
                    const u32x4 d = *(const u32x4*)(xs + (((2 * lk + (h & 1) + 8 * (h >> 1)) ^ (lr % NR)) << 4));
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[4 * h + i] = d[i];
                }
                u16x2 top2 = {0, 0};
#pragma unroll
                for (int i = 0; i < 16; ++i) top2 = __builtin_elementwise_max(top2, __builtin_bit_cast(u16x2, v[i] & 0x7fff7fffu));
                uint32_t top = max(top2[0], top2[1]), bad = 0;
                const bool odd = __ballot(top >= 0x7f80u) != 0;  // values that are not finite: rare, out of the way
                if (__builtin_expect(odd, 0)) top = amax_bf16(v, bad);
                byte[0] = scale_byte(max_over_rows_of_16(top) << 16);
                uint32_t packed[8];
                to_e4m3(v, byte[0], packed);
                if (__builtin_expect(odd, 0)) mark_bad(packed, bad);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[0][i] = (int)packed[i];
            } else {
#pragma unroll
                for (int m = 0; m < TM; ++m) {
                    x[m] = fetch(slot + kW * 1024 + m * 16 * 128);
                    byte[m] = *(const uint32_t*)(slot + (kW + kX) * 1024 + (16 * m + lr) * 4) >> sh;
                }
            }
            if (s + 1 < n) {  // the next slab's, if they lie in another word
                scale_word[0] = scalar_word(scale0, slab_at(s + 1) >> 2);
                if (SWIGLU) scale_word[1] = scalar_word(scale1, slab_at(s + 1) >> 2);
            }
#pragma unroll
            for (int m = 0; m < TM; ++m)
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    acc[q][m] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w[q], x[m], acc[q][m], 0, 0, 0, ws[q], 0, (int)byte[m]);
        };
        // A slab has landed when only younger requests are still out; its slot is refilled once its reads have returned.  The
        // first slabs' activations were requested behind all of their weights.
        for (int s = 0; s < n; ++s) {
            const int refilled = min(s, max(n - kRing, 0));  // slabs requested in this loop so far
            wait_for_all_but(max(ahead - 1 - s, 0) * (kX + kS) + (refilled - max(s - (ahead - 1), 0)) * kLoads);
            __builtin_amdgcn_sched_barrier(0);
            multiply(s);
            __builtin_amdgcn_sched_barrier(0);
            if (s + kRing < n) {
                __builtin_amdgcn_s_waitcnt(waitcnt_vm(63));  // this wave's reads have returned
                request_w(s + kRing);
                request_x(s + kRing);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        // ---- partial tiles meet in LDS (every wave in its own ring) and are added in wave order ----
        if (p.split > 1) {
            f32x4* mine = (f32x4*)ring;
            if (part > 0) {
#pragma unroll
                for (int q = 0; q < 2; ++q)
#pragma unroll
                    for (int m = 0; m < TM; ++m) mine[(q * TM + m) * 64 + lane] = acc[q][m];
            }
            __syncthreads();
            if (part > 0) return;
            for (int u = 1; u < p.split; ++u) {
                const f32x4* other = (const f32x4*)(ring + u * kThin8RingBytes);
#pragma unroll
                for (int q = 0; q < 2; ++q)
#pragma unroll
                    for (int m = 0; m < TM; ++m) {
                        const f32x4 o = other[(q * TM + m) * 64 + lane];
#pragma unroll
                        for (int v = 0; v < 4; ++v) acc[q][m][v] += o[v];
                    }
            }
        }
#pragma unroll
        for (int m = 0; m < TM; ++m) {
            const int r = m * 16 + lr;
            if (r >= rows) continue;
            const int col = n0 + 4 * lk;  // n is a multiple of 8: four columns are all inside or all behind
            uint16_t* out = p.y + (int64_t)(row0 + r) * p.n + col;
            if (SWIGLU) {
                float o[4];
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const float g = acc[0][m][v];
                    o[v] = g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.4426950408889634f)) * acc[1][m][v];
                }
                if (col < p.n) *(uint2*)out = make_uint2(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]));
            } else {
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const f32x4 o = acc[q][m];
                    if (col + 16 * q < p.n) *(uint2*)(out + 16 * q) = make_uint2(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]));
                }
            }
        }
    }
};

// The blocks take the experts in turn; one with more rows than a pass holds is done in passes over the same weights, which are
// then fetched to be kept.
template <bool SWIGLU, bool QUANT, bool STREAM>
__global__ __launch_bounds__(64 * kThin8Waves, 2) void fp8_thin_kernel(const Thin8Args p) {
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    constexpr int kMost = QUANT ? 16 : 32;  // rows of a pass
    ExpertRows x(p.expert_offset, p.experts);
    const int first = blockIdx.x / p.col_blocks, n0 = (blockIdx.x - first * p.col_blocks) * (kThin8Waves / p.split) * Thin8<16, SWIGLU, QUANT, STREAM>::kCols;
    const int step = gridDim.x / p.col_blocks;
    for (int t = first; x.find(t); t += step) {
        for (int at = 0; at < x.rows; at += kMost) {
            if (t > first || at > 0) __syncthreads();  // a wave may still read the others' sums out of their rings
            if (x.rows > kMost)
                Thin8<kMost, SWIGLU, QUANT, false>::run(p, x.e, x.row0 + at, min(x.rows - at, kMost), n0, smem);
            else if (QUANT && x.rows <= 4)
                Thin8<QUANT ? 4 : 16, SWIGLU, QUANT, STREAM>::run(p, x.e, x.row0, x.rows, n0, smem);
            else if (QUANT ? x.rows <= 8 : x.rows <= 16)
                Thin8<QUANT ? 8 : 16, SWIGLU, QUANT, STREAM>::run(p, x.e, x.row0, x.rows, n0, smem);
            else
                Thin8<kMost, SWIGLU, QUANT, STREAM>::run(p, x.e, x.row0, x.rows, n0, smem);
        }
    }
}

template <bool SWIGLU, bool QUANT, bool STREAM>
static void launch_thin8(Thin8Args a, int64_t tiles, hipStream_t st) {
    constexpr int lds = kThin8Waves * kThin8RingBytes;
    auto kern = fp8_thin_kernel<SWIGLU, QUANT, STREAM>;
    static std::atomic<uint64_t> configured{0};
    once_per_device(configured, [&] {
        (void)hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    });
    constexpr int cols = Thin8<16, SWIGLU, QUANT, STREAM>::kCols;
    a.split = fp8_thin_split(tiles * ((a.n + cols - 1) / cols), a.pitch / kFp8Block, compute_units());
    const int per_block = kThin8Waves / a.split * cols;
    a.col_blocks = (a.n + per_block - 1) / per_block;
    hipLaunchKernelGGL(kern, dim3((unsigned)(tiles * a.col_blocks)), dim3(64 * kThin8Waves), lds, st, a);
}

static Thin8Args thin8_args(const Fp8Gemm& g, const int32_t* expert_offset, const void* x, const uint8_t* x_scale, int64_t x_rows,
                            const int32_t* gather, const void* w, const uint8_t* w_scale, const void* up, const uint8_t* up_scale,
                            void* y) {
    Thin8Args a;
    a.x = x, a.x_scale = x_scale, a.x_rows = x_rows, a.gather = gather, a.expert_offset = expert_offset;
    a.w[0] = (const uint8_t*)w, a.w[1] = (const uint8_t*)up;
    a.w_scale[0] = w_scale, a.w_scale[1] = up_scale;
    a.y = (uint16_t*)y;
    a.experts = g.experts, a.k = g.k, a.pitch = g.pitch, a.n = g.n, a.n_pad = g.n_pad, a.scale_pitch = fp8_scale_pitch(g.k);
    a.col_blocks = a.split = 0;
    return a;
}
static int64_t thin8_tiles(const Fp8Gemm& g) { return std::min<int64_t>(g.max_rows, g.experts); }

void launch_fp8_thin(const Fp8Gemm& g, const int32_t* expert_offset, const void* x, const uint8_t* x_scale, int64_t x_rows,
                     const int32_t* gather, const void* w, const uint8_t* w_scale, void* y, bool stream, hipStream_t st) {
    const Thin8Args a = thin8_args(g, expert_offset, x, x_scale, x_rows, gather, w, w_scale, nullptr, nullptr, y);
    auto launch = x_scale ? (stream ? launch_thin8<false, false, true> : launch_thin8<false, false, false>)
                          : (stream ? launch_thin8<false, true, true> : launch_thin8<false, true, false>);
    launch(a, thin8_tiles(g), st);
}

void launch_fp8_thin_gate_up(const Fp8Gemm& g, const int32_t* expert_offset, const void* x, int64_t x_rows, const int32_t* gather,
                             const moe_fp8_experts_t& w, void* y, bool stream, hipStream_t st) {
    const Thin8Args a = thin8_args(g, expert_offset, x, nullptr, x_rows, gather, w.gate, w.gate_scale, w.up, w.up_scale, y);
    auto launch = stream ? launch_thin8<true, true, true> : launch_thin8<true, true, false>;
    launch(a, thin8_tiles(g), st);
}

}  // namespace capmoe
