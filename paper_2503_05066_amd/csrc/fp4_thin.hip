// Products on 4-bit expert weights for experts of few rows (fp4.hip has the others): decoding steps and any batch with a
// small capacity.
//
// The work is streaming weights.  As in the 8-bit kernel (fp8_thin.hip) a wave has 32 weight rows: 32 output columns, or the gate and up
// rows of 16 hidden columns; the waves of a block take different rows or parts of K, and each keeps a ring of its own in LDS, filled
// by direct loads, waits for its own slabs only and needs no barrier.  A slab is 128 bytes of a row, 256 k; with each come the 16 scale bytes of
// the row's 512 k around it (of every second slab from the L2: what a ring holds then has one form).
//
// The hidden activation leaves in 4 bits: 32 of its columns share a scale, which two neighbouring waves hold, so they exchange the
// largest magnitudes of their rows; with four waves to a weight row eight make a block, so that it has two neighbours.
#include <algorithm>

#include "fp4.h"
#include "narrow_tile.h"

namespace capmoe {

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(4))) int i32x4;

constexpr int kThin4WeightRows = 32;        // weight rows of a wave
constexpr int kThin4RingBytes = 20 * 1024;  // LDS of a wave
constexpr int kThin4Exchange = kThin4RingBytes - 256;  // of these, largest magnitudes of up to 32 rows

struct Thin4Args {
    const uint8_t *x, *x_scale;
    int64_t x_rows;       // rows of x (its window); permuted rows: those of the plan at most
    const int32_t* gather;
    const int32_t* expert_offset;
    const uint8_t* w[2];  // gate (or the only weights), up
    const uint8_t* w_scale[2];
    uint8_t* y;           // bf16 rows of n columns; with SWIGLU 4-bit rows of y_pitch bytes
    uint8_t* y_scale;     // with SWIGLU
    int experts, pitch, n, n_pad, scale_pitch, y_pitch, y_scale_pitch, col_blocks;
    int split;            // waves that share a row of weights, each with a part of K: 4, 2 or 1
};

__device__ __forceinline__ i32x8 operand4(const uint8_t* p) {
    const i32x4 v = *(const i32x4*)p;
    return __builtin_shufflevector(v, v, 0, 1, 2, 3, -1, -1, -1, -1);
}

// One pass: up to NR rows of an expert times a block's weight rows, of which those of its first wave begin at n0.
// ONCE: the weights' lines need not be kept.
template <int NR, bool SWIGLU, bool ONCE>
struct Thin4 {
    static constexpr int TM = (NR + 15) / 16;
    static constexpr int kCols = SWIGLU ? kThin4WeightRows / 2 : kThin4WeightRows;
    // wave-wide loads of a slab: eight rows of weights or x each, 16 rows' scales each
    static constexpr int kW = kThin4WeightRows / 8, kX = NR / 8, kWS = 2, kXS = TM;
    static constexpr int kLoads = kW + kWS + kX + kXS;
    static constexpr int kWAt = 0, kWSAt = kW * 1024, kXAt = kWSAt + kWS * 256, kXSAt = kXAt + kX * 1024;
    static constexpr int kSlot = kXSAt + kXS * 256;
    static constexpr int kRing = kThin4RingBytes / kSlot;  // slabs in flight
    static_assert(kRing >= 2 && kRing * kLoads < 64 && NR % 8 == 0, "ring");
    static_assert(2 * TM * 64 * 16 <= kThin4Exchange, "partial sums");

    static __device__ __forceinline__ void run(const Thin4Args& p, int e, int row0, int rows, int n0, uint8_t* smem) {
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));  // what follows from it is computed here, not for all shapes at the block's start
        const int lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int lr = lane & 15, lk = lane >> 4;
        n0 += wv / p.split * kCols;  // below n_pad: a block's columns divide 128
        const int slabs_all = p.pitch / kSlabBytes;
        const int part = wv & (p.split - 1);  // of K
        const int first = part * slabs_all / p.split, n = (part + 1) * slabs_all / p.split - first;
        // column blocks start their walks at different slabs: in step they would all read at the same offset of a
        // power-of-two pitch, i.e. from a few memory channels (see ffn.hip)
        const int turn = (int)((int64_t)n0 * n / p.n_pad);
        auto slab_at = [&](int s) {
            s += turn;
            return first + (s < n ? s : s - n);
        };
        uint8_t* const ring = smem + wv * kThin4RingBytes;

        // ---- rows of the activations first: through a plan their numbers take a fetch of their own ----
        // load i of rows: rows 8i .. 8i+7, lane l the piece (l % 8) ^ ((row >> 1) & 7) of row l / 8; of scales: rows 16i .. 16i+15, lane l
        // the word l % 4 of row l / 4
        uint32_t x_off[kX], xs_off[kXS];
        {
            uint32_t x_row[kX], xs_row[kXS];
#pragma unroll
            for (int i = 0; i < kX; ++i) {
                const int r = min(8 * i + (lane >> 3), rows - 1);  // rows past the end repeat the last one
                x_row[i] = p.gather ? (uint32_t)p.gather[row0 + r] : (uint32_t)r;
            }
#pragma unroll
            for (int i = 0; i < kXS; ++i) {
                const int r = min(16 * i + (lane >> 2), rows - 1);
                xs_row[i] = p.gather ? (uint32_t)p.gather[row0 + r] : (uint32_t)r;
            }
#pragma unroll
            for (int i = 0; i < kX; ++i) {
                const int r = 8 * i + (lane >> 3);
                x_off[i] = x_row[i] * (uint32_t)p.pitch + (((lane & 7) ^ ((r >> 1) & 7)) << 4);
            }
#pragma unroll
            for (int i = 0; i < kXS; ++i) xs_off[i] = xs_row[i] * (uint32_t)p.scale_pitch + ((lane & 3) << 2);
        }

        // ---- the weights' requests ----
        const int64_t w_at = (int64_t)e * p.n_pad + n0;
        auto window = [&](const uint8_t* base, int pitch) {
            return __builtin_amdgcn_make_buffer_rsrc((void*)(base + w_at * pitch), 0, kCols * pitch, kRsrcFlags);
        };
        const __amdgpu_buffer_rsrc_t r0 = window(p.w[0], p.pitch), s0 = window(p.w_scale[0], p.scale_pitch);
        const __amdgpu_buffer_rsrc_t r1 = SWIGLU ? window(p.w[1], p.pitch) : r0, s1 = SWIGLU ? window(p.w_scale[1], p.scale_pitch) : s0;
        uint32_t w_off[SWIGLU ? 2 : 4], ws_off[SWIGLU ? 1 : 2];  // of the loads of one tensor
#pragma unroll
        for (int i = 0; i < (SWIGLU ? 2 : 4); ++i) {
            const int r = 8 * i + (lane >> 3);
            w_off[i] = (uint32_t)(r * p.pitch) + (((lane & 7) ^ ((r >> 1) & 7)) << 4);
        }
#pragma unroll
        for (int i = 0; i < (SWIGLU ? 1 : 2); ++i) ws_off[i] = (uint32_t)((16 * i + (lane >> 2)) * p.scale_pitch) + ((lane & 3) << 2);
        auto request_w = [&](int s) {
            uint8_t* dst = ring + s % kRing * kSlot;
            const int at = slab_at(s);
#pragma unroll
            for (int i = 0; i < kW; ++i) {
                const __amdgpu_buffer_rsrc_t r = SWIGLU && i >= 2 ? r1 : r0;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lptr_t)(dst + kWAt + i * 1024), 16, w_off[SWIGLU ? i % 2 : i],
                                                         (uint32_t)at * kSlabBytes, 0, ONCE ? 2 : 0);
            }
#pragma unroll
            for (int i = 0; i < kWS; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(SWIGLU && i ? s1 : s0, (lptr_t)(dst + kWSAt + i * 256), 4, ws_off[SWIGLU ? 0 : i],
                                                         (uint32_t)(at >> 1) * 16u, 0, 0);
        };
        const int ahead = min(kRing, n);
        for (int u = 0; u < ahead; ++u) request_w(u);

        // ---- the activations' ----
        const int64_t x0 = p.gather ? 0 : row0;
        const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc(
            (void*)(p.x + x0 * p.pitch), 0, (int)(uint32_t)min((p.x_rows - x0) * p.pitch, (int64_t)kBeyond), kRsrcFlags);
        const __amdgpu_buffer_rsrc_t rxs = __builtin_amdgcn_make_buffer_rsrc(
            (void*)(p.x_scale + x0 * p.scale_pitch), 0, (int)(uint32_t)min((p.x_rows - x0) * p.scale_pitch, (int64_t)kBeyond), kRsrcFlags);
        auto request_x = [&](int s) {
            uint8_t* dst = ring + s % kRing * kSlot;
            const int at = slab_at(s);
#pragma unroll
            for (int i = 0; i < kX; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (lptr_t)(dst + kXAt + i * 1024), 16, x_off[i], (uint32_t)at * kSlabBytes, 0, 0);
#pragma unroll
            for (int i = 0; i < kXS; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rxs, (lptr_t)(dst + kXSAt + i * 256), 4, xs_off[i], (uint32_t)(at >> 1) * 16u, 0, 0);
        };
        for (int u = 0; u < ahead; ++u) request_x(u);
        __builtin_amdgcn_sched_barrier(0);

        f32x4 acc[2][TM];
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int m = 0; m < TM; ++m) acc[q][m] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int w_piece = lr * 128 + ((lk ^ ((lr >> 1) & 7)) << 4);  // this lane's first operand piece of a sub-tile
        const int xr = lr % NR, x_piece = xr * 128 + ((lk ^ ((xr >> 1) & 7)) << 4);  // rows past those that are fetched repeat them
        auto multiply = [&](int s) {
            const uint8_t* slot = ring + s % kRing * kSlot;
            const int half = (slab_at(s) & 1) * 2;
            i32x8 w[2][2], x[TM][2];
            int ws[2], xs[TM];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                w[q][0] = operand4(slot + kWAt + q * 2048 + w_piece), w[q][1] = operand4(slot + kWAt + q * 2048 + (w_piece ^ 64));
                ws[q] = *(const uint16_t*)(slot + kWSAt + q * 256 + lr * 16 + lk * 4 + half);
            }
#pragma unroll
            for (int m = 0; m < TM; ++m) {
                x[m][0] = operand4(slot + kXAt + m * 2048 + x_piece), x[m][1] = operand4(slot + kXAt + m * 2048 + (x_piece ^ 64));
                xs[m] = *(const uint16_t*)(slot + kXSAt + m * 256 + lr * 16 + lk * 4 + half);
            }
#pragma unroll
            for (int m = 0; m < TM; ++m)
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    acc[q][m] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w[q][0], x[m][0], acc[q][m], 4, 4, 0, ws[q], 0, xs[m]);
#pragma unroll
            for (int m = 0; m < TM; ++m)
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    acc[q][m] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w[q][1], x[m][1], acc[q][m], 4, 4, 1, ws[q], 1, xs[m]);
        };
        // A slab has landed when only younger requests are still out; its slot is refilled once its reads have returned.  The
        // first slabs' activations were requested behind all of their weights.
        for (int s = 0; s < n; ++s) {
            const int refilled = min(s, max(n - kRing, 0));  // slabs requested in this loop so far
            wait_for_all_but(max(ahead - 1 - s, 0) * (kX + kXS) + (refilled - max(s - (ahead - 1), 0)) * kLoads);
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
            for (int u = 1; u < p.split && part == 0; ++u) {
                const f32x4* other = (const f32x4*)(ring + u * kThin4RingBytes);
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
        if constexpr (SWIGLU) {
            // 16 hidden columns of each row, rounded to bf16; their largest magnitude with that of the neighbour's 16
            uint32_t v[TM][2], top[TM];
#pragma unroll
            for (int m = 0; m < TM; ++m) {
                float o[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float g = acc[0][m][k];
                    o[k] = g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.4426950408889634f)) * acc[1][m][k];
                }
                v[m][0] = pack_bf16x2(o[0], o[1]), v[m][1] = pack_bf16x2(o[2], o[3]);
                const u16x2 t = __builtin_elementwise_max(__builtin_bit_cast(u16x2, v[m][0] & 0x7fff7fffu), __builtin_bit_cast(u16x2, v[m][1] & 0x7fff7fffu));
                top[m] = max_over_rows_of_16((uint32_t)max(t[0], t[1]) << 16);
                if (part == 0 && lk == 0) *(uint32_t*)(ring + kThin4Exchange + (m * 16 + lr) * 4) = top[m];
            }
            __syncthreads();
            if (part > 0) return;
            const int block = n0 / kFp4Block;
            const bool second = (n0 & 16) != 0;
            const uint8_t* theirs = smem + (wv + (second ? -p.split : p.split)) * kThin4RingBytes + kThin4Exchange;
            auto place = [](int b) { return b / 16 * 16 + 4 * (b % 4) + b % 16 / 4; };
#pragma unroll
            for (int m = 0; m < TM; ++m) {
                const int r = m * 16 + lr;
                const uint32_t byte = fp4_scale_byte(max(top[m], *(const uint32_t*)(theirs + r * 4)));
                if (r >= rows) continue;
                uint32_t q = 0;
                if (byte != kFp4NoNumber) {
                    const float scale = __uint_as_float(byte << 23);
                    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(fp8_bf16x2, v[m][0]), scale, 0);
                    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(fp8_bf16x2, v[m][1]), scale, 1);
                }
                *(uint16_t*)(p.y + (int64_t)(row0 + r) * p.y_pitch + n0 / 2 + 2 * lk) = (uint16_t)q;
                uint8_t* s = p.y_scale + (int64_t)(row0 + r) * p.y_scale_pitch;
                if (!second && lk == 0) s[place(block)] = (uint8_t)byte;
                // behind an odd last 128 columns, what the next slab would read
                if (second && n0 + 16 == p.n_pad && p.n_pad % kFp4Slab != 0) s[place(block + 1 + lk)] = 0;
            }
        } else {
            if (part > 0) return;
#pragma unroll
            for (int m = 0; m < TM; ++m) {
                const int r = m * 16 + lr;
                if (r >= rows) continue;
                const int col = n0 + 4 * lk;  // n is a multiple of 8: four columns are all inside or all behind
                uint16_t* out = (uint16_t*)p.y + (int64_t)(row0 + r) * p.n + col;
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
template <bool SWIGLU, bool STREAM, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void fp4_thin_kernel(const Thin4Args p) {
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    constexpr int kMost = 32;  // rows of a pass
    ExpertRows x(p.expert_offset, p.experts);
    const int first = blockIdx.x / p.col_blocks, n0 = (blockIdx.x - first * p.col_blocks) * (WAVES / p.split) * Thin4<16, SWIGLU, STREAM>::kCols;
    const int step = gridDim.x / p.col_blocks;
    for (int t = first; x.find(t); t += step) {
        for (int at = 0; at < x.rows; at += kMost) {
            if (t > first || at > 0) __syncthreads();  // a wave may still read the others' sums out of their rings
            if (x.rows > kMost)
                Thin4<kMost, SWIGLU, false>::run(p, x.e, x.row0 + at, min(x.rows - at, kMost), n0, smem);
            else if (x.rows <= 8)
                Thin4<8, SWIGLU, STREAM>::run(p, x.e, x.row0, x.rows, n0, smem);
            else if (x.rows <= 16)
                Thin4<16, SWIGLU, STREAM>::run(p, x.e, x.row0, x.rows, n0, smem);
            else
                Thin4<kMost, SWIGLU, STREAM>::run(p, x.e, x.row0, x.rows, n0, smem);
        }
    }
}

template <bool SWIGLU, bool STREAM, int WAVES>
static void launch_thin4_waves(Thin4Args a, int64_t tiles, hipStream_t st) {
    constexpr int lds = WAVES * kThin4RingBytes;
    auto kern = fp4_thin_kernel<SWIGLU, STREAM, WAVES>;
    static std::atomic<uint64_t> configured{0};
    once_per_device(configured, [&] {
        (void)hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    });
    const int per_block = WAVES / a.split * Thin4<16, SWIGLU, STREAM>::kCols;
    a.col_blocks = (a.n + per_block - 1) / per_block;
    hipLaunchKernelGGL(kern, dim3((unsigned)(tiles * a.col_blocks)), dim3(64 * WAVES), lds, st, a);
}
template <bool SWIGLU, bool STREAM>
static void launch_thin4(Thin4Args a, int64_t tiles, hipStream_t st) {
    constexpr int cols = Thin4<16, SWIGLU, STREAM>::kCols;
    a.split = fp4_thin_split(tiles * ((a.n + cols - 1) / cols), a.pitch / kSlabBytes, STREAM, compute_units());
    if (SWIGLU && a.split == 4)
        launch_thin4_waves<SWIGLU, STREAM, SWIGLU ? 8 : 4>(a, tiles, st);
    else
        launch_thin4_waves<SWIGLU, STREAM, 4>(a, tiles, st);
}

void launch_fp4_thin(const Fp4Gemm& g, const int32_t* expert_offset, const void* x, const uint8_t* x_scale, int64_t x_rows,
                     const int32_t* gather, const void* w, const uint8_t* w_scale, const void* up, const uint8_t* up_scale, void* y,
                     uint8_t* y_scale, bool stream, hipStream_t st) {
    Thin4Args a;
    a.x = (const uint8_t*)x, a.x_scale = x_scale, a.x_rows = x_rows, a.gather = gather, a.expert_offset = expert_offset;
    a.w[0] = (const uint8_t*)w, a.w[1] = (const uint8_t*)up;
    a.w_scale[0] = w_scale, a.w_scale[1] = up_scale;
    a.y = (uint8_t*)y, a.y_scale = y_scale, a.y_pitch = fp4_pitch(g.n), a.y_scale_pitch = fp4_scale_pitch(g.n);
    a.experts = g.experts, a.pitch = g.pitch, a.n = g.n, a.n_pad = g.n_pad, a.scale_pitch = g.scale_pitch;
    a.col_blocks = a.split = 0;
    const int64_t tiles = std::min<int64_t>(g.max_rows, g.experts);
    auto launch = up ? (stream ? launch_thin4<true, true> : launch_thin4<true, false>)
                     : (stream ? launch_thin4<false, true> : launch_thin4<false, false>);
    launch(a, tiles, st);
}

}  // namespace capmoe
