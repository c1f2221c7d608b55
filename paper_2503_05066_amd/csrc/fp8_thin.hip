// Products on 8-bit expert weights for tiles of few rows (fp8.hip has the others): decoding steps and any batch with a
// small capacity.
//
// The work is streaming weights.  A block has 32 weight rows: 32 output columns, or the gate and up rows of 16 hidden
// columns.  Its four waves split K and share nothing until the end.  A weight byte is used by one wave once (tiles of up to
// 32 rows), so it goes from memory into registers, kRing slabs ahead, and never through LDS; so do the activations, of
// which lane l needs the pieces l >> 4 and (l >> 4) + 4 of row l & 15, as of the weights: both operands number the k of a
// slab alike, which is all a sum over k asks for.
//
// bf16 activations are quantised as they arrive (every block does it for itself: two thirds of the instructions of a slab,
// beside a stream that takes longer), which saves the launch and the round trip of a kernel that does it first.
#include <algorithm>

#include "ffn_tile.h"
#include "fp8.h"

namespace capmoe {

typedef __attribute__((ext_vector_type(8))) int i32x8;

constexpr int kThin8Rows = 32;         // activation rows of a pass, in sub-tiles of 16
constexpr int kThin8WeightRows = 32;   // weight rows of a block
constexpr int kThin8Waves = 4;

struct Thin8Args {
    const void* x;
    const uint8_t* x_scale;
    int64_t x_rows;       // rows of x (its window); permuted rows: those of the plan at most
    const int32_t* gather;
    const uint8_t* w[2];  // gate (or the only weights), up
    const uint8_t* w_scale[2];
    uint16_t* y;
    const int32_t *tile_expert, *tile_row0, *tile_rows, *n_tiles;
    int k, pitch, n, n_pad, scale_pitch, col_blocks;
};

// One pass: up to 16 * TM rows of an expert times a block's weight rows.
// QUANT: x is bf16.  ONCE: the weights' lines need not be kept.
template <int TM, bool SWIGLU, bool QUANT, bool ONCE>
struct Thin8 {
    static constexpr int kCols = SWIGLU ? kThin8WeightRows / 2 : kThin8WeightRows;
    static constexpr int kRing = TM == 1 ? 4 : 3;  // slabs of 128 k in flight
    static constexpr int kX = QUANT ? 4 : 2;       // 16-byte pieces of a row's slab that a lane holds
    struct Slab {
        u32x4 w[2][2], x[TM][kX];
        uint32_t w_scale[SWIGLU ? 2 : 1], x_scale[TM];
    };

    static __device__ __forceinline__ void run(const Thin8Args& p, int e, int row0, int rows, int n0, uint8_t* smem) {
        const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int lr = lane & 15, lk = lane >> 4;
        const int slabs_all = p.pitch / kFp8Block;
        const int first = wv * slabs_all / kThin8Waves, n = (wv + 1) * slabs_all / kThin8Waves - first;
        // column blocks start their walks at different slabs: in step they would all read at the same offset of a
        // power-of-two pitch, i.e. from a few memory channels (see ffn.hip)
        const int turn = (int)((int64_t)n0 * n / p.n_pad);

        __amdgpu_buffer_rsrc_t rw[2], rs[2];
#pragma unroll
        for (int u = 0; u < (SWIGLU ? 2 : 1); ++u) {
            const int64_t at = (int64_t)e * p.n_pad + n0;
            rw[u] = __builtin_amdgcn_make_buffer_rsrc((void*)(p.w[u] + at * p.pitch), 0, kCols * p.pitch, kRsrcFlags);
            rs[u] = __builtin_amdgcn_make_buffer_rsrc((void*)(p.w_scale[u] + at / kFp8Block * p.scale_pitch), 0, p.scale_pitch, kRsrcFlags);
        }
        const int64_t x_pitch = QUANT ? (int64_t)p.k * 2 : p.pitch;
        const int64_t x0 = p.gather ? 0 : row0;
        const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc(
            (void*)((const uint8_t*)p.x + x0 * x_pitch), 0, (int)(uint32_t)min((p.x_rows - x0) * x_pitch, (int64_t)kBeyond), kRsrcFlags);
        const __amdgpu_buffer_rsrc_t rxs =
            QUANT ? rx
                  : __builtin_amdgcn_make_buffer_rsrc((void*)(p.x_scale + x0 * p.scale_pitch), 0,
                                                      (int)(uint32_t)min((p.x_rows - x0) * p.scale_pitch, (int64_t)kBeyond), kRsrcFlags);
        uint32_t row[TM];
#pragma unroll
        for (int m = 0; m < TM; ++m) {
            const int r = min(16 * m + lr, rows - 1);  // rows past the expert's end repeat its last row
            row[m] = p.gather ? (uint32_t)p.gather[row0 + r] : (uint32_t)r;
        }
        // slab s of this wave's walk; past its end the same requests go out to places behind the windows, which fetch nothing
        // (without a branch the compiler knows how many requests are younger than the one it waits for)
        auto load = [&](Slab& b, int s) {
            int at = s + turn;
            at = first + (at < n ? at : at - n);
            const bool in = s < n;
            const uint32_t k0 = (uint32_t)at * kFp8Block;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const uint32_t off = in ? (uint32_t)((SWIGLU ? lr : 16 * q + lr) * p.pitch) + k0 + 16 * lk : kBeyond;
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    b.w[q][h] = __builtin_amdgcn_raw_buffer_load_b128(rw[SWIGLU ? q : 0], off + (in ? 64 * h : 0), 0, ONCE ? 2 : 0);
            }
#pragma unroll
            for (int u = 0; u < (SWIGLU ? 2 : 1); ++u)
                b.w_scale[u] = __builtin_amdgcn_raw_buffer_load_b8(rs[u], in ? (uint32_t)at : kBeyond, 0, 0);
#pragma unroll
            for (int m = 0; m < TM; ++m) {
                if (QUANT) {
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        const uint32_t col = k0 + 16 * lk + 64 * (h / 2) + 8 * (h % 2);
                        b.x[m][h] = __builtin_amdgcn_raw_buffer_load_b128(
                            rx, in && col < (uint32_t)p.k ? (row[m] * (uint32_t)p.k + col) * 2u : kBeyond, 0, 0);
                    }
                } else {
                    const uint32_t off = in ? row[m] * (uint32_t)p.pitch + k0 + 16 * lk : kBeyond;
#pragma unroll
                    for (int h = 0; h < 2; ++h) b.x[m][h % kX] = __builtin_amdgcn_raw_buffer_load_b128(rx, off + (in ? 64 * h : 0), 0, 0);
                    b.x_scale[m] = __builtin_amdgcn_raw_buffer_load_b8(rxs, in ? row[m] * (uint32_t)p.scale_pitch + at : kBeyond, 0, 0);
                }
            }
        };
        f32x4 acc[2][TM];
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int m = 0; m < TM; ++m) acc[q][m] = f32x4{0.f, 0.f, 0.f, 0.f};
        auto multiply = [&](const Slab& b) {
            i32x8 w[2];
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int i = 0; i < 8; ++i) w[q][i] = (int)b.w[q][i / 4][i % 4];
#pragma unroll
            for (int m = 0; m < TM; ++m) {
                i32x8 x;
                uint32_t byte;
                if constexpr (QUANT) {
                    uint32_t v[16], packed[8], bad;
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = b.x[m][i / 4][i % 4];
                    const uint32_t top = max_over_rows_of_16(amax_bf16(v, bad));
                    byte = scale_byte(top << 16);
                    to_e4m3(v, byte, packed);
                    mark_bad(packed, bad);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = (int)packed[i];
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = (int)b.x[m][i / 4][i % 4];
                    byte = b.x_scale[m];
                }
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    acc[q][m] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w[q], x, acc[q][m], 0, 0, 0,
                                                                                 (int)b.w_scale[SWIGLU ? q : 0], 0, (int)byte);
            }
        };
        Slab ring[kRing];
#pragma unroll
        for (int u = 0; u < kRing; ++u) load(ring[u], u);
        for (int s = 0; s < n; s += kRing) {
#pragma unroll
            for (int u = 0; u < kRing; ++u) {
                multiply(ring[u]);
                load(ring[u], s + u + kRing);
            }
        }
        // ---- the four partial tiles meet in LDS and are added in wave order ----
        f32x4* mine = (f32x4*)smem + (wv * 2 * TM) * 64;
        if (wv > 0) {
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int m = 0; m < TM; ++m) mine[(q * TM + m) * 64 + lane] = acc[q][m];
        }
        __syncthreads();
        if (wv > 0) return;
#pragma unroll
        for (int u = 1; u < kThin8Waves; ++u) {
            const f32x4* part = (const f32x4*)smem + (u * 2 * TM) * 64;
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int m = 0; m < TM; ++m) {
                    const f32x4 o = part[(q * TM + m) * 64 + lane];
#pragma unroll
                    for (int v = 0; v < 4; ++v) acc[q][m][v] += o[v];
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
                    o[v] = g * acc[1][m][v] * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.4426950408889634f));
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

// The blocks walk the joint tile list, as often around as it takes; a tile of more than 32 rows is done in passes over the
// same weights, which are then fetched to be kept.
template <bool SWIGLU, bool QUANT, bool STREAM>
__global__ __launch_bounds__(64 * kThin8Waves, 2) void fp8_thin_kernel(const Thin8Args p) {
    __shared__ __attribute__((aligned(16))) uint8_t smem[kThin8Waves * 2 * 2 * 64 * sizeof(f32x4)];
    const int first = blockIdx.x / p.col_blocks, n0 = (blockIdx.x - first * p.col_blocks) * Thin8<1, SWIGLU, QUANT, STREAM>::kCols;
    const int step = gridDim.x / p.col_blocks, nt = *p.n_tiles;
    for (int tile = first; tile < nt; tile += step) {
        const int e = p.tile_expert[tile], row0 = p.tile_row0[tile], rows = p.tile_rows[tile] & kTileRowsMask;
        for (int at = 0; at < rows; at += kThin8Rows) {
            if (tile > first || at > 0) __syncthreads();  // the first wave reads the others' sums
            const int left = rows - at;
            if (rows > kThin8Rows)
                Thin8<2, SWIGLU, QUANT, false>::run(p, e, row0 + at, min(left, kThin8Rows), n0, smem);
            else if (rows > 16)
                Thin8<2, SWIGLU, QUANT, STREAM>::run(p, e, row0, rows, n0, smem);
            else
                Thin8<1, SWIGLU, QUANT, STREAM>::run(p, e, row0, rows, n0, smem);
        }
    }
}

template <bool SWIGLU, bool QUANT, bool STREAM>
static void launch_thin8(Thin8Args a, int64_t tiles, hipStream_t st) {
    constexpr int cols = Thin8<1, SWIGLU, QUANT, STREAM>::kCols;
    a.col_blocks = (a.n + cols - 1) / cols;
    hipLaunchKernelGGL((fp8_thin_kernel<SWIGLU, QUANT, STREAM>), dim3((unsigned)(tiles * a.col_blocks)), dim3(64 * kThin8Waves), 0, st, a);
}

void launch_fp8_thin(const Fp8Gemm& g, const FfnWorkspace& ws, const void* x, const uint8_t* x_scale, int64_t x_rows,
                     const int32_t* gather, const void* w, const uint8_t* w_scale, const void* up, const uint8_t* up_scale,
                     void* y, bool stream, hipStream_t st) {
    Thin8Args a;
    a.x = x, a.x_scale = x_scale, a.x_rows = x_rows, a.gather = gather;
    a.w[0] = (const uint8_t*)w, a.w[1] = (const uint8_t*)up;
    a.w_scale[0] = w_scale, a.w_scale[1] = up_scale;
    a.y = (uint16_t*)y;
    a.tile_expert = ws.all.expert, a.tile_row0 = ws.all.row0, a.tile_rows = ws.all.rows, a.n_tiles = ws.all.count;
    a.k = g.k, a.pitch = g.pitch, a.n = g.n, a.n_pad = g.n_pad, a.scale_pitch = fp8_scale_pitch(g.k), a.col_blocks = 0;
    const int64_t tiles = std::min<int64_t>(g.max_rows, g.experts);
    const int form = (up ? 4 : 0) + (x_scale ? 0 : 2) + (stream ? 1 : 0);
    switch (form) {
        case 0: launch_thin8<false, false, false>(a, tiles, st); break;
        case 1: launch_thin8<false, false, true>(a, tiles, st); break;
        case 2: launch_thin8<false, true, false>(a, tiles, st); break;
        case 3: launch_thin8<false, true, true>(a, tiles, st); break;
        case 6: launch_thin8<true, true, false>(a, tiles, st); break;
        default: launch_thin8<true, true, true>(a, tiles, st); break;
    }
}

}  // namespace capmoe
