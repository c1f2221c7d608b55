// What the products on 8-bit and on 4-bit rows share: on high row tiles (fp8.hip, fp4.hip) the order of the work and the bf16 output, on
// few rows (fp8_thin.hip, fp4_thin.hip) the experts that have any.
#pragma once

#include "ffn_tile.h"
#include "fp8_forms.h"

namespace capmoe {

constexpr int kSlabBytes = 128;  // of a row

// f(r) for the r in [FROM, N) with at(r) == POS, all known at compile time (at keeps no values)
template <int FROM, int N, int POS, class At, class F>
__device__ __forceinline__ void each_at(At at, F&& f) {
    auto find = [](At where) constexpr {
        int r = FROM;
        while (r < N && where(r) != POS) ++r;
        return r;
    };
    constexpr int r = find(at);
    if constexpr (r < N) {
        f(std::integral_constant<int, r>{});
        each_at<r + 1, N, POS>(at, f);
    }
}

// Writes sub-tile row j of a block's bf16 output (see TileWriter in ffn_tile.h); columns at or behind n are not written.
template <class S>
struct ColumnWriter {
    __amdgpu_buffer_rsrc_t c;
    uint32_t at, pitch;
    int col, n;
    template <class Args>
    __device__ __forceinline__ ColumnWriter(const Args& p, const WorkItem& w, int wm, int wn, int lane) {
        const int lr = lane & 15, lk = lane >> 4;
        n = p.n;
        pitch = (uint32_t)p.n * 2u;
        c = __builtin_amdgcn_make_buffer_rsrc((void*)(p.y + ((size_t)w.row0 * p.n + w.n0) * 2), 0,
                                              (int)((uint32_t)(w.rows - 1) * pitch + (uint32_t)min(S::kNCols, p.n - w.n0) * 2u), kRsrcFlags);
        const int in = wn * (S::kNCols / 2) + (lk & 1) * 16 + (lk >> 1) * 8;
        col = w.n0 + in;
        at = (uint32_t)(wm * 16 + lr) * pitch + (uint32_t)in * 2u;
        asm volatile("" : "+v"(at));  // what follows from it is computed for each item, not kept in registers through the loop
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

// The sum of the lanes' values up to and including the lane's own.  (By shuffles through LDS, four scans of six one after the other:
// a launch's first request 4.1 instead of 3.5 us behind its start.)
__device__ __forceinline__ int sum_up_to(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // row_shr: in rows of 16 lanes
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // row_bcast:15: a row's last lane to the next row
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // row_bcast:31
    return v;
}

// The order of the work, found by every wave for itself from the experts' offsets: no launch ahead of this one builds a
// schedule, whose lists would cost the same two dependent fetches (4 us less for each product or pair of them).
//
// First the full row tiles (256 rows, or 128 or 64: see fp8_tile_shift), expert by expert, then what is left of the experts'
// rows, higher tiles first, so that the last items are short ones.  Chunks of `deal` tiles by `group` column blocks go to the
// XCDs in turn (block id mod 8), and the blocks of an XCD take the items of its chunks in turn.  About as many tiles as an
// expert has make a chunk: those that run together on an XCD then share weight tiles in its L2, and the XCDs' shares differ little.
// Which chunk follows: with few rounds of items (up to 4.5 a block) the next column group of the same tiles, so that the heights
// fall all along, and every other round, of a block's turns and of the XCDs', runs backwards: who had the higher tile of one gets
// the lower of the next.  With more rounds the next tiles of the same column group: the heights fall once per column group, and low
// tiles, which wait for weights, run beside high ones.  The latter and the former order, us: products of 3000 tokens on
// 64 x 2048 x 1024 (1.3 rounds) 55.8, 48.2; 4096 on 32 x 4096 x 2048 (1.4) 130, 112; 9000 top-1 on 8 x 1024 x 4096 (1.8) 46.6, 50.0; 6000 on
// 8 x 4096 x 4096 (2.2) 146, 137; 12413 on 60 x 512 x 1280 (4.3) 77, 71; 8192 on 64 x 2048 x 2048 (4.6) 164, 165; 3000 on 32 x 4096 x 8192 (5.3) 304, 340;
// FFN of 3000 tokens on 8 x 4096 x 4096 (2.4) 275, 246; 4096 on 64 x 2048 x 1024 (2.7) 172, 171 to 176; 6500 (4.1) 266, 254; 8192 on
// 32 x 2048 x 2048 (5.0) 285, 298; 12413 on 60 x 512 x 1280 (8.6) 210, 218.
//
// (A ticket per item instead of turns: the same within 2 % where all items are alike, and counters that somebody has to clear.)
template <class S>
struct TileOrder {
    static constexpr int kChunks = kMaxExperts / kWave;
    const int32_t* offset;
    int ends[kChunks];  // of expert 64 c + lane: full tiles up to and including its own
    uint32_t parts;     // of place 64 c + lane among the partly filled tiles: its expert, in byte c
    int sh, full, tiles, slabs, n_pad, group, deal, inner, chunks;  // 1 << sh: rows of a full tile
    bool stream, few_rounds;

    template <class Args>
    __device__ __forceinline__ TileOrder(const Args& p, int lane, uint8_t* scratch)
        : offset(p.expert_offset), sh(p.tile_shift), slabs(p.pitch / kSlabBytes), n_pad(p.n_pad), group(p.col_group), stream(p.stream) {
        int rows[kChunks];
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int e = c * kWave + lane;
            const int lo = e < p.experts ? offset[e] : 0, hi = e < p.experts ? offset[e + 1] : 0;
            rows[c] = hi - lo;
        }
        full = 0;
        int active = 0;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            ends[c] = full + sum_up_to(rows[c] >> sh);
            full = __builtin_amdgcn_readlane(ends[c], kWave - 1);
            active += __popcll(__ballot(rows[c] > 0));
        }
        // places of the partly filled tiles: by height in steps of 32 rows, then by expert
        int n_parts = 0;
        const uint64_t below = ((uint64_t)1 << lane) - 1;
        auto word = [&](int i) { return (lds_int_t)(scratch + i * 4); };
#pragma unroll
        for (int height = 8; height > 0; --height)
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
                if (c * kWave >= p.experts) continue;
                const bool mine = ((rows[c] & ((1 << sh) - 1)) + 31) >> 5 == height;
                const uint64_t all = __ballot(mine);
                if (mine) *word(n_parts + __popcll(all & below)) = c * kWave + lane;
                n_parts += __popcll(all);
            }
        parts = 0;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) parts |= ((uint32_t)*word(c * kWave + lane) & 255u) << (8 * c);
        n_parts = __builtin_amdgcn_readfirstlane(n_parts);  // behind the branches the compiler would take it for a lane's own
        tiles = full + n_parts;
        const int columns = n_pad / S::kNCols;
        const int each = tiles / max(active, 1);  // tiles of an expert, on average
        deal = each >= 6 ? 8 : (each >= 3 ? 4 : (each >= 2 ? 2 : 1));
        // No expert has two tiles: a weight tile is one block's alone, only rows are shared, and all column blocks of a row tile make
        // a chunk (FFN of 1531 tokens on 60 x 2048 x 1408, eleven column blocks: 127 -> 120 us; where experts have two, 4096 on
        // 64 x 2048 x 1024, it would be 176 -> 191).
        if (tiles == active && tiles >= 4 * 8) group = columns;
        const int row_chunks = (tiles + deal - 1) / deal, col_groups = columns / group;
        chunks = row_chunks * col_groups;
        few_rounds = 2 * tiles * columns <= 9 * (int)gridDim.x;
        inner = few_rounds ? col_groups : row_chunks;
    }
    // position p of this XCD's share; past its end: not valid, `more` false; a place that the last chunk of a column group
    // leaves empty: not valid, `more` true
    __device__ __forceinline__ WorkItem at(int xcd, int p, bool& more) const {
        WorkItem w;
        w.valid = 0;
        const int per_chunk = deal * group, j = p / per_chunk, in = p - j * per_chunk;
        const int chunk = 8 * j + (few_rounds && (j & 1) ? 7 - xcd : xcd);
        more = chunk < chunks;
        if (!more) return w;
        const int first = chunk / inner, rest = chunk - first * inner;
        const int cg = few_rounds ? rest : first, tr = in / group;
        int tile = (few_rounds ? first : rest) * deal + tr, col = cg * group + in - tr * group;
        tile = __builtin_amdgcn_readfirstlane(tile), col = __builtin_amdgcn_readfirstlane(col);
        if (tile >= tiles) return w;
        const bool whole = tile < full;
        int e = 0, before = 0;
        if (whole) {
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {  // experts whose full tiles all come before this one
                const int n = __popcll(__ballot(ends[c] <= tile));
                e += n;
                if (n > 0) before = __builtin_amdgcn_readlane(ends[c], n - 1);
            }
        } else {
            const int at = tile - full;
            e = __builtin_amdgcn_readlane((int)parts, at & (kWave - 1)) >> (8 * (at >> 6)) & 255;
        }
        const int lo = scalar_word(offset, e), hi = scalar_word(offset, e + 1);
        w.valid = 1;
        w.e = e;
        w.n0 = col * S::kNCols;
        w.row0 = whole ? lo + ((tile - before) << sh) : lo + ((hi - lo) >> sh << sh);
        w.rows = whole ? 1 << sh : (hi - lo) & ((1 << sh) - 1);
        // an expert's only tile, in a layer whose weights the memory-side cache does not keep (see ffn.hip)
        w.once = stream && hi - lo <= 1 << sh;
        w.first = 0;
        w.slabs = slabs;
        w.turn = w.once ? (int)((long long)w.n0 * slabs / n_pad) : 0;
        return w;
    }
    // the item that block `turn` of an XCD's `blocks` takes in its round `round`, or the next one that it has
    __device__ __forceinline__ WorkItem next(int xcd, int& round, int turn, int blocks) const {
        bool more = true;
        WorkItem w;
        do {
            w = at(xcd, round * blocks + (few_rounds && (round & 1) ? blocks - 1 - turn : turn), more);
            ++round;
        } while (more && !w.valid);
        return w;
    }
};

// The t-th expert that has rows: its id and rows, or false.  Every wave looks it up for itself.
struct ExpertRows {
    int e, row0, rows;
    int lo[kMaxExperts / kWave], hi[kMaxExperts / kWave];
    __device__ __forceinline__ ExpertRows(const int32_t* offset, int experts) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int c = 0; c < kMaxExperts / kWave; ++c) {
            const int i = c * kWave + lane;
            lo[c] = i < experts ? offset[i] : 0;
            hi[c] = i < experts ? offset[i + 1] : 0;
        }
    }
    __device__ __forceinline__ bool find(int t) {
        bool found = false;
#pragma unroll
        for (int c = 0; c < kMaxExperts / kWave; ++c) {
            const uint64_t has = __ballot(hi[c] > lo[c]);
            const int n = __popcll(has);
            if (!found && t < n) {
                const int rank = __builtin_amdgcn_mbcnt_hi((uint32_t)(has >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)has, 0));
                const uint64_t it = __ballot(hi[c] > lo[c] && rank == t);
                const int at = __builtin_ctzll(it);
                e = c * kWave + at;
                row0 = __builtin_amdgcn_readlane(lo[c], at);
                rows = __builtin_amdgcn_readlane(hi[c], at) - row0;
                found = true;
            }
            t -= n;
        }
        return found;
    }
};

}  // namespace capmoe
