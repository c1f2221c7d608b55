// Sizes of the 8-bit format and the rules by which a call on 8-bit experts takes its kernels and their shapes (host code; the
// kernels are in fp8_thin.hip, few rows, and fp8.hip, high row tiles).
#pragma once

#include <algorithm>

#include "common.h"

namespace capmoe {

constexpr int kFp8Block = 128;          // values of a row, and rows of a weight matrix, that share a scale
constexpr int kFp8MaxWidth = 1 << 21;   // columns of a matrix: offsets inside a tile of 256 rows stay below 2^32
constexpr uint32_t kBeyond = 0xfffffff0u;  // a buffer offset that lies behind every window

__host__ __device__ inline int fp8_blocks(int cols) { return (cols + kFp8Block - 1) / kFp8Block; }
__host__ __device__ inline int fp8_pitch(int cols) { return fp8_blocks(cols) * kFp8Block; }
__host__ __device__ inline int fp8_scale_pitch(int cols) { return (fp8_blocks(cols) + 3) / 4 * 4; }

// One product on 8-bit weights as the kernels take it.
struct Fp8Gemm {
    int experts;
    int64_t max_rows;
    int k;      // columns of the activations as they are
    int pitch;  // bytes of an 8-bit row: k filled up to a multiple of 128
    int n;      // output columns
    int n_pad;  // weight rows of an expert
};
inline Fp8Gemm fp8_gemm(int experts, int64_t max_rows, int k, int n) {
    return Fp8Gemm{experts, max_rows, k, fp8_pitch(k), n, fp8_pitch(n)};
}

// Weights that the memory-side cache does not keep from one pass to the next are fetched with a policy of their own (see
// ffn_weights_stream in ffn.hip).
inline bool fp8_weights_stream(double bytes) { return bytes > (double)(320ull << 20); }

// Which kernels an FFN or a product takes: those for few rows (fp8_thin.hip) need one launch less, and none for the quantising of
// x, but make passes of 16 (FFN) or 32 rows over an expert's weights.  Few rows against tiles, FFN: one token, 64 experts of
// 2048 x 1024 18.9 and 32.1 us, 16 (2 rows an expert) 74.6 and 80.3, 32 (4) 75.8 and 81.5, 48 (6) 86.6 and 81.9, 128 128 and 83;
// 16 tokens, 8 of 4096 x 14336 (4) 227 and 247, 32 (8) 257 and 240, 64 353 and 247; where the weights are few, and the launches
// weigh more: 64 tokens, 8 of 2048 x 1024 (16) 24.0 and 31.0; 32 and 64, 1 of 4096 x 2048 26.8 and 38.1, 48.0 and 41.2.
// Products: 64 of 2048 x 1024, 2 and 4 rows an expert 23.9 and 25.5, 24.2 and 25.6, 16 35.2 and 25.9; 8 of 14336 x 4096, 4 74.1 and 76.9,
// 16 87.9 and 81.0; 1 of 2056 x 5640, 32, 64, 96 rows 7.9 and 10.6, 10.1 and 11.5, 13.9 and 11.7.
// How the rows lie is known on the device only, and the passes over a long expert run one after the other in its own blocks, so the most
// rows that an expert may have are four passes.  Few rows against tiles, dealt evenly, half on one expert, all on one (FFN: on as few as hold
// them): products, 64 of 2048 x 1024, 128 rows 25.9 and 28.3, 43.3 and 39.3, 36.8 and 14.6, 512 26.3 and 29.2, 93.5 and 39.6, 140 and 15.6;
// 60 of 512 x 1280, 120 rows 13.3 and 16.9, 13.4 and 16.7, 14.8 and 12.0, 960 13.7 and 17.1, 54 and 21, 93 and 17; 256 of 512 x 512, 8192 rows
// 19.6 and 22.3, 395 and 34, 769 and 19.5; 8 of 14336 x 4096, 64 rows 72.5 and 74.2, 80 and 80, 32 and 63.  FFN: 16 of 1024 x 1024, 64 tokens
// top-4 18.6 and 28.8, 37.4 and 31.0, 31.7 and 25.4; 128 of 2048 x 768, 64 top-8 111 and 113, 161 and 112, 72 and 36; 256 of 256 x 256, 128 top-8
// 21 and 34, 57 and 41, 43 and 25, 512 top-8 22 and 35, 171 and 52, 158 and 32.  (Over plans whose experts' shares are e^x of normal x, Zipf's or
// one in twenty's, products of 64 to 127 rows take 0.87 of the tiles' time, of 1024 and more 1.31, at worst 4.6.)
constexpr int kFp8MostPasses = 4;
inline bool fp8_few_weights(double bytes) { return bytes <= (double)(64ull << 20); }
inline bool fp8_ffn_is_few_rows(const moe_desc_t& d, const Sizes& s) {
    const bool few = fp8_few_weights(3.0 * d.n_experts * fp8_pitch(d.d_model) * fp8_pitch(d.d_hidden));
    const int64_t most = std::min<int64_t>((int64_t)s.n_blocks * s.cap, d.n_tokens);  // rows of an expert
    return most <= (few ? 32 : 16) || (most <= kFp8MostPasses * 16 && s.max_rows <= (few ? 16ll : 4ll) * d.n_experts);
}
inline bool fp8_gemm_is_few_rows(const Fp8Gemm& g) {
    const bool few = fp8_few_weights((double)g.experts * g.pitch * g.n_pad);
    return g.max_rows <= (few ? 64 : 32) || (g.max_rows <= kFp8MostPasses * 32 && g.max_rows <= (few ? 32ll : 8ll) * g.experts);
}

// Which width a product on high tiles takes, 256 or 128 columns: narrower tiles where the wide ones would leave a quarter of the
// compute units without an item: 8 experts of 14336 columns by 4096 (128 wide items), 8 to 128 rows an expert 110 -> 77, 121 -> 83 us;
// of 64 x 2048 x 1024 (512) they take 4 % more.
inline bool fp8_tiles_are_wide(const Fp8Gemm& g, int cus) {
    const int64_t tiles = g.max_rows / kFfnTileM + std::min<int64_t>(g.max_rows, g.experts);
    return g.n_pad % 256 == 0 && 4 * tiles * (g.n_pad / 256) > 3 * cus;
}

// Rows of a full row tile (1 << the result; columns: column blocks of the product): lower tiles as long as their items still fit one
// round of the compute units and an eighth (the bound counts a partly filled tile of every expert).  Tiles of 64, 128, 256 rows, us, on 256
// compute units: one expert, 203 rows of 2056 x 5640 11.8, 14.4, 17.6, 512 rows 20.0, 15.7, 19.5, 1024 29.5, 26.9, 23.6; the FFN of one expert
// of 4096 x 2048, 512 tokens 45.5, 54.9, 77.1, 2048 95.6, 82.3, 96.0 (its products take different ones: 73.5), 4096 162, 131, 112; 512 tokens
// top-2 on 8 experts of 2048 x 1024 34.1, 39.4, 38.5, 1024 45.9, 42.8, 55.7, 2048 62.2, 56.1, 60.4 (taken: 35.5, 46.6, 60.2); 1500 on 8 of
// 4096 x 4096 247, 202, 168.
inline int fp8_tile_shift(int64_t max_rows, int experts, int columns, int cus) {
    const int64_t partly = std::min<int64_t>(max_rows, experts);
    int shift = 8;
    while (shift > 6 && columns * ((max_rows >> (shift - 1)) + partly) <= cus + cus / 8) --shift;
    return shift;
}

// How many waves share a weight row.  Eight waves fill a compute unit; whole rows keep a wave's ring full for longer, shorter parts
// end sooner.  Products at 4, 2, 1 (256 compute units): one token's 8 experts of 64 x 2048 x 1024 (512 waves with whole rows) FFN 18.6, 19.4, 24.9 us;
// two tokens' (960) 32.7, 27.0, 27.2; four tokens' (2048) 58, 48, 41; 16 tokens', 108, 86, 75; 64 x 4096 x 1408 (5632) 227, 190, 185;
// 8 experts of 14336 columns by 4096 (1024, but long) 73.4, 77.0, 76.4.
inline int fp8_thin_split(int64_t waves, int slabs, int cus) {
    if (waves <= 2 * cus || (waves <= 4 * cus && slabs >= 64)) return 4;
    return waves <= 4 * cus ? 2 : 1;
}

}  // namespace capmoe
