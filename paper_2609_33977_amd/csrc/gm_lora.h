// Sizes and layouts that the host layer and the kernels of the low-rank
// adapters share (host arithmetic only).
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace gm {

constexpr int kLoraTile = 64;       // tokens of one adapter that a block of the products works on
constexpr int kLoraMaxParts = 4;    // projections stacked side by side
constexpr int kLoraSlice = 512;     // contraction length that a block takes at a time: 128 per wave
constexpr int kLoraGradCols = 128;  // columns of a gradient tile
constexpr int32_t kLoraMagic = 0x61d7a3c5;

// Tokens of one adapter whose gradient products one block sums up: the plan
// holds a table for each of these lengths.
constexpr int kLoraGradLens = 4;
constexpr int kLoraGradTokens = 256;  // the shortest; each is twice the last
constexpr int kLoraGradMost = kLoraGradTokens << (kLoraGradLens - 1);

// Most tiles of `tile` tokens that T tokens in m buckets can need.
inline int64_t lora_tiles(int64_t T, int64_t buckets, int64_t tile) {
  const int64_t m = buckets < T ? buckets : T;
  return (T + (tile - 1) * m) / tile;
}

// The plan, in 4-byte words: a header (magic, T, n, tiles, gradient tiles of
// each length); the tile table, tokens of one adapter at a time, those without
// one last (first position in that order, tokens, adapter, 0); 64 tokens for
// every tile (the last one repeated); for each length the gradient tile table (first
// tile, tokens, adapter, only tile of its adapter) and each adapter's first entry in it.
struct LoraPlanLayout {
  size_t tiles, tokens, gtiles[kLoraGradLens], gstart[kLoraGradLens], words;
  int64_t max_tiles, max_gtiles[kLoraGradLens];
};

inline LoraPlanLayout lora_plan_layout(int64_t T, int64_t n) {
  LoraPlanLayout L;
  size_t at = 16;
  auto take = [&](size_t& w, size_t words) {
    w = at;
    at = (at + words + 15) / 16 * 16;
  };
  L.max_tiles = lora_tiles(T, n + 1, kLoraTile);
  take(L.tiles, size_t(L.max_tiles) * 4);
  take(L.tokens, size_t(L.max_tiles) * kLoraTile);
  for (int i = 0; i < kLoraGradLens; ++i) {
    L.max_gtiles[i] = lora_tiles(T, n, kLoraGradTokens << i);
    take(L.gtiles[i], size_t(L.max_gtiles[i]) * 4);
    take(L.gstart[i], size_t(n) + 1);
  }
  L.words = at;
  return L;
}

// Which length the gradients of T tokens take: the longest with enough blocks
// of 128 columns (`col_blocks` for all tokens once) to fill the chip, since every
// tile of an adapter beyond the first leaves partial sums to be written and added.  Gradients (with dX) and the adding, us,
// with tiles of 256 / 512 / 1024 / 2048 tokens: one adapter, 8192 tokens, 4096 and 11008 columns, 64 ranks 131 + 21,
// 114 + 11, 109 + 8, 97 + 5 (taken: 2048); 2048 tokens, 4096 and 3 x 4096 columns, 3 x 16 ranks 27 + 5, 26 + 5, 28 + 5,
// 45 + 5 (512); 1000 tokens of five adapters, 2816 and 2056 columns, 24 ranks 10 + 3, 13 + 4, 14 + 4, 14 + 4 (256).
constexpr int kLoraGradBlocks = 400;
inline int lora_grad_len(int64_t T, int64_t col_blocks) {
  int i = kLoraGradLens - 1;
  while (i > 0 && (T + (kLoraGradTokens << i) - 1) / (kLoraGradTokens << i) * col_blocks < kLoraGradBlocks) --i;
  return i;
}

// Blocks of 16, 32 or 64 ranks.
inline int lora_rank_tiles(int ranks) { return ranks <= 16 ? 1 : ranks <= 32 ? 2 : 4; }

// Blocks that share a tile's contraction over K: two blocks per CU (what fits at once; a
// sixteenth more, since the tiles are the most that there can be), at least two and at most one per slice.  8192
// tokens of 11008 columns, 64 ranks: 51 us with three splits of 128 tiles, 48 with four.  Splits for three blocks per CU
// gave nothing (4099 tokens of 4096 columns, 16 ranks: 9.1 us with two, 10.1 with three).
inline int lora_splits(int64_t tiles, int ranks, int64_t K) {
  const int rt = lora_rank_tiles(ranks);
  const int64_t slices = (K + kLoraSlice - 1) / kLoraSlice, chunks = (ranks + 16 * rt - 1) / (16 * rt);
  int64_t ks = 544 / (tiles * chunks);
  if (ks < 2) ks = 2;
  return int(ks < slices ? ks : slices);
}

// The products with the rank contracted: blocks of 16, 32, 64 or 128 ranks, the columns whose weights are in LDS at a
// time, and how many blocks run at once (LDS: three per CU at 64 ranks, one beyond; there a sixteenth more, since the
// tiles are the most that there can be).
constexpr int lora_up_rank_tiles(int ranks) { return ranks <= 16 ? 1 : ranks <= 32 ? 2 : ranks <= 64 ? 4 : 8; }
constexpr int lora_up_cols(int rank_tiles) { return rank_tiles <= 2 ? 512 : 256; }
constexpr int lora_up_resident(int ranks) { return ranks <= 64 ? 768 : 272; }

inline int64_t lora_up_blocks(const int* widths, int parts, int span, int64_t tiles) {
  int64_t n = 0;
  for (int p = 0; p < parts; ++p) n += (widths[p] + span - 1) / span;
  return n * tiles;
}

// Columns of such a block, 1024 to 256.  Up to 32 ranks, and for dX, narrower ones until there are four blocks per CU to
// hide latency (4099 tokens of 12 adapters, 11008 columns, 16 ranks: 50 us with two, 45 with four), or two where the
// terms that every block stages count for more, in tiles of few tokens (64 tokens of 32 adapters, 15360
// columns: 9.0 us with two, 11.4 with four).  Beyond, where staging costs a block
// about as much as 384 columns, the width whose rounds of blocks cost least: 8192 tokens of one
// adapter, 4096 columns, 64 ranks, one round of 1024 columns 36 us, two of 512 43; 203 tokens of 40 adapters,
// 22016 columns, two rounds of 1024 33, three of 512 29.  At 128 ranks, the whole forward with 256 / 512 / 1024
// columns: 2048 tokens of 4096 columns 30.1, 25.2, 33.1 us (taken: 512); 1024 of 11008 40.1, 38.8, 34.6 (1024).
// Past 128 ranks (dX of stacked parts) the sums of all rounds are in registers, for the columns in LDS.
inline int lora_up_span(const int* widths, int parts, int64_t T, int64_t tiles, int ranks, bool dx) {
  if (ranks > 128) return lora_up_cols(8);
  int span = 1024;
  if (dx || ranks <= 32) {
    const int want = dx || T >= tiles * (kLoraTile / 2) ? 1024 : 512;
    while (span > 256 && lora_up_blocks(widths, parts, span, tiles) < want) span /= 2;
    return span;
  }
  const int64_t at_once = lora_up_resident(ranks);
  auto cost = [&](int s) { return (lora_up_blocks(widths, parts, s, tiles) + at_once - 1) / at_once * (s + 384); };
  for (int s = 512; s >= 256; s /= 2)
    if (cost(s) < cost(span)) span = s;
  return span;
}

}  // namespace gm
