// Host rules that choose how attention over the 4-bit cache is launched.  No
// device code, so that they can be checked without a GPU.
#pragma once
#include <algorithm>
#include <cstdint>

namespace eq_attn {

// Few query columns (attn_kernel): tokens a wavefront takes at a time, and the
// columns of a block.  Many (prompt_kernel): tokens and columns of a block.
constexpr uint32_t kTile = 128, kCols = 16;
constexpr uint32_t kPromptTile = 64, kPromptCols = 128;

// How a call is launched.
//
// Which kernel: prompt_kernel's tiles of 128 columns pay where they fill the card
// by themselves, a block for each of 256 compute units, or where a long cache can
// be cut into chunks; attn_kernel spreads fewer columns better.  Columns of a
// key/value head, sequences x heads, cached tokens: us of attn_kernel / of
// prompt_kernel
//   64, 8 x 32, 1024: 26.8 / 27.7    128, 8 x 32, 1024: 46.0 / 31.2
//   384, 8 x 8, 1024: 27.7 / 28.8    512, 8 x 8, 1024: 35.2 / 29.8
//   1024, 1 x 8, 2048: 16.5 / 36.9   1024, 1 x 8, 8192: 68 / 58
//   512, 1 x 8, 8192: 39.2 / 38.0    2048, 1 x 8, 32768: 418 / 301
//
// Chunks: the token tiles are cut so that the blocks fill the card (prompt_kernel:
// twice over), none shorter than four tiles (attn_kernel: one for each wavefront)
// and, where there is less than that to fill it with, none longer than 4096 tokens
// (prompt_kernel: 2048): a ragged batch's longest sequence then spreads over the
// card too.  attn_kernel filling the card twice: 8 sequences x 8 heads of 4096
// tokens 13.9 us, once 13.4.  Short caches are one chunk in attn_kernel: a further
// tile for a wavefront is 1.1 us, the second launch 3.7 (2 x 8 and 16 x 8, 2048
// tokens: 9.0 and 10.6 us in one chunk, 9.4 and 14.6 in more); up to 4096 tokens
// where that fills half the card (16 x 8, 4096 tokens: 16.2 / 18.9, 3000 tokens:
// 13.2 / 16.6; 8 x 8, 4096 tokens: 15.5 / 13.4).  prompt_kernel's partial sums are
// larger (4096 columns, 1 x 8, 8192 tokens: 165 us in one chunk, 187 in two), so
// it has chunks only where the columns do not fill the card.
struct Plan {
  bool prompt;
  uint32_t cols, tile, q_tiles, chunks, chunk_tiles;
};

constexpr uint32_t kFewCols = 64, kFillBlocks = 256, kLongTokens = 8192;
// attn_kernel: tiles of one chunk, and with half the card's blocks or more
constexpr uint32_t kWholeTiles = 16, kWholeFilled = 32;

inline Plan plan_attn(uint32_t n_seqs, uint32_t kv_heads, uint32_t group, uint32_t max_new,
                      uint32_t max_len, uint32_t window) {
  Plan p;
  const uint64_t cols = uint64_t(max_new) * group;
  const uint64_t prompts = uint64_t(n_seqs) * kv_heads * ((cols + kPromptCols - 1) / kPromptCols);
  p.prompt = cols > kFewCols && (prompts >= kFillBlocks || max_len >= kLongTokens);
  p.cols = p.prompt ? kPromptCols : kCols;
  p.tile = p.prompt ? kPromptTile : kTile;
  p.q_tiles = uint32_t((cols + p.cols - 1) / p.cols);
  const uint64_t work = uint64_t(n_seqs) * kv_heads * p.q_tiles;
  const uint32_t tiles = (max_len + p.tile - 1) / p.tile;
  const uint32_t whole_tiles = 2 * work >= kFillBlocks ? kWholeFilled : kWholeTiles;
  const bool whole = p.prompt ? work >= kFillBlocks : tiles <= whole_tiles;
  const uint64_t fill = p.prompt ? 2 * kFillBlocks : kFillBlocks;
  const uint64_t want = whole ? 1 : std::max<uint64_t>(1, (fill + work - 1) / work);
  auto round4 = [](uint64_t v) { return uint32_t(std::max<uint64_t>((v + 3) / 4 * 4, 4)); };
  uint32_t ct = round4((tiles + want - 1) / want);
  if (!whole && work < 2048) ct = std::min(ct, (p.prompt ? 2048 : 4096) / p.tile);
  p.chunks = std::max((tiles + ct - 1) / ct, 1u);
  ct = round4((tiles + p.chunks - 1) / p.chunks);  // chunks of one length
  // a window leaves fewer tiles (a query's window and the others' of its
  // sequence), in at most as many chunks: the workspace does not depend on it
  uint32_t seen = tiles;
  if (window)
    seen = uint32_t(std::min<uint64_t>(tiles, (uint64_t(window) + max_new + p.tile - 2) / p.tile + 1));
  if (seen < tiles) {
    ct = round4((seen + p.chunks - 1) / p.chunks);
    if (!p.prompt && seen <= whole_tiles) ct = round4(seen);
    p.chunks = std::max((seen + ct - 1) / ct, 1u);
  }
  p.chunk_tiles = ct;
  return p;
}

// Up to 8 columns take both terms in one product (attn_kernel's PAIR).
inline bool pair_columns(uint32_t max_new, uint32_t group) {
  return uint64_t(max_new) * group <= kCols / 2;
}

// Codes that are read once in all, and more of them than the memory-side cache
// keeps, pass the caches as streams: 303 MB of 8 heads 74 -> 70 us.  Fewer stay in
// it between calls (16 MiB: 7.5 us, as streams 8.1), and query tiles share what the
// first of them has read.  The limit is three quarters of its 256 MiB: the call's
// other data pass through it too.  max_len and the window bound what is read.
inline bool stream_cache(const Plan &p, uint32_t n_seqs, uint32_t kv_heads, uint32_t head_dim,
                         uint32_t max_new, uint32_t max_len, uint32_t window) {
  const uint64_t tokens =
      window ? std::min<uint64_t>(max_len, uint64_t(window) + max_new - 1) : max_len;
  return p.q_tiles == 1 && n_seqs * tokens * kv_heads * (head_dim + head_dim / 32 + 1) >
                               uint64_t(192) << 20;
}

}  // namespace eq_attn
