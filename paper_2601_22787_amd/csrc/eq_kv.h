// The 4-bit key/value cache as the kernels see it (layout: include/eq.h), and
// the host checks that its entry points share.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "eq.h"

namespace eq_kv {

constexpr uint32_t kUnit = 32;  // tokens that share a block of value codes
constexpr uint32_t kMaxNodes = EQ_TREE_NODES;  // of a drafted tree
// A launch has fewer than 2^32 threads along x: the most blocks of 256.
constexpr uint32_t kMaxBlocks = (1u << 24) - 1;

// Offsets within a head's part of a page, and the batch, by value for kernels.
struct View {
  uint8_t *pages;
  uint32_t page_bytes;  // (below 2^30: 1024 heads, 4096 tokens of 133 bytes)
  uint32_t head_bytes;
  uint32_t v_off, ks_off, vs_off;  // value codes, key scales, value scales
  uint32_t page_shift;             // log2 page_tokens
  uint32_t n_pages, kv_heads;
  const int32_t *seq_start, *kv_len, *page_table;
  uint32_t n_seqs, max_pages, n_tokens, max_new, max_len;
};

inline bool sizes_ok(uint32_t kv_heads, uint32_t head_dim, uint32_t page_tokens) {
  return kv_heads >= 1 && kv_heads <= 1024 && (head_dim == 64 || head_dim == 128) &&
         page_tokens >= 32 && page_tokens <= 4096 && (page_tokens & (page_tokens - 1)) == 0;
}

inline uint32_t head_bytes(uint32_t head_dim, uint32_t page_tokens) {
  return (page_tokens * (head_dim + head_dim / 32 + 1) + 127) / 128 * 128;
}

inline bool batch_ok(const eq_kv_cache *c, const eq_kv_batch *b) {
  return c && b && sizes_ok(c->kv_heads, c->head_dim, c->page_tokens) && c->pages &&
         (reinterpret_cast<uintptr_t>(c->pages) & 127) == 0 && c->n_pages >= 1 &&
         c->n_pages <= 0x7FFFFFFFu && b->n_seqs <= 65535 && b->max_new <= b->n_tokens &&
         b->n_tokens <= 1u << 30 && b->max_len <= 1u << 30 &&
         b->max_len <= uint64_t(b->max_pages) * c->page_tokens &&
         (b->n_seqs == 0 || (b->seq_start && b->kv_len && b->page_table && b->max_pages >= 1));
}

inline View view(const eq_kv_cache *c, const eq_kv_batch *b) {
  View w{};
  const uint32_t n = c->page_tokens, d = c->head_dim;
  w.pages = c->pages;
  w.head_bytes = head_bytes(d, n);
  w.page_bytes = w.head_bytes * c->kv_heads;
  w.v_off = n * d / 2;
  w.ks_off = n * d;
  w.vs_off = n * d + n * (d / 32);
  while ((1u << w.page_shift) < n) ++w.page_shift;
  w.n_pages = c->n_pages;
  w.kv_heads = c->kv_heads;
  w.seq_start = b->seq_start;
  w.kv_len = b->kv_len;
  w.page_table = b->page_table;
  w.n_seqs = b->n_seqs;
  w.max_pages = b->max_pages;
  w.n_tokens = b->n_tokens;
  w.max_new = b->max_new;
  w.max_len = b->max_len;
  return w;
}

// A sequence's rows [row, row + count), of which row i is at position base + i,
// and its tokens; count and len are cut to the host's bounds.
struct Seq {
  int32_t row, count, base, len;
};

__device__ inline Seq sequence(const View &w, uint32_t s) {
  const int32_t row = w.seq_start[s], end = w.seq_start[s + 1], len = w.kv_len[s];
  Seq q{row, 0, 0, 0};
  q.len = len < 0 ? 0 : min(len, int32_t(w.max_len));
  if (row < 0 || end <= row || uint32_t(row) >= w.n_tokens || len < 0) return q;
  q.base = len - (end - row);
  q.count = min(min(end - row, int32_t(w.max_new)), int32_t(w.n_tokens) - row);
  return q;
}

// The page of position p >= 0 of sequence s (p below max_len), or -1.
__device__ inline int32_t page_of(const View &w, uint32_t s, uint32_t p) {
  const int32_t page = w.page_table[size_t(s) * w.max_pages + (p >> w.page_shift)];
  return uint32_t(page) < w.n_pages ? page : -1;
}

}  // namespace eq_kv
