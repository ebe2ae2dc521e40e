// Attention over the 4-bit key/value cache (declared in include/eq.h).
//
// For one key/value head the queries that read it (its query heads at every
// new token of a sequence) are columns, cached tokens are rows:
//   S = K q^T,  P = exp2(c S - m),  O = V^T (w P),  out = O / sum P
// with c = scale log2 e, m the running maximum of a column and w_t the scale of
// token t's value.  Both products run on the scaled matrix instructions, which
// take E2M1 codes with one power-of-two scale for 32 of them as they lie in the
// cache, so neither keys nor values are ever decoded.  The other operand has to
// be 8 bits wide: q and w P enter as the sum of two E4M3 numbers, x = h + l with
// h = e4m3(x) and l = e4m3(x - h), 4 significant bits each, at one scale for a
// query's 32 channels and for w P of a column's 128 tokens.  That holds all of a
// BF16 query that is at least 2^-14 of the largest, and w P to 8 significant bits
// from there on; what is smaller is held to 2^-22 of the largest.  (The lower term's
// step is 2^-14 where the largest is 2^7 to 2^8.)
#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

#include "eq.h"
#include "eq_attn_rules.h"
#include "eq_device.h"
#include "eq_kv.h"

namespace {

using namespace eq_attn;
using namespace eq_kv;

typedef int int4v __attribute__((ext_vector_type(4)));
typedef int int8v __attribute__((ext_vector_type(8)));
typedef short short2v __attribute__((ext_vector_type(2)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

constexpr uint32_t kWaves = 4;
constexpr int kUnitScale = 127;  // scale byte of 1

struct AttnArgs {
  View w;
  const uint16_t *q;
  uint64_t q_stride;
  uint16_t *out;
  float *part;       // [n_seqs][kv_heads][q_tiles][chunks][columns][D] sums of a chunk
  float2 *stat;      // the same without D: maximum and sum of P
  uint32_t group;    // query heads of a key/value head
  uint32_t window;
  uint32_t q_tiles, chunks, chunk_tiles;
  float c;           // scale log2 e
  const uint32_t *mask;      // trees: [n_tokens][mask_words], bit j: new token j is seen
  const int32_t *positions;  // trees with a window: [n_tokens]
  uint32_t mask_words;
  uint32_t *even;            // trees: prompt_kernel's chunk_tiles for join_kernel, or null
};

// Columns [col0, col0 + COLS) of a sequence, and the cached tokens they see.
struct Span {
  uint32_t cols;          // columns of the sequence
  uint32_t first, last;   // tiles [first, last) of TILE tokens
  uint32_t chunks;
  uint32_t seen;          // tokens [0, seen) hold all that is seen
  int32_t hi_min, lo_max; // tokens in [lo_max, hi_min) are seen by every column
};

__device__ inline int32_t end_of(const Seq &q, int32_t pos) { return max(min(pos + 1, q.len), 0); }
__device__ inline int32_t start_of(uint32_t window, int32_t pos) {
  return window && pos >= 0 && uint32_t(pos) >= window ? pos + 1 - int32_t(window) : 0;
}

// TREE: all columns see the tokens before the new ones (what a window hides of them
// and lanes without a node are the kernels' own), and new ones by their masks, those of
// the rows that count: what is behind them would be more than the host has chunks for.
struct Tiles {
  uint32_t seen, first, last;
};
template <uint32_t TILE>
__device__ inline Tiles tree_tiles(uint32_t window, const Seq &q) {
  Tiles t;
  t.seen = uint32_t(min(max(q.base + q.count, 0), q.len));
  t.first = uint32_t(start_of(window, max(q.base, 0))) / TILE;
  t.last = max((t.seen + TILE - 1) / TILE, t.first);
  return t;
}

template <uint32_t COLS, uint32_t TILE, bool TREE>
__device__ inline Span span_of(const AttnArgs &a, const Seq &q, uint32_t col0) {
  Span p{};
  p.cols = uint32_t(q.count) * a.group;
  if (col0 >= p.cols) return p;
  if constexpr (TREE) {
    const Tiles t = tree_tiles<TILE>(a.window, q);
    p.hi_min = min(max(q.base, 0), q.len);
    p.seen = t.seen, p.first = t.first, p.last = t.last;
    p.chunks = min((p.last - p.first + a.chunk_tiles - 1) / a.chunk_tiles, a.chunks);
    return p;
  }
  const int32_t pos0 = q.base + int32_t(col0 / a.group);
  const int32_t pos1 = q.base + int32_t((min(col0 + COLS, p.cols) - 1) / a.group);
  p.hi_min = end_of(q, pos0);
  p.lo_max = start_of(a.window, pos1);
  p.seen = uint32_t(end_of(q, pos1));
  p.first = uint32_t(start_of(a.window, pos0)) / TILE;
  p.last = max((p.seen + TILE - 1) / TILE, p.first);
  p.chunks = min((p.last - p.first + a.chunk_tiles - 1) / a.chunk_tiles, a.chunks);
  return p;
}

// A tree's column: the cached tokens [lo, hi) that it sees, and its bits of new ones.
struct Node {
  const uint32_t *mask;  // readable for every lane
  int32_t lo, hi, base;
  bool alive;            // a node, which sees itself at least
};

// words: the column's mask (what a narrower one has behind it, its last word again).
constexpr int kMaskWords = kMaxNodes / 32;
__device__ inline Node node_of(const AttnArgs &a, const Seq &q, uint32_t token, bool real,
                               uint32_t (&words)[kMaskWords]) {
  const bool on = real && q.base + int32_t(token) >= 0;
  const uint64_t row = on ? uint64_t(q.row) + token : 0;
  Node n{a.mask + row * a.mask_words, 0, 0, q.base, false};
  int32_t pos = 0;
  if (a.window) pos = a.positions[row];
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < kMaskWords; ++i) {  // (one wait for all)
    words[i] = n.mask[min(uint32_t(i), a.mask_words - 1)];
    any |= words[i];
  }
  if (!on || !any) return n;
  n.alive = true;
  n.hi = min(max(q.base, 0), q.len);
  if (a.window) n.lo = min(start_of(a.window, max(pos, max(q.base, 0))), n.hi);
  return n;
}

// Word i of a column's mask, 0 outside it.
__device__ inline uint32_t mask_word(const AttnArgs &a, const uint32_t *mask, int32_t i) {
  const uint32_t w = mask[min(max(i, 0), int32_t(a.mask_words) - 1)];
  return uint32_t(i) < a.mask_words ? w : 0u;
}

// The largest x of a wavefront.
__device__ inline int32_t wave_max(int32_t x) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) x = max(x, __shfl_xor(x, d));
  return x;
}

// v of the lane that CTRL names, 0 where there is none or the row is not in ROWS.
template <int CTRL, int ROWS, typename T>
__device__ inline T from_lane(T v) {
  return __builtin_bit_cast(
      T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xF, true));
}
// Sums of the lanes up to each: within rows of 16, then from row to row.
template <typename T>
__device__ inline T wave_scan(T x) {
  x += from_lane<0x111, 0xF>(x);
  x += from_lane<0x112, 0xF>(x);
  x += from_lane<0x114, 0xF>(x);
  x += from_lane<0x118, 0xF>(x);
  x += from_lane<0x142, 0xA>(x);  // row_bcast:15
  x += from_lane<0x143, 0xC>(x);  // row_bcast:31
  return x;
}
template <typename T>
__device__ inline T wave_sum(T x) {
  return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, wave_scan(x)), 63));
}

// What block `number` of a head does for a batch of trees, up to 64 of them: the host
// knows no lengths, so chunks of one length are set here that make about as many blocks
// as run at once, and these are numbered without gaps (blocks go round the shader
// engines by their numbers: with gaps some got twice the work of others).  Two sequences
// of 32768 tokens and 64 nodes, 64 heads on 8: 159 -> 154 us; three of 25529 to 32768
// tokens and 19 to 64 nodes 190 -> 168.  A sequence for a lane.
struct Share {
  uint32_t seq, qt, chunk, chunk_tiles;
  bool any;
};

__device__ inline Share even_share(const AttnArgs &a, uint32_t number) {
  const View &w = a.w;
  const uint32_t lane = threadIdx.x & 63;
  uint32_t tiles = 0, q_tiles = 0;
  if (lane < w.n_seqs) {
    const Seq q = sequence(w, lane);
    const Tiles t = tree_tiles<kPromptTile>(a.window, q);
    tiles = t.last - t.first;
    q_tiles = (uint32_t(q.count) * a.group + kPromptCols - 1) / kPromptCols;
  }
  const uint32_t run = head_blocks(w.kv_heads);
  // (a product may pass 32 bits; a chunk of 2^24 tiles is any sequence whole)
  const float even = ceilf(wave_sum(float(q_tiles) * float(tiles)) / float(run));
  uint32_t ct = max(a.chunk_tiles, uint32_t(fminf(even, 0x1p24f)));
  // (as span_of counts them)
  auto blocks = [&]() { return max(min((tiles + ct - 1) / ct, a.chunks), 1u) * q_tiles; };
  for (int i = 0; i < 24 && wave_sum(blocks()) > run; ++i) ct += (ct + 31) / 32;
  const uint32_t mine = blocks(), end = wave_scan(mine);
  const uint64_t m = __ballot(number < end);
  Share r{0, 0, 0, ct, m != 0};
  if (!m) return r;
  r.seq = uint32_t(__ffsll((unsigned long long)m)) - 1;
  const uint32_t at = number - uint32_t(__builtin_amdgcn_readlane(int(end - mine), int(r.seq)));
  const uint32_t each = uint32_t(__builtin_amdgcn_readlane(int(mine), int(r.seq)));
  const uint32_t chunks = each / uint32_t(__builtin_amdgcn_readlane(int(q_tiles), int(r.seq)));
  r.chunk = at % chunks, r.qt = at / chunks;
  return r;
}

// x / scale as two E4M3 terms, of four values: h at `scale`, l at scale / 32 (what h
// leaves of magnitudes below 256 is at most 8, 256 of its units; E4M3 ends at 448).
__device__ inline void split4(const float *x, float scale, int &h, int &l) {
  int a0, b0;  // each conversion fills one half of a register, whatever it held
  asm("" : "=v"(a0));
  asm("" : "=v"(b0));
  short2v a = __builtin_bit_cast(short2v, a0), b = __builtin_bit_cast(short2v, b0);
  a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(a, x[0], x[1], scale, false);
  a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(a, x[2], x[3], scale, true);
  h = __builtin_bit_cast(int, a);
  const float2v u = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(h, scale, false);
  const float2v v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(h, scale, true);
  const float s = scale * 0.03125f;
  b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(b, x[0] - u[0], x[1] - u[1], s, false);
  b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(b, x[2] - v[0], x[3] - v[1], s, true);
  l = __builtin_bit_cast(int, b);
}

// Scale byte that brings magnitudes of the exponent of `top` to [128, 256);
// 255 for an infinity or NaN.  Its lower term's byte is 5 less.
__device__ inline int top_byte(uint32_t top) {
  const int e = int(top >> 23);
  return e == 255 ? 255 : max(e - 7, 8);
}
__device__ inline int low_byte(int b) { return b == 255 ? 255 : b - 5; }
__device__ inline float byte_value(int b) { return __uint_as_float(uint32_t(b) << 23); }

// 2^(byte E of bytes - 127), by a shift that takes the byte itself: the compiler has an
// "and" besides for three of the four, 24 instructions of attn_kernel's tile.
template <int E>
__device__ inline float byte_scale(uint32_t bytes) {
  uint32_t x;
  const uint32_t shift = 23;
#define EQ_BYTE(n) \
  asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_" n \
      : "=v"(x) : "v"(shift), "v"(bytes))
  if constexpr (E == 0) EQ_BYTE("0");
  if constexpr (E == 1) EQ_BYTE("1");
  if constexpr (E == 2) EQ_BYTE("2");
  if constexpr (E == 3) EQ_BYTE("3");
#undef EQ_BYTE
  return __uint_as_float(x);
}

__device__ inline float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// The query columns as the second operand of the key product.  Lane (col, g)
// holds channels 16 g .. of the first half of the operand's 128 steps and 16 g ..
// of the second, and lane group b the scale of steps 32 b ..  At D = 128 the
// steps are the channels, and the two terms are two operands; at D = 64 the
// halves are the two terms, met by the same keys twice.
template <int D>
struct Query {
  int8v h, l;
  int hs, ls;
  // a lane's channels of `row` (zeros where that is null)
  __device__ inline void read(const uint16_t *row, uint32_t g, uint32_t (&raw)[D / 8]) {
#pragma unroll
    for (int i = 0; i < D / 8; ++i) raw[i] = 0;
    if (!row) return;
#pragma unroll
    for (int i = 0; i < D / 8; i += 4)
      *reinterpret_cast<uint4 *>(raw + i) =
          *reinterpret_cast<const uint4 *>(row + i / 8 * 64 + 16 * g + i % 8 * 2);
  }
  __device__ inline void split(const uint32_t (&raw)[D / 8], uint32_t col, uint32_t g) {
    float x[D / 4];
    int byte[D / 64];
#pragma unroll
    for (int k = 0; k < D / 64; ++k) {
      uint32_t top = 0;
#pragma unroll
      for (int i = 8 * k; i < 8 * k + 8; ++i) {
        x[2 * i] = __uint_as_float(raw[i] << 16);
        x[2 * i + 1] = __uint_as_float(raw[i] & 0xFFFF0000u);
        top = max(top, max(raw[i] << 16 & 0x7FFFFFFFu, raw[i] & 0x7FFF0000u));
      }
      byte[k] = top_byte(max(top, uint32_t(__shfl_xor(int(top), 16))));
    }
    const int from_a = __shfl(byte[0], int(32 * (g & 1) + col));
    if constexpr (D == 128) {
      const int from_b = __shfl(byte[1], int(32 * (g & 1) + col));
      hs = g < 2 ? from_a : from_b;
      ls = low_byte(hs);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        int u = 0, v = 0;
        split4(x + 4 * i, byte_value(byte[i / 4]), u, v);
        h[i] = u;
        l[i] = v;
      }
    } else {
      hs = g < 2 ? from_a : low_byte(from_a);
      ls = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        int u = 0, v = 0;
        split4(x + 4 * i, byte_value(byte[0]), u, v);
        h[i] = u;
        h[4 + i] = v;
      }
    }
  }
};

__device__ inline int8v widen(int4v v) { return int8v{v[0], v[1], v[2], v[3], 0, 0, 0, 0}; }

// Codes 2 I and 2 I + 1 of a dword as BF16.
template <int I>
__device__ inline uint32_t code_pair(uint32_t codes) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, 1.0f, I));
}

// acc + codes x terms: 32 x 32 over 64 steps, the codes' scales in byte BYTE of as.
template <int BYTE>
__device__ inline floatx16 mul32(int8v codes, int8v terms, floatx16 acc, int as, int bs) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(codes, terms, acc, 4, 0, BYTE, as, 0, bs);
}

// acc + codes x terms: 16 x 16 over 128 steps, the codes' scales in byte BYTE of as.
template <int BYTE>
__device__ inline floatx4 mul16(int8v codes, int8v terms, floatx4 acc, int as, int bs) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(codes, terms, acc, 4, 0, BYTE, as, 0, bs);
}

// All ones where bit i of m is set, else 0.
__device__ inline uint32_t bit_mask(uint32_t m, int i) { return uint32_t(int32_t(m << (31 - i)) >> 31); }

// Bits 0 to n - 1.
__device__ inline uint32_t bits_below(int32_t n) { return n >= 32 ? ~0u : (1u << max(n, 0)) - 1; }

// x of the lane 8 columns on (of 16).
__device__ inline float other_half(float x) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x128, 0xF, 0xF, true));
}

// The largest x of the lanes (col, g) of a column; PAIR: and of those 8 columns on.
template <bool PAIR>
__device__ inline float column_max(float x) {
  if constexpr (PAIR) x = fmaxf(x, other_half(x));
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}

// 32 codes; STREAM: which nothing reads again before the caches are full of others.
template <bool STREAM>
__device__ inline int4v load_codes(const uint8_t *p) {
  const int4v *const v = reinterpret_cast<const int4v *>(p);
  return STREAM ? __builtin_nontemporal_load(v) : *v;
}

// One block: kCols query columns of a key/value head against a chunk of token
// tiles, dealt to its 4 wavefronts in turn; each keeps its own maximum, sum and
// O, joined through LDS at the end.
//
// Layout.  The product of 16 tokens leaves lane (col, g) with rows 4 g + r, r =
// 0..3, of its column; the second product wants w P in lane (col, g) for steps
// 16 g .. + 15 and 64 + 16 g .. + 15.  Which token a row is, is free: row 4 g +
// r of product i (0..7) is token 64 (i / 4) + 16 g + 4 (i % 4) + r of the tile.
// Then a lane's 32 scores are the 32 tokens of its steps in order, and P passes
// from the first product to the second without leaving the lane.  V lies along
// the tokens in the cache, 32 to a 16-byte row, as the second product takes it.
//
// PAIR: up to 8 columns.  The other 8 of a product then take the second terms: of
// the queries (the scores of columns c and c + 8 add up to column c's; at D = 64
// they are the same queries again, one product having both terms already), and of
// w P (columns c and c + 8 of O add up at the end).  Half the products, and each
// of the two lanes has the softmax of 16 of the 32 tokens (284 000 tokens: 64.2 ->
// 61.9 us; 512 tokens 5.75 -> 5.6).
//
// Long caches are bound by memory: one token of 14 sequences with 284 000 cached
// ones, 64 query heads on 8, 303 MB in 62 us, 4.9 TB/s (a 1 GiB device copy:
// 5.07); 3 wavefronts a SIMD by force spilled and took 82 us.  Short caches are
// bound by the chain of one tile (page number, codes, two products with the
// softmax between): 512 tokens of 32 heads 5.6 us, 8 x 4096 tokens 13.3 with the
// join.
//
// TREE: a column's new tokens are its mask's, 16 bits of it for 16 tokens in a row.
// Here 16 columns see a tile of 128 tokens, 460 vector instructions: eight trees of 16
// nodes, 64 heads on 8, 4096 tokens in 26 us.  No unit is full (vector 0.4, matrix 0.2 of
// the launch): it is the latency of a tile's chain with 5 wavefronts a compute unit, which
// wait for issue in a quarter of their cycles; fewer instructions shorten the chain (by 80
// of 540: 28.8 -> 27.3).  A form of 32 columns a wavefront, with half the loads, took 29
// to 32.
template <int D, bool ONE, bool STREAM, bool PAIR, bool TREE>
__global__ __launch_bounds__(256, 2) void attn_kernel(AttnArgs a) {
  constexpr int ND = D / 16;
  constexpr uint32_t kStride = D + 4;  // floats a column in LDS
  __shared__ __attribute__((aligned(16))) float lds_o[kWaves * kCols * kStride];
  __shared__ float2 lds_s[kWaves][kCols];
  const View &w = a.w;
  const uint32_t s = blockIdx.y;
  // heads first: the blocks that run together then read whole pages, not a head's
  // part of pages all over the pool (284 000 tokens of 8 heads: 69 -> 62 us)
  const uint32_t h = blockIdx.x % w.kv_heads, rest = blockIdx.x / w.kv_heads;
  const uint32_t chunk = rest % a.chunks, qt = rest / a.chunks;
  const uint32_t col0 = qt * kCols;
  const uint32_t lane = threadIdx.x & 63, wave = eq_dev::uniform(threadIdx.x >> 6);
  const uint32_t col = lane & 15, g = lane >> 4;
  const Seq q = sequence(w, s);
  const Span sp = span_of<kCols, kTile, TREE>(a, q, col0);

  // Page numbers of a tile's four 32-token units (one page when it holds them
  // all), by scalar loads.  The table is read up to its width, not up to the
  // sequence's length, so that the first ones need not wait for that; what they
  // name beyond it is masked.
  const int32_t *const table = w.page_table + size_t(s) * w.max_pages;
  const uint32_t page_mask = (1u << w.page_shift) - 1;
  const uint8_t *const base = w.pages + uint64_t(h) * w.head_bytes;
  struct Ids {
    uint32_t u[ONE ? 1 : 4];
  };
  auto load_ids = [&](uint32_t tile) {
    Ids d;
#pragma unroll
    for (uint32_t u = 0; u < (ONE ? 1 : 4); ++u)
      d.u[u] = eq_dev::as_const(table)[min((tile * 4 + u) * kUnit >> w.page_shift, w.max_pages - 1)];
    return d;
  };
  uint32_t first = 0;
  if (a.window) first = sp.first;
  uint32_t t = first + chunk * a.chunk_tiles + wave;
  Ids ids = load_ids(t);
  if (col0 >= sp.cols || chunk >= max(sp.chunks, 1u)) return;
  const uint32_t t_end = min(sp.first + (chunk + 1) * a.chunk_tiles, sp.last);
  // the wavefront's last tile, which is loaded again where there is no next one
  // (loads under a condition would be waited for where the branches meet)
  const uint32_t t_last = t < t_end ? t + (t_end - 1 - t) / kWaves * kWaves : t;

  // this lane's column
  const bool upper = PAIR && col >= 8;
  const uint32_t index = col0 + (PAIR ? col & 7 : col);
  const bool real = index < sp.cols;
  const uint32_t token = index / a.group;
  const int32_t pos = q.base + int32_t(token);
  int32_t hi = real ? end_of(q, pos) : 0, lo = real ? start_of(a.window, pos) : 0;
  int32_t hi_min = sp.hi_min, lo_max = sp.lo_max;
  Node node{};
  if constexpr (TREE) {
    uint32_t words[kMaskWords];
    node = node_of(a, q, token, real, words);
    hi = node.hi, lo = node.lo;
    if (__any(real && !node.alive)) hi_min = 0;
    if (a.window) lo_max = wave_max(lo);
  }

  // a lane's parts of a tile: keys of units gk/2 and 2 + gk/2, values of unit g,
  // value scales of units g/2 and 2 + g/2
  const uint32_t gk = col >> 2, r = lane & 3, kg = D == 128 ? g : g & 1;
  auto part_of = [&](const Ids &d, uint32_t unit) {
    uint32_t id = d.u[0];
    if constexpr (!ONE) {
      const uint32_t low = unit & 1 ? d.u[1] : d.u[0], high = unit & 1 ? d.u[3] : d.u[2];
      id = unit & 2 ? high : low;
    }
    return base + uint64_t(id < w.n_pages ? id : 0) * w.page_bytes;
  };
  auto slot_of = [&](uint32_t tile, uint32_t unit) { return (tile * 4 + unit) * kUnit & page_mask; };
  int4v kreg[8], vreg[ND];
  uint4 va, vb;  // (PAIR: va is of the lane's own 16 tokens)
  int ksa, ksb;
  auto load_k = [&](uint32_t tile, const Ids &d) {
    const uint8_t *const pa = part_of(d, gk >> 1), *const pb = part_of(d, 2 + (gk >> 1));
    const uint32_t a0 = slot_of(tile, gk >> 1) + 16 * (gk & 1);
    const uint32_t b0 = slot_of(tile, 2 + (gk >> 1)) + 16 * (gk & 1);
    const uint32_t at = r * (D / 2) + 16 * kg, ks_at = w.ks_off + (r * (D / 32) + kg) * 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      kreg[i] = load_codes<STREAM>(pa + (a0 * (D / 2) + at + i * 2 * D));
      kreg[4 + i] = load_codes<STREAM>(pb + (b0 * (D / 2) + at + i * 2 * D));
    }
    ksa = *reinterpret_cast<const int *>(pa + (ks_at + a0 * (D / 32)));
    ksb = *reinterpret_cast<const int *>(pb + (ks_at + b0 * (D / 32)));
  };
  auto load_vs = [&](uint32_t tile, const Ids &d) {
    const uint32_t at = w.vs_off + 16 * (g & 1), unit = (g >> 1) + (upper ? 2 : 0);
    va = *reinterpret_cast<const uint4 *>(part_of(d, unit) + (at + slot_of(tile, unit)));
    if constexpr (!PAIR)
      vb = *reinterpret_cast<const uint4 *>(part_of(d, 2 + unit) + (at + slot_of(tile, 2 + unit)));
  };
  auto load_v = [&](uint32_t tile, const Ids &d) {
    const uint8_t *const p = part_of(d, g) + (w.v_off + slot_of(tile, g) * (D / 2) + col * 16);
#pragma unroll
    for (int m = 0; m < ND; ++m) vreg[m] = load_codes<STREAM>(p + m * 256);
  };

  // TREE: new tokens lie in three tiles at most, so in one of this wavefront's; the
  // mask words of a lane's tokens there
  uint32_t ma[2] = {}, mb[2] = {}, new_tile = 0;
  if constexpr (TREE) {
    static_assert((eq_kv::kMaxNodes + kTile - 2) / kTile + 1 <= kWaves);
    const uint32_t tb = uint32_t(max(q.base, 0)) / kTile;
    new_tile = tb + ((t - tb) & (kWaves - 1));
    const int32_t i = (int32_t(new_tile * kTile + 16 * g) + (upper ? 64 : 0) - node.base) >> 5;
    ma[0] = mask_word(a, node.mask, i), ma[1] = mask_word(a, node.mask, i + 1);
    if constexpr (!PAIR)
      mb[0] = mask_word(a, node.mask, i + 2), mb[1] = mask_word(a, node.mask, i + 3);
  }

  float m_run = -INFINITY, m_use = 0.0f, l_run = 0.0f;
  int8v ph{}, pq{};  // w P of a tile, as two terms (PAIR: ph is the lane's term)
  floatx4 o[ND];
#pragma unroll
  for (int m = 0; m < ND; ++m) o[m] = floatx4{0, 0, 0, 0};

  if (t < t_end) {
    Query<D> query;
    const uint16_t *const row =
        real ? a.q + uint64_t(q.row + token) * a.q_stride + uint64_t(h * a.group + index % a.group) * D
             : nullptr;
    uint32_t raw[D / 8];
    query.read(row, g, raw);
    load_k(t, ids);
    load_vs(t, ids);
    load_v(t, ids);
    Ids next = load_ids(min(t + kWaves, t_last));
    query.split(raw, col, g);
    if (PAIR && D == 128 && upper) query.h = query.l, query.hs = query.ls;
    for (; t < t_end; t += kWaves) {
      const uint32_t t_next = min(t + kWaves, t_last);
      floatx4 sc[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int8v k8 = widen(kreg[i]);
        const int ks = i < 4 ? ksa : ksb;
        sc[i] = floatx4{0, 0, 0, 0};
        auto mul = [&](int8v b, int bs) {
          switch (i & 3) {
            case 0: sc[i] = mul16<0>(k8, b, sc[i], ks, bs); break;
            case 1: sc[i] = mul16<1>(k8, b, sc[i], ks, bs); break;
            case 2: sc[i] = mul16<2>(k8, b, sc[i], ks, bs); break;
            default: sc[i] = mul16<3>(k8, b, sc[i], ks, bs); break;
          }
        };
        mul(query.h, query.hs);
        if constexpr (D == 128 && !PAIR) mul(query.l, query.ls);
      }
      load_k(t_next, next);
      // masks, where some column does not see the whole tile
      const int32_t at = int32_t(t * kTile);
      uint32_t gone = 0;  // bit u: unit u's page is not there
#pragma unroll
      for (uint32_t u = 0; u < (ONE ? 1 : 4); ++u) gone |= uint32_t(ids.u[u] >= w.n_pages) << u;
      if (ONE && gone) gone = 15;
      const bool masked = at + int32_t(kTile) > hi_min || at < lo_max || gone;
      // a lane's scores: all 32 of its tokens, or, with PAIR, 16 of them and the
      // sum of both terms, whose other half the lane 8 columns on holds
      constexpr int NS = PAIR ? 16 : 32;
      float x[NS];
      if constexpr (PAIR) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float low = sc[i / 4][i % 4], high = sc[4 + i / 4][i % 4];
          x[i] = upper ? high : low;
          if constexpr (D == 128) x[i] += other_half(upper ? low : high);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) x[i] = sc[i / 4][i % 4];
      }
      uint32_t visible = ~0u;  // bit i: this lane's column sees token i of them
      if (masked) {
        auto bits = [&](uint32_t unit, int32_t from, const uint32_t (&m)[2]) {  // of 16 tokens
          const int32_t u = min(max(lo - from, 0), 16), v = min(max(hi - from, u), 16);
          uint32_t b = (1u << v) - (1u << u);
          if constexpr (TREE) {
            const int32_t there = min(max(int32_t(sp.seen) - from, 0), 16);
            const uint32_t own = __builtin_amdgcn_alignbit(m[1], m[0], uint32_t(from - node.base) & 31);
            b |= node.alive && t == new_tile ? own & ((1u << there) - 1) : 0u;
          }
          return gone >> unit & 1 ? 0u : b;
        };
        const uint32_t unit = (g >> 1) + (upper ? 2 : 0);
        const int32_t from = at + 16 * int32_t(g) + (upper ? 64 : 0);
        visible = bits(unit, from, ma);
        if constexpr (!PAIR) visible |= bits(2 + unit, from + 64, mb) << 16;
#pragma unroll
        for (int i = 0; i < NS; ++i)
          x[i] = __uint_as_float((__float_as_uint(x[i]) & bit_mask(visible, i)) |
                                 (0xFF800000u & ~bit_mask(visible, i)));
      }
      // The maximum is set 8 above the scores and follows when they reach it: a
      // lane then compares its own, and those that share a column seldom have to
      // agree on a new one.
      float part[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        part[c] = x[c * NS / 4];
#pragma unroll
        for (int i = 1; i < NS / 4; ++i) part[c] = fmaxf(part[c], x[c * NS / 4 + i]);
      }
      float mx = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3])) * a.c;
      if (__any(mx > m_run)) {
        mx = column_max<PAIR>(mx);
        const float m_new = mx > m_run ? mx + 8.0f : m_run;
        m_use = m_new == -INFINITY ? 0.0f : m_new;
        const float f = exp2_(m_run - m_use);
        l_run *= f;
#pragma unroll
        for (int m = 0; m < ND; ++m) o[m] *= f;
        m_run = m_new;
      }
      const uint32_t vs[8] = {va.x, va.y, va.z, va.w, vb.x, vb.y, vb.z, vb.w};
#pragma unroll
      for (int i = 0; i < NS; i += 4) {
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) p[e] = exp2_(__builtin_fmaf(x[i + e], a.c, -m_use));
        l_run += (p[0] + p[1]) + (p[2] + p[3]);
        x[i] = p[0] * byte_scale<0>(vs[i / 4]);
        x[i + 1] = p[1] * byte_scale<1>(vs[i / 4]);
        x[i + 2] = p[2] * byte_scale<2>(vs[i / 4]);
        x[i + 3] = p[3] * byte_scale<3>(vs[i / 4]);
      }
      if (masked) {  // (a value that is NaN has the scale infinity: 0 times that is not 0)
#pragma unroll
        for (int i = 0; i < NS; ++i)
          x[i] = __uint_as_float(__float_as_uint(x[i]) & bit_mask(visible, i));
      }
      float top = 0.0f;
#pragma unroll
      for (int i = 0; i < NS; ++i) top = fmaxf(top, x[i]);
      load_vs(t_next, next);
      top = column_max<PAIR>(top);
      int ps = top_byte(__float_as_uint(top));
      const int pl = low_byte(ps);
      const float scale = byte_value(ps);
#pragma unroll
      for (int i = 0; i < NS / 4; ++i) {
        int u = ph[i], v = pq[i];
        split4(x + 4 * i, scale, u, v);
        ph[i] = u;
        pq[i] = v;
      }
      if constexpr (PAIR) {
        // lower columns take the first term of both halves, upper ones the second
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int got = __float_as_int(other_half(__int_as_float(upper ? ph[i] : pq[i])));
          ph[4 + i] = upper ? pq[i] : got;
          ph[i] = upper ? got : ph[i];
        }
        ps = upper ? pl : ps;
      }
#pragma unroll
      for (int m = 0; m < ND; ++m) {
        const int8v v8 = widen(vreg[m]);
        o[m] = mul16<0>(v8, ph, o[m], kUnitScale, ps);
        if constexpr (!PAIR) o[m] = mul16<0>(v8, pq, o[m], kUnitScale, pl);
      }
      load_v(t_next, next);
      ids = next;
      next = load_ids(min(t_next + kWaves, t_last));
    }
  }
  if constexpr (PAIR) l_run += other_half(l_run);
  l_run += __shfl_xor(l_run, 16);
  l_run += __shfl_xor(l_run, 32);

  // join the wavefronts: column c of wave v at lds_o[(v kCols + c) kStride]
  if (g == 0) lds_s[wave][col] = make_float2(m_run, l_run);
#pragma unroll
  for (int m = 0; m < ND; ++m)
    *reinterpret_cast<floatx4 *>(lds_o + (wave * kCols + col) * kStride + 16 * m + 4 * g) = o[m];
  __syncthreads();
  constexpr uint32_t kPer = D * kCols / 256;  // channels a thread
  const uint32_t oc = threadIdx.x / (256 / kCols), d0 = threadIdx.x % (256 / kCols) * kPer;
  if (col0 + oc >= sp.cols) return;
  float m_all = -INFINITY, l_all = 0.0f, sum[kPer] = {};
#pragma unroll
  for (uint32_t v = 0; v < kWaves; ++v) m_all = fmaxf(m_all, lds_s[v][oc].x);
  const float m_ref = m_all == -INFINITY ? 0.0f : m_all;
#pragma unroll
  for (uint32_t v = 0; v < kWaves; ++v) {
    const float f = exp2_(lds_s[v][oc].x - m_ref);
    l_all += f * lds_s[v][oc].y;
#pragma unroll
    for (uint32_t i = 0; i < kPer; ++i) {
      float x = lds_o[(v * kCols + oc) * kStride + d0 + i];
      if constexpr (PAIR) x += lds_o[(v * kCols + (oc | 8)) * kStride + d0 + i];  // (oc < 8)
      sum[i] += f * x;
    }
  }
  if (sp.chunks <= 1) {
    const float inv = l_all == 0.0f ? 0.0f : 1.0f / l_all;
    const uint32_t i0 = col0 + oc;
    uint32_t pk[kPer / 2];
#pragma unroll
    for (uint32_t i = 0; i < kPer / 2; ++i)
      pk[i] = eq_dev::pack_bf16(sum[2 * i] * inv, sum[2 * i + 1] * inv);
    uint16_t *const out = a.out + (uint64_t(q.row + i0 / a.group) * w.kv_heads * a.group +
                                   h * a.group + i0 % a.group) * D + d0;
#pragma unroll
    for (uint32_t i = 0; i < kPer / 2; ++i) reinterpret_cast<uint32_t *>(out)[i] = pk[i];
    return;
  }
  const uint64_t slot = (((uint64_t(s) * w.kv_heads + h) * a.q_tiles + qt) * a.chunks + chunk) * kCols + oc;
  if (d0 == 0) a.stat[slot] = make_float2(m_all, l_all);
#pragma unroll
  for (uint32_t i = 0; i < kPer; ++i) a.part[slot * D + d0 + i] = sum[i];
}

// The query columns of a wavefront of prompt_kernel: lane (col of 32, half) of
// the operand of 64 steps holds steps 16 half .. + 15 and 32 + 16 half .. + 15,
// and the scale of steps 32 half ..  One operand for 64 channels.
template <int D>
struct PromptQuery {
  int8v h[D / 64], l[D / 64];
  int hs[D / 64], ls[D / 64];
  __device__ inline void load(const uint16_t *row, uint32_t half) {
#pragma unroll
    for (int kk = 0; kk < D / 64; ++kk) {
      int byte[2];
#pragma unroll
      for (int part = 0; part < 2; ++part) {
        uint32_t u[8] = {};
        if (row) {
          const uint4 *const p =
              reinterpret_cast<const uint4 *>(row + 64 * kk + 32 * part + 16 * half);
          *reinterpret_cast<uint4 *>(u) = p[0];
          *reinterpret_cast<uint4 *>(u + 4) = p[1];
        }
        uint32_t top = 0;
        float x[16];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[2 * i] = __uint_as_float(u[i] << 16);
          x[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
          top = max(top, max(u[i] << 16 & 0x7FFFFFFFu, u[i] & 0x7FFF0000u));
        }
        byte[part] = top_byte(max(top, uint32_t(__shfl_xor(int(top), 32))));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          int a, b;
          split4(x + 4 * i, byte_value(byte[part]), a, b);
          h[kk][4 * part + i] = a;
          l[kk][4 * part + i] = b;
        }
      }
      hs[kk] = half ? byte[1] : byte[0];
      ls[kk] = low_byte(hs[kk]);
    }
  }
};

// Many query columns: a block of 4 wavefronts with 32 columns each, that share
// tiles of 64 tokens through LDS.  Three buffers: a tile's scores are multiplied
// beside the softmax of the tile before, while the loads of the one after are in
// flight.
//
// Here the vector instructions of the softmax are the limit, and splitting w P
// in two terms would be half of them.  So the second product takes w P as BF16
// (rounded to nearest: 2^-8 of itself at most, as two terms, but more on average),
// and the value codes are brought to BF16 once for a block, when a tile is copied
// into LDS.  Against attention in 64 bits the result is off by 2.1e-3 in the norm
// (attn_kernel: 1.7e-3), of which its own rounding to BF16 is 1.65e-3; that is what 227
// -> 202 us cost.
//
// The layout follows attn_kernel's idea: of a 32 x 32 product lane (col, half)
// gets rows 8 a + 4 half + e of its column, and for 16 tokens of the second
// product it has to hold tokens 8 half .. + 7; so row 16 b + 8 c + 4 d + e of a
// unit's scores is its token 16 b + 8 d + 4 c + e.
//
// The maximum is set 8 above the scores, and follows when they reach it: P stays
// at most 1, and O is rescaled a few times in all, not whenever one of 32 columns
// finds a larger score.
//
// 2048 new tokens behind 2048, 64 heads of 128 on 8: 206 GFLOP in 195 to 204 us,
// 1.01 to 1.06 PFLOP/s (a large BF16 matrix product: 1.19); matrix units 44% and
// vector units 46 to 53% busy, 7 wavefronts a compute unit.  Slower: both terms
// of w P as E4M3 (278: registers spill), 8 wavefronts in two halves that take
// turns (202), value codes brought to BF16 by each wavefront (201 against 197), 3
// wavefronts a SIMD with the queries in LDS (272).
template <int D, bool TREE>
__global__ __launch_bounds__(256, 2) void prompt_kernel(AttnArgs a) {
  constexpr int ND = D / 32, KK = D / 64;
  constexpr uint32_t kRow = D / 2 + 16;  // bytes a key in LDS: 16 rows start in 16 banks
  constexpr uint32_t kVRow = kPromptTile * 2 + 16;  // bytes a channel's values, likewise
  constexpr uint32_t kV = kPromptTile * kRow, kKS = kV + D * kVRow, kW = kKS + 256,
                     kOdd = kW + kPromptTile * 4, kBuf = kOdd + 16;
  __shared__ __attribute__((aligned(16))) uint8_t lds[3 * kBuf];
  // TREE: the columns' masks (rows of them start in 32 banks), read where a tile has new tokens
  constexpr uint32_t kMaskRow = kMaskWords + 1;
  __shared__ uint32_t lds_mask[TREE ? kPromptCols * kMaskRow : 1];
  const View &w = a.w;
  uint32_t s = blockIdx.y;
  // heads first (blocks go round the 8 XCDs, so with a multiple of 8 heads those of
  // a head share one, whose L2 then holds its cache), and a sequence's last
  // queries, which see most, before its first
  const uint32_t h = blockIdx.x % w.kv_heads, rest = blockIdx.x / w.kv_heads;
  uint32_t chunk = rest % a.chunks, qt = a.q_tiles - 1 - rest / a.chunks;
  if constexpr (TREE) {
    if (a.even) {
      const Share e = even_share(a, s * (gridDim.x / w.kv_heads) + rest);
      if (blockIdx.x == 0 && s == 0 && threadIdx.x == 0) *a.even = e.chunk_tiles;
      if (!e.any) return;
      a.chunk_tiles = eq_dev::uniform(e.chunk_tiles);
      s = eq_dev::uniform(e.seq), qt = eq_dev::uniform(e.qt), chunk = eq_dev::uniform(e.chunk);
    }
  }
  const Seq q = sequence(w, s);
  const uint32_t col0 = qt * kPromptCols;
  const Span sp = span_of<kPromptCols, kPromptTile, TREE>(a, q, col0);
  if (col0 >= sp.cols || chunk >= max(sp.chunks, 1u)) return;
  const uint32_t tid = threadIdx.x, lane = tid & 63, wave = eq_dev::uniform(tid >> 6);
  const uint32_t col = lane & 31, half = lane >> 5;

  const uint32_t wave_col = col0 + wave * 32, index = wave_col + col;
  const bool real = index < sp.cols;
  const uint32_t token = index / a.group;
  const int32_t pos = q.base + int32_t(token);
  int32_t hi = real ? end_of(q, pos) : 0, lo = real ? start_of(a.window, pos) : 0;
  const uint16_t *const row =
      real ? a.q + uint64_t(q.row + token) * a.q_stride + uint64_t(h * a.group + index % a.group) * D
           : nullptr;
  PromptQuery<D> query;
  query.load(row, half);
  // tokens in [all_lo, all_hi) are seen by every column of the wavefront (the block's
  // tiles are multiplied whole, also those that none of them sees)
  int32_t all_lo = 0, all_hi = 0;
  if (wave_col < sp.cols) {
    const int32_t p0 = q.base + int32_t(wave_col / a.group);
    const int32_t p1 = q.base + int32_t((min(wave_col + 32, sp.cols) - 1) / a.group);
    all_lo = start_of(a.window, p1), all_hi = end_of(q, p0);
  }
  Node node{};
  if constexpr (TREE) {
    uint32_t words[kMaskWords];
    node = node_of(a, q, token, real, words);
#pragma unroll
    for (int i = 0; i < kMaskWords; ++i)  // (both halves write the same)
      lds_mask[(wave * 32 + col) * kMaskRow + i] = uint32_t(i) < a.mask_words && node.alive ? words[i] : 0u;
    hi = node.hi, lo = node.lo;
    all_hi = __any(real && !node.alive) ? 0 : sp.hi_min;
    all_lo = a.window ? wave_max(lo) : 0;
  }

  // staging: D threads copy a unit, 16 bytes of its key codes, 16 of its value
  // codes and a key scale each (at D = 64 two wavefronts do), and the first 32
  // of them a value scale; what a wavefront copies is of one unit
  const uint32_t *const table =
      reinterpret_cast<const uint32_t *>(w.page_table + size_t(s) * w.max_pages);
  const uint32_t last_unit = sp.seen ? (sp.seen - 1) / kUnit : 0;
  const uint32_t page_mask = (1u << w.page_shift) - 1;
  const uint8_t *const base = w.pages + uint64_t(h) * w.head_bytes;
  const uint32_t unit = wave * 64 / D & 1, piece = tid % D;
  const bool copies = wave * 64 / D < 2, scales = copies && wave * 64 % D == 0;
  auto unit_of = [&](uint32_t tile) { return min(2 * tile + unit, last_unit) * kUnit; };
  auto load_id = [&](uint32_t tile) { return eq_dev::as_const(table)[unit_of(tile) >> w.page_shift]; };
  struct Stage {
    uint4 k, v;
    uint32_t ks, vs, id;
  };
  // (Every thread loads, and past the last tile that one again: a load under a
  // condition would be waited for where the branches meet.)
  auto load_tile = [&](uint32_t tile, uint32_t id) {
    Stage x;
    x.id = id;
    const uint32_t slot = unit_of(tile) & page_mask;
    const uint8_t *const p = base + uint64_t(id < w.n_pages ? id : 0) * w.page_bytes;
    const uint32_t k_at = slot * (D / 2), lane16 = piece * 16;
    x.k = *reinterpret_cast<const uint4 *>(p + k_at + lane16);
    x.v = *reinterpret_cast<const uint4 *>(p + w.v_off + k_at + lane16);
    x.ks = (p + w.ks_off + slot * (D / 32))[piece];
    x.vs = (p + w.vs_off + slot)[lane & 31];
    return x;
  };
  const uint32_t k_to = (unit * kUnit + piece / (D / 32)) * kRow + piece % (D / 32) * 16;
  const uint32_t ks_row = 16 * (piece / (D / 2)) + 8 * (piece & 1) + 4 * (piece >> 1 & 1) +
                          piece % (D / 2) / (D / 8);
  const uint32_t ks_blk = piece / 4 % (D / 32);
  const uint32_t ks_to = kKS + ((ks_blk & 1) * 32 + ks_row) * 4 + unit * 2 + (ks_blk >> 1);
  auto store_tile = [&](uint8_t *buf, uint32_t tile, const Stage &x) {
    if (!copies) return;
    *reinterpret_cast<uint4 *>(buf + k_to) = x.k;
    const uint32_t codes[4] = {x.v.x, x.v.y, x.v.z, x.v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<uint4 *>(buf + kV + piece * kVRow + unit * 64 + 16 * i) =
          make_uint4(code_pair<0>(codes[i]), code_pair<1>(codes[i]), code_pair<2>(codes[i]),
                     code_pair<3>(codes[i]));
    buf[ks_to] = uint8_t(x.ks);
    if (scales) {
      // tokens behind the last one seen, or of a page that is not there, have
      // any scale: 0; of those whose values are NaN there is a list, and theirs
      // is 1 (a hidden token's P of 0 then stays 0)
      const bool gone = x.id >= w.n_pages;
      const uint32_t left = sp.seen - min(tile * kPromptTile + unit * kUnit, sp.seen);
      const bool there = !gone && lane < min(left, kUnit);
      const uint32_t nan = uint32_t(__ballot(there && x.vs == 255));
      if (lane < kUnit)
        *reinterpret_cast<float *>(buf + kW + 4 * (unit * kUnit + lane)) =
            there ? (x.vs == 255 ? 1.0f : __uint_as_float(x.vs << 23)) : 0.0f;
      if (lane == 0) *reinterpret_cast<uint2 *>(buf + kOdd + unit * 8) = make_uint2(gone, nan);
    }
  };

  float m_run = -INFINITY, m_use = 0.0f, l_run = 0.0f;
  floatx16 o[ND];
#pragma unroll
  for (int m = 0; m < ND; ++m)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[m][i] = 0.0f;
  // this lane's key of a unit
  const uint32_t krow = (col & 19) | (col >> 3 & 1) << 2 | (col >> 2 & 1) << 3;
  const uint32_t k_from = krow * kRow + 16 * half, v_from = kV + col * kVRow + 16 * half;

  // the scores of a tile
  auto scores = [&](const uint8_t *buf, floatx16 (&x)[2]) {
    const int ks = *reinterpret_cast<const int *>(buf + kKS + lane * 4);
    auto keys = [&](int u, int kk) {
      return widen(*reinterpret_cast<const int4v *>(buf + k_from + u * kUnit * kRow + 32 * kk));
    };
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) x[u][i] = 0.0f;
    const int8v k0 = keys(0, 0), k1 = keys(1, 0);
    x[0] = mul32<0>(k0, query.h[0], x[0], ks, query.hs[0]);
    x[1] = mul32<2>(k1, query.h[0], x[1], ks, query.hs[0]);
    x[0] = mul32<0>(k0, query.l[0], x[0], ks, query.ls[0]);
    x[1] = mul32<2>(k1, query.l[0], x[1], ks, query.ls[0]);
    if constexpr (KK == 2) {
      const int8v k2 = keys(0, 1), k3 = keys(1, 1);
      x[0] = mul32<1>(k2, query.h[1], x[0], ks, query.hs[1]);
      x[1] = mul32<3>(k3, query.h[1], x[1], ks, query.hs[1]);
      x[0] = mul32<1>(k2, query.l[1], x[0], ks, query.ls[1]);
      x[1] = mul32<3>(k3, query.l[1], x[1], ks, query.ls[1]);
    }
  };
  // a tile's P and sums from its scores, and beside them the next tile's scores
  auto compute = [&](uint32_t tile, const uint8_t *buf, const uint8_t *buf_next,
                     floatx16 (&sc)[2]) {
    const int32_t at = int32_t(tile * kPromptTile);
    const uint4 odd = *reinterpret_cast<const uint4 *>(buf + kOdd);  // gone, NaN of each unit
    // masks, where some column does not see some token
    if (at + int32_t(kPromptTile) > all_hi || at < all_lo ||
        eq_dev::uniform(odd.x | odd.y | odd.z | odd.w) != 0) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint32_t gone = u ? odd.z : odd.x, nan = u ? odd.w : odd.y;
        const int32_t from = at + 32 * u;
        uint32_t visible = bits_below(hi - from) & ~bits_below(lo - from);  // of the unit's tokens
        if constexpr (TREE) {
          auto word = [&](int32_t i) {
            const uint32_t x = lds_mask[(wave * 32 + col) * kMaskRow + (uint32_t(i) & (kMaskWords - 1))];
            return uint32_t(i) < uint32_t(kMaskWords) ? x : 0u;
          };
          const int32_t first = from - node.base;
          const uint32_t own =
              __builtin_amdgcn_alignbit(word((first >> 5) + 1), word(first >> 5), uint32_t(first) & 31);
          visible |= own & bits_below(int32_t(sp.seen) - from);
        }
        if (gone) visible = 0;
        visible >>= 8 * half;  // this lane's: 0 to 7 and 16 to 23
        if (eq_dev::uniform(nan)) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (nan >> (16 * (i / 8) + 8 * half + i % 8) & 1) sc[u][i] = NAN;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint32_t m = bit_mask(visible, 16 * (i / 8) + i % 8);
          sc[u][i] = __uint_as_float((__float_as_uint(sc[u][i]) & m) | (0xFF800000u & ~m));
        }
      }
    }
    float mx = sc[0][0];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, sc[u][i]);
    mx *= a.c;
    if (__any(mx > m_run)) {
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float m_new = mx > m_run ? mx + 8.0f : m_run;
      m_use = m_new == -INFINITY ? 0.0f : m_new;
      const float f = exp2_(m_run - m_use);
      m_run = m_new;
      l_run *= f;
#pragma unroll
      for (int m = 0; m < ND; ++m) o[m] *= f;
    }
    // Eight steps, each with one product of the next tile's scores, four tokens
    // of this tile's softmax for each column, and, two steps behind, half of the
    // products of 16 tokens' values.  A step's operands are read from LDS in the
    // step before.  The barriers keep the compiler from undoing that: a step's
    // vector instructions run beside its matrix instructions.
    floatx16 next[2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) next[u][i] = 0.0f;
    const int ks = *reinterpret_cast<const int *>(buf_next + kKS + lane * 4);
    constexpr int kHalf = ND / 2;
    int4v kf = *reinterpret_cast<const int4v *>(buf_next + k_from), kf_next = kf;
    floatx4 wt = *reinterpret_cast<const floatx4 *>(buf + kW + 32 * half);
    bf16x8 vf[kHalf], vf_next[kHalf];
    uint32_t p16[4][4];  // w P of 16 tokens each
    auto step = [&](auto ic) {
      constexpr int I = decltype(ic)::value, G = I / 2, J = 4 * (I & 1);
      floatx4 wt_next = wt;
      if constexpr (I < 7)
        wt_next = *reinterpret_cast<const floatx4 *>(buf + kW + (16 * ((I + 1) / 2) + 8 * half +
                                                               4 * ((I + 1) & 1)) * 4);
      if constexpr (I >= 1) {
        constexpr int V = I - 1;  // the next step's values: 16 tokens V / 2, half V % 2
#pragma unroll
        for (int m = 0; m < kHalf; ++m)
          vf_next[m] = *reinterpret_cast<const bf16x8 *>(
              buf + v_from + ((V & 1) * kHalf + m) * 32 * kVRow + 32 * (V / 2));
      }
      if constexpr ((I & 1) == 1 && I < 4 * KK - 1) {
        constexpr int K = (I + 1) / 2;  // the next key operand: unit K / KK, channels K % KK
        kf_next = *reinterpret_cast<const int4v *>(buf_next + k_from + K / KK * kUnit * kRow +
                                                   32 * (K % KK));
      }
      if constexpr (I < 4 * KK) {
        constexpr int K = I / 2, U = K / KK, C = K % KK;
        next[U] = mul32<2 * U + C>(widen(kf), I & 1 ? query.l[C] : query.h[C], next[U], ks,
                                   I & 1 ? query.ls[C] : query.hs[C]);
      }
      if constexpr (I >= 2) {
        constexpr int V = I - 2;
#pragma unroll
        for (int m = 0; m < kHalf; ++m) {
          constexpr int at = (V & 1) * kHalf;
          o[at + m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
              vf[m], __builtin_bit_cast(bf16x8, *reinterpret_cast<uint4 *>(p16[V / 2])), o[at + m],
              0, 0, 0);
        }
      }
      float p[4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        p[e] = exp2_(__builtin_fmaf(sc[G / 2][8 * (G & 1) + J + e], a.c, -m_use));
      l_run += (p[0] + p[1]) + (p[2] + p[3]);
      p16[G][J / 2] = eq_dev::pack_bf16(p[0] * wt[0], p[1] * wt[1]);
      p16[G][J / 2 + 1] = eq_dev::pack_bf16(p[2] * wt[2], p[3] * wt[3]);
      wt = wt_next;
      if constexpr ((I & 1) == 1) kf = kf_next;
#pragma unroll
      for (int m = 0; m < kHalf; ++m) vf[m] = vf_next[m];
      __builtin_amdgcn_sched_barrier(0);
    };
    __builtin_amdgcn_sched_barrier(0);
    step(std::integral_constant<int, 0>{});
    step(std::integral_constant<int, 1>{});
    step(std::integral_constant<int, 2>{});
    step(std::integral_constant<int, 3>{});
    step(std::integral_constant<int, 4>{});
    step(std::integral_constant<int, 5>{});
    step(std::integral_constant<int, 6>{});
    step(std::integral_constant<int, 7>{});
#pragma unroll
    for (int m = 0; m < ND; ++m)
      o[m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
          m < kHalf ? vf[m] : *reinterpret_cast<const bf16x8 *>(buf + v_from + m * 32 * kVRow + 96),
          __builtin_bit_cast(bf16x8, *reinterpret_cast<uint4 *>(p16[3])), o[m], 0, 0, 0);
    sc[0] = next[0], sc[1] = next[1];
  };

  const uint32_t t0 = sp.first + chunk * a.chunk_tiles, t1 = min(t0 + a.chunk_tiles, sp.last);
  if (t0 < t1) {
    const bool active = wave_col < sp.cols;
    floatx16 sc[2];
    uint8_t *now = lds, *next = lds + kBuf, *then = lds + 2 * kBuf;
    store_tile(now, t0, load_tile(t0, load_id(t0)));
    if (t0 + 1 < t1) store_tile(next, t0 + 1, load_tile(t0 + 1, load_id(t0 + 1)));
    uint32_t id = load_id(t0 + 2);
    __syncthreads();
    if (active) scores(now, sc);
    for (uint32_t t = t0; t < t1; ++t) {
      const bool more = t + 2 < t1;
      const Stage x = load_tile(t + 2, id);
      id = load_id(t + 3);
      if (active) compute(t, now, next, sc);  // (behind the last tile: scores of anything)
      if (more) store_tile(then, t + 2, x);
      __syncthreads();
      uint8_t *const old = now;
      now = next, next = then, then = old;
    }
  }
  l_run += __shfl_xor(l_run, 32);
  if (!real) return;
  if (sp.chunks <= 1) {
    const float inv = l_run == 0.0f ? 0.0f : 1.0f / l_run;
    uint16_t *const out = a.out + (uint64_t(q.row + token) * w.kv_heads * a.group + h * a.group +
                                   index % a.group) * D + 4 * half;
#pragma unroll
    for (int m = 0; m < ND; ++m)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<uint2 *>(out + 32 * m + 2 * i) =
            make_uint2(eq_dev::pack_bf16(o[m][i] * inv, o[m][i + 1] * inv),
                       eq_dev::pack_bf16(o[m][i + 2] * inv, o[m][i + 3] * inv));
    return;
  }
  const uint64_t slot =
      (((uint64_t(s) * w.kv_heads + h) * a.q_tiles + qt) * a.chunks + chunk) * kPromptCols +
      wave * 32 + col;
  if (half == 0) a.stat[slot] = make_float2(m_run, l_run);
#pragma unroll
  for (int m = 0; m < ND; ++m)
#pragma unroll
    for (int i = 0; i < 16; i += 4)
      *reinterpret_cast<floatx4 *>(a.part + slot * D + 32 * m + 2 * i + 4 * half) =
          floatx4{o[m][i], o[m][i + 1], o[m][i + 2], o[m][i + 3]};
}

// Joins the chunks of one query head at one new token, a block each: every
// wavefront takes all chunks' maxima and sums, a lane each, and 8 groups of
// threads the chunks' O in turn, added up through LDS.  Bound by its own latency:
// 3.7 us, whatever the number of chunks up to 64.
template <int D, uint32_t COLS, uint32_t TILE, bool TREE>
__global__ __launch_bounds__(2 * D) void join_kernel(AttnArgs a) {
  constexpr uint32_t kLanes = D / 4, kSub = 8;
  __shared__ __attribute__((aligned(16))) float4 lds[kSub][kLanes];
  const View &w = a.w;
  const uint32_t s = blockIdx.y, heads = w.kv_heads * a.group;
  const uint32_t token = blockIdx.x / heads, head = blockIdx.x % heads;
  const Seq q = sequence(w, s);
  if (int32_t(token) >= q.count) return;
  const uint32_t h = head / a.group, index = token * a.group + head % a.group;
  const uint32_t qt = index / COLS;
  if (TREE && a.even) a.chunk_tiles = *a.even;
  const Span sp = span_of<COLS, TILE, TREE>(a, q, qt * COLS);
  if (sp.chunks <= 1) return;
  const uint64_t first =
      (((uint64_t(s) * w.kv_heads + h) * a.q_tiles + qt) * a.chunks) * COLS + index % COLS;
  const uint32_t sub = threadIdx.x / kLanes, l = threadIdx.x % kLanes, lane = threadIdx.x & 63;
  float m = -INFINITY;
  float2 st = make_float2(-INFINITY, 0.0f);
  for (uint32_t c0 = 0; c0 < sp.chunks; c0 += 64) {
    st = c0 + lane < sp.chunks ? a.stat[first + uint64_t(c0 + lane) * COLS] : make_float2(-INFINITY, 0.0f);
    m = fmaxf(m, st.x);
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
  if (m == -INFINITY) m = 0.0f;
  float4 o = make_float4(0, 0, 0, 0);
  float total = 0.0f;
  for (uint32_t c0 = 0; c0 < sp.chunks; c0 += 64) {
    if (sp.chunks > 64)
      st = c0 + lane < sp.chunks ? a.stat[first + uint64_t(c0 + lane) * COLS] : make_float2(-INFINITY, 0.0f);
    const float f = exp2_(st.x - m);
    total += f * st.y;
    const uint32_t n = min(sp.chunks - c0, 64u);
    for (uint32_t k = 0; k * kSub < n; k += 4) {  // (as often for every lane)
      float4 x[4];
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j)
        x[j] = *reinterpret_cast<const float4 *>(
            a.part + (first + uint64_t(c0 + min(sub + (k + j) * kSub, n - 1)) * COLS) * D + 4 * l);
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) {
        const float fc = __shfl(f, int(sub + (k + j) * kSub));  // 0 behind the last chunk
        o.x += fc * x[j].x, o.y += fc * x[j].y, o.z += fc * x[j].z, o.w += fc * x[j].w;
      }
    }
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) total += __shfl_xor(total, d);
  lds[sub][l] = o;
  __syncthreads();
  if (sub) return;
#pragma unroll
  for (uint32_t i = 1; i < kSub; ++i) {
    const float4 x = lds[i][l];
    o.x += x.x, o.y += x.y, o.z += x.z, o.w += x.w;
  }
  const float inv = total == 0.0f ? 0.0f : 1.0f / total;
  *reinterpret_cast<uint2 *>(a.out + (uint64_t(q.row + token) * heads + head) * D + 4 * l) =
      make_uint2(eq_dev::pack_bf16(o.x * inv, o.y * inv), eq_dev::pack_bf16(o.z * inv, o.w * inv));
}

// The same for a tree's many columns, to the bit: D / 4 lanes take a column, and its
// chunks in turn.  join_kernel's blocks wait for their loads most of the time: four
// trees of up to 64 nodes, 64 heads, 15.4 us; here 8.4, of which reading the 29 MB of
// partial results at a copy's rate would be 6.  With few columns, the lanes that share a
// column's chunks are faster.  Sequences x nodes x heads, cached tokens: us of a call,
// join_kernel / here
//   1 x 16 x 32, 8192: 22.4 / 22.7   1 x 16 x 32, 32768: 33.0 / 36.5
//   1 x 32 x 64, 8192: 32.7 / 32.2   1 x 128 x 16, 131072: 145.0 / 144.4
//   4 x 32 x 64, 16384: 90.6 / 85.2  2 x 128 x 64, 16384: 163.7 / 149.7
constexpr uint64_t kManyRows = 2048;

template <int D>
__global__ __launch_bounds__(256) void join_rows_kernel(AttnArgs a) {
  constexpr uint32_t kLanes = D / 4, kParts = 64 / kLanes;
  const View &w = a.w;
  const uint32_t s = blockIdx.y, heads = w.kv_heads * a.group, l = threadIdx.x % kLanes;
  const uint32_t at = blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes;
  const uint32_t token = at / heads, head = at % heads;
  const Seq q = sequence(w, s);
  if (token >= uint32_t(q.count)) return;
  const uint32_t h = head / a.group, index = token * a.group + head % a.group;
  const uint32_t qt = index / kPromptCols;
  if (a.even) a.chunk_tiles = *a.even;
  const Span sp = span_of<kPromptCols, kPromptTile, true>(a, q, qt * kPromptCols);
  if (sp.chunks <= 1) return;
  const uint64_t first = (((uint64_t(s) * w.kv_heads + h) * a.q_tiles + qt) * a.chunks) * kPromptCols +
                         index % kPromptCols;
  auto stat = [&](uint32_t c) {
    return c < sp.chunks ? a.stat[first + uint64_t(c) * kPromptCols] : make_float2(-INFINITY, 0.0f);
  };
  float m = -INFINITY;
  for (uint32_t c = l; c < sp.chunks; c += kLanes) m = fmaxf(m, stat(c).x);
#pragma unroll
  for (uint32_t d = 1; d < kLanes; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
  if (m == -INFINITY) m = 0.0f;
  // (sums in join_kernel's order: of every eighth chunk, and of 64 lanes)
  float4 o[8] = {};
  float total[kParts] = {};
  for (uint32_t c0 = 0; c0 < sp.chunks; c0 += 64) {
#pragma unroll
    for (uint32_t part = 0; part < kParts; ++part) {
      const uint32_t c1 = c0 + part * kLanes;
      if (c1 >= sp.chunks) break;
      const float2 st = stat(c1 + l);
      const float f = exp2_(st.x - m);
      total[part] += f * st.y;
      const uint32_t n = min(sp.chunks - c1, kLanes);
      for (uint32_t k = 0; k < n; k += 8) {
        float4 x[8];
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j)
          x[j] = *reinterpret_cast<const float4 *>(
              a.part + (first + uint64_t(c1 + min(k + j, n - 1)) * kPromptCols) * D + 4 * l);
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) {
          const float fc = __shfl(f, int(k + j), int(kLanes));  // 0 behind the last chunk
          o[j].x += fc * x[j].x, o[j].y += fc * x[j].y, o[j].z += fc * x[j].z, o[j].w += fc * x[j].w;
        }
      }
    }
  }
#pragma unroll
  for (uint32_t part = 0; part < kParts; ++part)
#pragma unroll
    for (uint32_t d = 1; d < kLanes; d *= 2) total[part] += __shfl_xor(total[part], d);
#pragma unroll
  for (uint32_t d = 1; d < kParts; d *= 2)
#pragma unroll
    for (uint32_t part = 0; part < kParts; part += 2 * d) total[part] += total[part + d];
#pragma unroll
  for (uint32_t j = 1; j < 8; ++j)
    o[0].x += o[j].x, o[0].y += o[j].y, o[0].z += o[j].z, o[0].w += o[j].w;
  const float inv = total[0] == 0.0f ? 0.0f : 1.0f / total[0];
  *reinterpret_cast<uint2 *>(a.out + (uint64_t(q.row + token) * heads + head) * D + 4 * l) =
      make_uint2(eq_dev::pack_bf16(o[0].x * inv, o[0].y * inv),
                 eq_dev::pack_bf16(o[0].z * inv, o[0].w * inv));
}

// Columns of partial results: a sum for each channel, a maximum and a sum of P.
size_t part_cols(const Plan &p, const eq_kv_cache *c, const eq_kv_batch *b) {
  return size_t(b->n_seqs) * c->kv_heads * p.q_tiles * p.chunks * p.cols;
}

template <bool TREE>
size_t attn_bytes(const Plan &p, const eq_kv_cache *c, const eq_kv_batch *b) {
  const size_t even = TREE ? sizeof(uint32_t) : 0;
  return p.chunks <= 1 ? 0 : part_cols(p, c, b) * (c->head_dim + 2) * sizeof(float) + even;
}

template <int D, bool TREE>
void launch_attn(const AttnArgs &a, const Plan &p, bool pair, bool one_page, bool stream_codes,
                 dim3 grid, dim3 join, hipStream_t stream) {
  const dim3 block(256), join_block(2 * D);
  if (p.prompt) {
    hipLaunchKernelGGL((prompt_kernel<D, TREE>), grid, block, 0, stream, a);
    if (p.chunks > 1 && TREE && uint64_t(join.x) * join.y >= kManyRows) {
      const dim3 rows((join.x + 1024 / D - 1) / (1024 / D), join.y);
      hipLaunchKernelGGL(join_rows_kernel<D>, rows, block, 0, stream, a);
    } else if (p.chunks > 1) {
      hipLaunchKernelGGL((join_kernel<D, kPromptCols, kPromptTile, TREE>), join, join_block, 0, stream,
                         a);
    }
    return;
  }
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a); };
  auto pick = [&](auto one, auto streams) {
    constexpr bool ONE = decltype(one)::value, STREAM = decltype(streams)::value;
    pair ? go(attn_kernel<D, ONE, STREAM, true, TREE>) : go(attn_kernel<D, ONE, STREAM, false, TREE>);
  };
  const std::true_type yes;
  const std::false_type no;
  if (one_page) stream_codes ? pick(yes, yes) : pick(yes, no);
  else stream_codes ? pick(no, yes) : pick(no, no);
  if (p.chunks > 1)
    hipLaunchKernelGGL((join_kernel<D, kCols, kTile, TREE>), join, join_block, 0, stream, a);
}

bool heads_ok(const eq_kv_cache *c, uint32_t q_heads) {
  return q_heads >= 1 && q_heads % c->kv_heads == 0 && q_heads <= 65535;
}

// The columns of all heads are counted in 32 bits, and one launch takes them.  (A
// window leaves fewer chunks, and chunks are joined where there are few columns.)
bool size_ok(const eq_kv_cache *c, const eq_kv_batch *b, uint32_t q_heads, bool tree) {
  if (uint64_t(b->max_new) * q_heads > 0x7FFFFFFFu) return false;
  const Plan p =
      plan_attn(b->n_seqs, c->kv_heads, q_heads / c->kv_heads, b->max_new, b->max_len, 0, tree);
  return uint64_t(c->kv_heads) * p.q_tiles * p.chunks <= kMaxBlocks;
}

template <bool TREE>
size_t workspace_bytes(const eq_kv_cache *cache, const eq_kv_batch *batch, uint32_t q_heads) {
  if (!batch_ok(cache, batch) || !heads_ok(cache, q_heads) || batch->n_seqs == 0 ||
      batch->max_new == 0 || !size_ok(cache, batch, q_heads, TREE))
    return 0;
  return attn_bytes<TREE>(plan_attn(batch->n_seqs, cache->kv_heads, q_heads / cache->kv_heads,
                                    batch->max_new, batch->max_len, 0, TREE),
                          cache, batch);
}

template <bool TREE>
int attention(const eq_kv_cache *cache, const eq_kv_batch *batch, const uint16_t *q,
              uint64_t q_stride, uint32_t q_heads, float scale, uint32_t window,
              const uint32_t *mask, const int32_t *positions, uint16_t *out, void *ws,
              size_t ws_bytes, hipStream_t stream) {
  if (!batch_ok(cache, batch) || !heads_ok(cache, q_heads) || !(scale > 0.0f) || !std::isfinite(scale))
    return EQ_EINVAL;
  if (TREE && batch->max_new > kMaxNodes) return EQ_EINVAL;
  if (batch->n_seqs == 0 || batch->max_new == 0) return EQ_OK;
  if (!q || !out || ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & 15) ||
      q_stride % 8 || (batch->n_tokens > 1 && q_stride < uint64_t(q_heads) * cache->head_dim))
    return EQ_EINVAL;
  if (TREE && (!mask || (window && !positions))) return EQ_EINVAL;
  const uint32_t group = q_heads / cache->kv_heads;
  if (!size_ok(cache, batch, q_heads, TREE)) return EQ_EINVAL;
  const Plan p = plan_attn(batch->n_seqs, cache->kv_heads, group, batch->max_new, batch->max_len,
                           window, TREE);
  const size_t need = attn_bytes<TREE>(p, cache, batch);
  if (need && (!ws || ws_bytes < need || (reinterpret_cast<uintptr_t>(ws) & 15))) return EQ_EINVAL;
  AttnArgs a{view(cache, batch), q, q_stride, out, static_cast<float *>(ws), nullptr, group, window,
             p.q_tiles, p.chunks, p.chunk_tiles, scale * 1.44269504088896340736f, mask, positions,
             (batch->max_new + 31) / 32, nullptr};
  if (need)
    a.stat = reinterpret_cast<float2 *>(a.part + part_cols(p, cache, batch) * cache->head_dim);
  if (TREE && need && p.prompt && batch->n_seqs <= kShareSeqs)
    a.even = reinterpret_cast<uint32_t *>(a.stat + part_cols(p, cache, batch));
  dim3 grid(cache->kv_heads * p.q_tiles * p.chunks, batch->n_seqs);
  if (a.even)  // each sequence's last chunks beside what runs at once, and a rounding
    grid = dim3(cache->kv_heads * std::min(head_blocks(cache->kv_heads) + batch->n_seqs * p.q_tiles + 1,
                                           batch->n_seqs * p.q_tiles * p.chunks));
  const dim3 join(batch->max_new * q_heads, batch->n_seqs);
  // a tile in one page has one page number to read and take addresses from (284 000
  // tokens: 61.9 us, as four 62.8)
  const bool one_page = cache->page_tokens >= kTile;
  const bool pair = pair_columns(batch->max_new, group);
  const bool stream_codes = stream_cache(p, batch->n_seqs, cache->kv_heads, cache->head_dim,
                                         batch->max_new, batch->max_len, window);
  if (cache->head_dim == 128)
    launch_attn<128, TREE>(a, p, pair, one_page, stream_codes, grid, join, stream);
  else
    launch_attn<64, TREE>(a, p, pair, one_page, stream_codes, grid, join, stream);
  return hipGetLastError() == hipSuccess ? EQ_OK : EQ_EHIP;
}

}  // namespace

extern "C" size_t eq_attn_kv4_workspace_bytes(const eq_kv_cache *cache, const eq_kv_batch *batch,
                                              uint32_t q_heads) {
  return workspace_bytes<false>(cache, batch, q_heads);
}

extern "C" int eq_attn_kv4(const eq_kv_cache *cache, const eq_kv_batch *batch, const uint16_t *q,
                           uint64_t q_stride, uint32_t q_heads, float scale, uint32_t window,
                           uint16_t *out, void *ws, size_t ws_bytes, hipStream_t stream) {
  return attention<false>(cache, batch, q, q_stride, q_heads, scale, window, nullptr, nullptr, out, ws,
                          ws_bytes, stream);
}

extern "C" size_t eq_attn_kv4_tree_workspace_bytes(const eq_kv_cache *cache, const eq_kv_batch *batch,
                                                   uint32_t q_heads) {
  return batch && batch->max_new > kMaxNodes ? 0 : workspace_bytes<true>(cache, batch, q_heads);
}

extern "C" int eq_attn_kv4_tree(const eq_kv_cache *cache, const eq_kv_batch *batch, const uint16_t *q,
                                uint64_t q_stride, uint32_t q_heads, float scale, uint32_t window,
                                const uint32_t *mask, const int32_t *positions, uint16_t *out, void *ws,
                                size_t ws_bytes, hipStream_t stream) {
  return attention<true>(cache, batch, q, q_stride, q_heads, scale, window, mask, positions, out, ws,
                         ws_bytes, stream);
}
