// Drafted trees (declared in include/eq.h): their masks and positions, and the
// verification of drafted tokens against the target's distributions.
//
// Verification.  p and q are the softmax of a target's and a draft's logits.  With
// r_0 = p, the children x_1, x_2, .. of a node are tested in order: x_j is accepted
// with probability min(1, r(x_j) / q(x_j)), else r becomes max(r - q, 0) and q loses
// x_j, both normalised again.  All of that is one family of functions,
//   r ~ max(p - t q, 0),  G(t) = sum max(p - t q, 0),  Q = sum of the q not rejected,
// from t = 0 (G = 1, Q = 1), with t + G / Q in the place of t after a rejection:
//   max(p - t q, 0) / G - q / Q = (max(p - t q, 0) - (G / Q) q) / G.
// A rejected x has p(x) < t q(x) from then on, so that q need not be cut there.  x is
// accepted when u G q(x) < max(p(x) - t q(x), 0) Q.  A rejection thus costs one pass
// over the vocabulary for G, and for Q where another child is there.  (Q is no 1 - q: a
// draft that is sure of a token leaves 2^-40 and less, of which the difference, off by
// 2^-38, holds nothing; and a target that rejects the token comes here often.)
//
// Everything is in 64 bits.  A token is where a running sum of probabilities passes u
// times the whole: the sum's error, over the probabilities near it, is how often a
// rounding would decide, 2^-24 times thousands of tokens in 32 bits.  What is left of p
// after rejections is a difference: probabilities are right to 2^-37.8, sums of it to
// about 2^-35 of the whole, and a border to 2^-35 / G.  64-bit vector
// instructions issue at half to two thirds the rate of 32-bit ones here (a fused
// multiply-add 6.3 cycles a wavefront against 3.3), and an exponential is 14 to 17.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "eq.h"
#include "eq_device.h"

namespace {

typedef int int2v __attribute__((ext_vector_type(2)));

constexpr uint32_t kMaxNodes = EQ_TREE_NODES;
constexpr uint32_t kChunk = 1024;  // logits a wavefront takes at a time
constexpr uint32_t kMaxVocab = 1u << 24;

// A sequence's rows [row, row + count), n of them by seq_start, as the batch bounds them.
struct Rows {
  int32_t row, count, n;
};

struct BatchArgs {
  const int32_t *seq_start, *kv_len;
  uint32_t n_seqs, n_tokens, max_new;
};

__device__ inline Rows rows_of(const BatchArgs &b, uint32_t s) {
  const int32_t row = int32_t(eq_dev::as_const(b.seq_start)[s]);
  const int32_t end = int32_t(eq_dev::as_const(b.seq_start)[s + 1]);
  Rows r{row, 0, 0};
  if (row < 0 || end <= row || uint32_t(row) >= b.n_tokens) return r;
  r.n = end - row;
  r.count = min(min(r.n, int32_t(b.max_new)), int32_t(b.n_tokens) - row);
  return r;
}

// ---------------------------------------------------------------- tree masks

struct MaskArgs {
  BatchArgs b;
  const int32_t *parents;
  uint32_t *mask;
  int32_t *positions;
  uint32_t window, words;
};

// A block for a sequence, a thread for a node, which walks up through the parents in
// LDS: as many steps as the node is deep.  64 trees of up to 60 nodes 3.7 us, one launch
// and its chain of loads.
__global__ __launch_bounds__(kMaxNodes) void tree_mask_kernel(MaskArgs a) {
  __shared__ int32_t up[kMaxNodes];
  const uint32_t s = blockIdx.x, i = threadIdx.x;
  const Rows r = rows_of(a.b, s);
  const int32_t len = a.b.kv_len[s];
  if (r.count <= 0 || len < 0) return;
  const bool on = int32_t(i) < r.count;
  int32_t p = on ? a.parents[r.row + int32_t(i)] : -1;
  if (p < -1 || p >= int32_t(i)) p = -2;  // hangs on nothing
  up[i] = p;
  __syncthreads();
  if (!on) return;
  uint32_t bits[kMaxNodes / 32] = {};
  int32_t depth = -1;
  int32_t j = int32_t(i);
  while (j >= 0) {
    ++depth;
    if (a.window == 0 || uint32_t(depth) < a.window) {
#pragma unroll
      for (uint32_t w = 0; w < kMaxNodes / 32; ++w)
        bits[w] |= uint32_t(j) >> 5 == w ? 1u << (j & 31) : 0u;
    }
    j = up[j];
  }
  const bool node = j == -1;
  uint32_t *const out = a.mask + uint64_t(r.row + int32_t(i)) * a.words;
#pragma unroll
  for (uint32_t w = 0; w < kMaxNodes / 32; ++w)
    if (w < a.words) out[w] = node ? bits[w] : 0u;
  a.positions[r.row + int32_t(i)] = node ? len - r.n + depth : -1;
}

// -------------------------------------------------------------- verification

// Of a chunk or a few: the sum of exp((x - max) / T), max being the largest logit or one
// near it (at temperature 0 the largest, and no sum); the first place of the largest (at
// temperature 0, else any), -1 where there is a NaN or +infinity.
struct Part {
  double sum;
  float max;
  int32_t arg;
};

// A row's distribution: exp((x - max) / T) inv, with max as above; best: its first largest
// logit (at temperature 0, else any token), or -1 where the row has no distribution.
struct Stat {
  double inv;
  float max;
  int32_t best;
};

// Where a sequence's walk stands: at node `cur`, whose children before `child` have been
// rejected.
struct State {
  double t, mass, left;  // mass: G(t), or what the rejected points have left of p; left: Q
  uint32_t cur, child, kept;
  uint32_t waits;        // for the sums of max(p - t q, 0): 1; of the q too: 2
  uint32_t out;          // different tokens among the rejected children of `cur`
  int32_t token;         // the last of them
};

// A node's place among the others.
struct Link {
  uint16_t first, next;  // its first child, the next child of its parent; kNone
  uint32_t again;        // an earlier child of its parent has the same token
};
constexpr uint32_t kNone = 0xFFFF;

constexpr double kLeast = 0x1p-32;  // of p: less is taken for nothing
// Of q: with less left no further child is tested.  Above it no product here leaves the
// range of numbers, nor does a q that counts; the token is then of what is left of p,
// which is the target's distribution whatever was not tested.
constexpr double kLeastDraft = 0x1p-900;
constexpr uint32_t kRounds = 4;
constexpr uint32_t kLocalChunks = 1024;  // chunks whose sums a block keeps in LDS
constexpr uint32_t kStatWaves = 3 * 1024, kMostPer = 3;  // (three for each SIMD)

struct VerifyArgs {
  BatchArgs b;
  const int32_t *parents, *tokens;
  const void *target, *draft;
  uint64_t target_stride, draft_stride;
  const float *temperature, *random;
  int32_t *path, *kept, *next;
  // workspace
  Part *part;                      // [n_tokens][chunks], of the target's rows
  Part *target_group, *draft_group;  // [n_tokens][groups], `per` chunks of 4 wavefronts each
  double *sums[2];                 // [n_seqs][2][chunks], of even and odd passes: of
                                   // max(p - t q, 0), and of the q not rejected
  double *rest;                    // [n_seqs][chunks], where those are more than kLocalChunks
  double *px, *qx;                 // [n_tokens]
  Stat *target_stat, *draft_stat;  // [n_tokens]
  Link *link;                      // [n_tokens]
  State *state[2];                 // [n_seqs], behind even and odd passes
  uint32_t vocab, chunks, per, groups;
  bool replace;
};

// 2^f for |f| <= 1/2: the polynomial that meets it at 0 and at the 8 Chebyshev points,
// 2^-38.8 relative.
__device__ inline double exp2_near(double f) {
  double z = 1.325080551750225e-06;
  z = __builtin_fma(z, f, 1.5303700711365693e-05);
  z = __builtin_fma(z, f, 0.00015403475186530786);
  z = __builtin_fma(z, f, 0.0013333478473685416);
  z = __builtin_fma(z, f, 0.00961812913523614);
  z = __builtin_fma(z, f, 0.055504109063258665);
  z = __builtin_fma(z, f, 0.24022650695888503);
  z = __builtin_fma(z, f, 0.6931471805568324);
  return __builtin_fma(z, f, 1.0);
}

// exp(d / T) for d up to 0 or not far above, c = log2 e / T; 0 far down (and for
// -infinity, also times 0, and for NaN).
__device__ inline double exp_down(double d, double c) {
  const double y = fmax(d * c, -1100.0), z = y + 0x1.8p52;  // y rounded, in the low bits
  return __builtin_ldexp(exp2_near(y - (z - 0x1.8p52)), int(__builtin_bit_cast(uint64_t, z)));
}

// exp((x - ref) / T) of logits near ref, but for a common factor, `shift`: in 13 64-bit
// instructions and an integer one, where exp_down has 17.  With K = ref c rounded, adding
// 3 2^51 - K to x c leaves it rounded, with the exponent that is wanted in the low bits.
// For x in [low, high], where that exponent stays in range; fast: ref c is not so large
// that its own rounding would show.
struct Power {
  double c, add, shift;  // shift: 2^(K - ref c)
  float ref, low, high;
  bool fast;
  __device__ inline Power(float r, double per_temp, double temp) : c(per_temp), ref(r) {
    const double top = double(r) * c, k = __builtin_rint(top), far = 0.6931471805599453 * temp;
    fast = c >= 0x1p-100 && fabs(top) <= 4096.0;
    add = 0x1.8p52 - k;
    shift = fast ? exp2_near(-__builtin_fma(double(r), c, -k)) : 1.0;
    low = fast ? float((k - 900.0) * far) : INFINITY;
    high = fast ? float((k + 500.0) * far) : NAN;  // (nothing is below that)
  }
  __device__ inline double operator()(float x) const {
    const double d = double(x), z = __builtin_fma(d, c, add);
    const double y = exp2_near(__builtin_fma(d, c, -(z - add)));
    int2v u = __builtin_bit_cast(int2v, y);
    u[1] += __builtin_bit_cast(int2v, z)[0] << 20;
    return __builtin_bit_cast(double, u);
  }
};

// The next N of 16 values to the front.  Loops over a few at a time stay loops by it:
// unrolled, the exponentials of a chunk are 10 KB of code that a wavefront runs through
// once, and fetching that took longer than the rest (128 chunks of 32 rows, two logits
// each: 21 us, as a loop 8).
template <int N>
__device__ inline void next(float (&x)[16]) {
#pragma unroll
  for (int i = 0; i < 16 - N; ++i) x[i] = x[i + N];
}

template <typename T>
__device__ inline float logit(const T *row, uint32_t i) {
  if constexpr (sizeof(T) == 4) return row[i];
  else return eq_dev::bf16_to_f32(row[i]);
}

// A lane's 16 logits of a chunk, four in a row: number `first + step i + e` is element 4 i
// + e, with first = 4 lane and step = 256, or 16 lane and 4.  Rows start at any element.
// In two parts, so that loads stay in flight: what was loaded, and its values.  (A load
// under a condition would be waited for where the branches meet: fours that reach
// behind the vocabulary are read before its end and moved up.)
template <typename T>
struct Raw {
  T v[4][4];
};
template <typename T>
__device__ inline Raw<T> load16(const T *row, uint32_t vocab, uint32_t first, uint32_t step) {
  Raw<T> r;
  if (vocab >= 4) {
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i)
      __builtin_memcpy(r.v[i], row + min(first + step * i, vocab - 4), sizeof(r.v[i]));
  } else {
    T v[3];
#pragma unroll
    for (uint32_t e = 0; e < 3; ++e) v[e] = row[min(e, vocab - 1)];
#pragma unroll
    for (uint32_t i = 0; i < 16; ++i) r.v[i / 4][i % 4] = v[min(i % 4, 2u)];
  }
  return r;
}
// cut: some are behind the vocabulary, and become -infinity.
template <typename T>
__device__ inline void values(const Raw<T> &r, uint32_t vocab, uint32_t first, uint32_t step, bool cut,
                              float (&x)[16]) {
#pragma unroll
  for (uint32_t i = 0; i < 16; ++i) x[i] = logit(r.v[i / 4], i % 4);
  if (!cut) return;
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    const uint32_t at = first + step * i, up = vocab >= 4 ? at - min(at, vocab - 4) : 0;
    float *const y = x + 4 * i;
    if (up & 1) y[0] = y[1], y[1] = y[2], y[2] = y[3];
    if (up & 2) y[0] = y[2], y[1] = y[3];
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) y[e] = at + e < vocab ? y[e] : -INFINITY;
  }
}

// v of the lane that CTRL names, `none` where there is none or the row is not in ROWS.
template <int CTRL, int ROWS>
__device__ inline float from_lane(float v, float none) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(none), __float_as_int(v), CTRL,
                                                    ROWS, 0xF, false));
}
template <int CTRL, int ROWS>
__device__ inline double from_lane(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = uint32_t(__builtin_amdgcn_update_dpp(0, int(uint32_t(u)), CTRL, ROWS, 0xF, true));
  const uint32_t hi = uint32_t(__builtin_amdgcn_update_dpp(0, int(uint32_t(u >> 32)), CTRL, ROWS, 0xF, true));
  return __builtin_bit_cast(double, uint64_t(hi) << 32 | lo);
}
__device__ inline double lane_value(double v, int lane) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = uint32_t(__builtin_amdgcn_readlane(int(uint32_t(u)), lane));
  const uint32_t hi = uint32_t(__builtin_amdgcn_readlane(int(uint32_t(u >> 32)), lane));
  return __builtin_bit_cast(double, uint64_t(hi) << 32 | lo);
}

// Sums of the lanes up to each: within rows of 16, then from row to row.
__device__ inline double wave_scan(double v) {
  v += from_lane<0x111, 0xF>(v);
  v += from_lane<0x112, 0xF>(v);
  v += from_lane<0x114, 0xF>(v);
  v += from_lane<0x118, 0xF>(v);
  v += from_lane<0x142, 0xA>(v);  // row_bcast:15
  v += from_lane<0x143, 0xC>(v);  // row_bcast:31
  return v;
}
__device__ inline double wave_sum(double v) { return lane_value(wave_scan(v), 63); }

__device__ inline float wave_max(float v) {
  v = fmaxf(v, from_lane<0x111, 0xF>(v, -INFINITY));
  v = fmaxf(v, from_lane<0x112, 0xF>(v, -INFINITY));
  v = fmaxf(v, from_lane<0x114, 0xF>(v, -INFINITY));
  v = fmaxf(v, from_lane<0x118, 0xF>(v, -INFINITY));
  v = fmaxf(v, from_lane<0x142, 0xA>(v, -INFINITY));
  v = fmaxf(v, from_lane<0x143, 0xC>(v, -INFINITY));
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

__device__ inline float temperature_of(const VerifyArgs &a, uint32_t s) {
  return a.temperature ? __uint_as_float(eq_dev::as_const(a.temperature)[s]) : 1.0f;
}
__device__ inline double per_temperature(float temp) {
  return temp > 0.0f ? 1.4426950408889634 / double(temp) : 0.0;
}

// A chunk's first largest logit.
__device__ inline Part largest(const float (&x)[16], uint32_t chunk, float top) {
  bool bad = false;
  int32_t arg = -1;
#pragma unroll
  for (int i = 3; i >= 0; --i) {
    uint32_t mine = 4;  // the first of four that is the largest
#pragma unroll
    for (int e = 3; e >= 0; --e) {
      bad = bad || !(x[4 * i + e] < INFINITY);
      mine = x[4 * i + e] == top ? e : mine;
    }
    const uint64_t m = __ballot(mine < 4);
    if (m) {
      const int l = __ffsll((unsigned long long)m) - 1;
      arg = int32_t(chunk * kChunk) + 256 * i + 4 * l + __builtin_amdgcn_readlane(int(mine), l);
    }
  }
  return Part{0.0, top, __any(bad) ? -1 : arg};
}

// The statistics of a row's chunks, `per` of them for a wavefront, one's loads in flight
// beside another's exponentials, and of the block's chunks together.  Draft rows of nodes
// without children are left out.
//
// A wavefront's first chunk sets the reference of its exponentials, and others keep it
// while they are near: a chunk then has no maximum to agree on first.  A NaN comes out in
// the sum.  Chunks with far or infinite logits take exp_down.  Between memory and the
// 64-bit instructions: 192 rows of 131072 logits and the draft's in BF16, 128 MB in 33.5
// us, 3.8 TB/s (a copy: 5.2); without exponentials 21 us for 100 MB.  One chunk a
// wavefront 38 us, eight 40; 4 wavefronts a SIMD 35, 6 and more spill (37 and up).
template <typename T>
__device__ __forceinline__ void row_stats(const T *row, uint32_t vocab, uint32_t chunk, uint32_t end,
                                          uint32_t lane, float temp, double per_temp, Part *out) {
  const bool greedy = !(temp > 0.0f);
  auto load = [&](uint32_t c) { return load16(row, vocab, c * kChunk + 4 * lane, 256); };
  Power power(INFINITY, per_temp, double(temp));  // (near nothing)
  Raw<T> raw;
  if (chunk < end) raw = load(chunk);
#pragma unroll 1
  for (; chunk < end; ++chunk, ++out) {
    float x[16];
    values(raw, vocab, chunk * kChunk + 4 * lane, 256, (chunk + 1) * kChunk > vocab, x);
    raw = load(min(chunk + 1, end - 1));
    float high = x[0], low = x[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) high = fmaxf(high, x[e]), low = fminf(low, x[e]);
    if (greedy) {
      const Part p = largest(x, chunk, wave_max(high));
      if (lane == 0) *out = p;
      continue;
    }
    if (!__all(high <= power.high)) power = Power(wave_max(high), per_temp, double(temp));
    double sum = 0.0;
    bool bad = false;
    if (power.fast && __all(low >= power.low)) {
#pragma unroll 1
      for (int i = 0; i < 16; i += 8, next<8>(x)) {
#pragma unroll
        for (int h = 0; h < 8; h += 4) {
          sum += (power(x[h]) + power(x[h + 1])) + (power(x[h + 2]) + power(x[h + 3]));
          __builtin_amdgcn_sched_barrier(0);  // (eight side by side would take 130 registers)
        }
      }
      sum = wave_sum(sum) * power.shift;
      bad = sum != sum;
    } else {  // (of -infinity alone: 0)
#pragma unroll 1
      for (int i = 0; i < 16; i += 4, next<4>(x)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          bad = bad || !(x[e] < INFINITY);
          sum += exp_down(double(x[e]) - double(power.ref), per_temp);
        }
      }
      sum = wave_sum(sum);
      bad = __any(bad);
    }
    if (lane == 0) *out = Part{sum, power.ref, bad ? -1 : int32_t(chunk * kChunk)};
  }
}

// Statistics of parts, a lane's each, in all lanes: the largest, its first place, and the
// sum of exp((x - max) / T).
__device__ inline Part join_lanes(Part p, bool on, double per_temp) {
  const bool bad = __any(on && p.arg < 0);
  const float top = wave_max(on ? p.max : -INFINITY);
  const uint64_t m = __ballot(on && p.max == top);
  const int32_t arg = m ? __builtin_amdgcn_readlane(p.arg, __ffsll((unsigned long long)m) - 1) : -1;
  const double sum = on && p.max > -INFINITY ? p.sum * exp_down(double(p.max) - double(top), per_temp) : 0.0;
  return Part{wave_sum(sum), top, bad ? -1 : arg};
}

template <typename TT, typename TD>
__global__ __launch_bounds__(256, 5) void row_stats_kernel(VerifyArgs a) {
  __shared__ Part parts[4 * kMostPer];
  const uint32_t s = blockIdx.z, i = blockIdx.y;
  const bool drafted = blockIdx.x >= a.groups;
  const Rows r = rows_of(a.b, s);
  if (int32_t(i) >= r.count) return;
  const float temp = temperature_of(a, s);
  if (drafted) {
    if (!(temp > 0.0f)) return;
    const int32_t j = int32_t(threadIdx.x);
    if (!__syncthreads_or(j > int32_t(i) && j < r.count && a.parents[r.row + j] == int32_t(i))) return;
  }
  const uint32_t lane = threadIdx.x & 63, wave = eq_dev::uniform(threadIdx.x >> 6);
  const uint32_t group = blockIdx.x - (drafted ? a.groups : 0), first = group * 4 * a.per;
  const uint32_t chunk = first + wave * a.per, end = min(chunk + a.per, a.chunks);
  const uint64_t row = uint64_t(r.row) + i;
  const double per_temp = per_temperature(temp);
  Part *const out = parts + wave * a.per;
  const TT *const target = static_cast<const TT *>(a.target) + row * a.target_stride;
  const TD *const draft = static_cast<const TD *>(a.draft) + row * a.draft_stride;
  if constexpr (std::is_same<TT, TD>::value)
    row_stats(drafted ? draft : target, a.vocab, chunk, end, lane, temp, per_temp, out);
  else if (drafted)
    row_stats(draft, a.vocab, chunk, end, lane, temp, per_temp, out);
  else
    row_stats(target, a.vocab, chunk, end, lane, temp, per_temp, out);
  __syncthreads();
  if (wave) return;
  const bool on = lane < min(4 * a.per, a.chunks - first);
  const Part p = parts[on ? lane : 0];
  if (!drafted && on) a.part[row * a.chunks + first + lane] = p;
  const Part all = join_lanes(p, on, per_temp);
  if (lane == 0) (drafted ? a.draft_group : a.target_group)[row * a.groups + group] = all;
}

// A row's statistics from its groups', by `lanes` neighbouring lanes: the same in all.
__device__ inline Stat join_groups(const Part *part, uint32_t groups, uint32_t lane, uint32_t lanes,
                                   double per_temp) {
  float top = -INFINITY;
  int32_t arg = 0x7FFFFFFF;
  bool bad = false;
  double sum = 0.0;
#pragma unroll 1
  for (uint32_t c0 = 0; c0 < groups; c0 += 8 * lanes) {
    Part p[8];
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) p[j] = part[min(c0 + lanes * j + lane, groups - 1)];
    float high = top;
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) {
      bad = bad || p[j].arg < 0;
      if (p[j].max > high || arg == 0x7FFFFFFF) high = p[j].max, arg = p[j].arg;
    }
    if (high > -INFINITY) {
      sum *= exp_down(double(top) - double(high), per_temp);
#pragma unroll 1
      for (uint32_t c = c0 + lane; c < min(groups, c0 + 8 * lanes); c += lanes) {
        sum += p[0].sum * exp_down(double(p[0].max) - double(high), per_temp);
#pragma unroll
        for (uint32_t j = 0; j < 7; ++j) p[j].sum = p[j + 1].sum, p[j].max = p[j + 1].max;
      }
    }
    top = high;
  }
  float all = top;
#pragma unroll 1
  for (uint32_t d = 1; d < lanes; d *= 2) {
    const float m = __shfl_xor(all, int(d));
    const int32_t j = __shfl_xor(arg, int(d)), b = __shfl_xor(int(bad), int(d));
    bad = bad || b;
    if (m > all || (m == all && j < arg)) all = m, arg = j;
  }
  sum = top > -INFINITY ? sum * exp_down(double(top) - double(all), per_temp) : 0.0;
#pragma unroll 1
  for (uint32_t d = 1; d < lanes; d *= 2) sum += __shfl_xor(sum, int(d));
  return Stat{1.0 / sum, all, bad || all == -INFINITY ? -1 : arg};
}

struct Node {
  int32_t up, token;  // up: -2 for what hangs on nothing
  float random;
};

// What a block holds of a sequence's tree.
struct Tree {
  Stat target[kMaxNodes], draft[kMaxNodes];
  double px[kMaxNodes], qx[kMaxNodes];  // p and q of a node's token at its parent
  float random[kMaxNodes];
  int32_t up[kMaxNodes], token[kMaxNodes];
  Link link[kMaxNodes];
  uint32_t hidden[kChunk / 32];
  double weight[16][64];  // of a chunk's tokens, 16 a lane; or the chunks' sums
  __device__ inline void put(uint32_t i, const Node &n) {
    up[i] = n.up, token[i] = n.token, random[i] = n.random;
    link[i] = Link{kNone, kNone, 0};
  }
};

// A sequence's node; behind the last one, none.
__device__ inline Node load_node(const VerifyArgs &a, const Rows &r, uint32_t i) {
  const bool on = int32_t(i) < r.count;
  const int32_t row = r.row + int32_t(on ? i : 0);
  const int32_t p = a.parents[row];
  return Node{on && i > 0 && p >= 0 && p < int32_t(i) ? p : -2, a.tokens[row], a.random[row]};
}

// The nodes' links: a wavefront takes every `waves`-th node and finds its children, whose
// parents its lanes hold, by a ballot.
__device__ inline void link_tree(Tree &tree, uint32_t count, uint32_t wave, uint32_t waves, uint32_t lane) {
  constexpr uint32_t kSets = kMaxNodes / 64;
  const uint32_t sets = (count + 63) / 64;
  int32_t up[kSets], token[kSets];
#pragma unroll
  for (uint32_t b = 0; b < kSets; ++b) {
    up[b] = b < sets ? tree.up[64 * b + lane] : -2;
    token[b] = b < sets ? tree.token[64 * b + lane] : 0;
  }
#pragma unroll 1
  for (uint32_t i = wave; i < count; i += waves) {
    uint64_t kids[kSets];
    uint32_t behind = kNone;  // the first child of the sets behind
#pragma unroll
    for (uint32_t b = kSets; b-- > 0;) {
      const bool mine = up[b] == int32_t(i);
      kids[b] = b < sets ? __ballot(mine) : 0;
      if (!kids[b]) continue;
      const uint64_t later = kids[b] & ~((uint64_t(2) << lane) - 1);
      if (mine)
        tree.link[64 * b + lane].next =
            uint16_t(later ? 64 * b + uint32_t(__ffsll((unsigned long long)later)) - 1 : behind);
      behind = 64 * b + uint32_t(__ffsll((unsigned long long)kids[b])) - 1;
    }
    if (lane == 0) tree.link[i].first = uint16_t(behind);
#pragma unroll
    for (uint32_t b = 0; b < kSets; ++b) {
      for (uint64_t left = kids[b]; left; left &= left - 1) {
        const uint32_t c = uint32_t(__ffsll((unsigned long long)left)) - 1;
        const int32_t t = __builtin_amdgcn_readlane(token[b], int(c));
#pragma unroll
        for (uint32_t d = b; d < kSets; ++d)
          if (up[d] == int32_t(i) && token[d] == t && (d > b || lane > c)) tree.link[64 * d + lane].again = 1;
      }
    }
  }
}

// A wavefront's walk through a tree.
template <typename TT, typename TD, bool POINTS>
struct Walk {
  const VerifyArgs &a;
  Tree &tree;
  Rows r;
  uint32_t s, count, lane;
  bool greedy, writes;  // writes: the one of a sequence's blocks that does
  double per_temp;
  double *sums;
  State st;

  __device__ inline Walk(const VerifyArgs &args, Tree &t, uint32_t seq, const Rows &rows, bool writer,
                         double *chunk_sums)
      : a(args), tree(t), r(rows), s(seq), count(uint32_t(rows.count)), lane(threadIdx.x & 63),
        writes(writer), sums(POINTS ? nullptr : chunk_sums + 2 * uint64_t(seq) * args.chunks) {
    const float temp = temperature_of(a, s);
    greedy = !(temp > 0.0f);
    per_temp = per_temperature(temp);
  }

  __device__ inline const TT *target_row(uint32_t i) const {
    return static_cast<const TT *>(a.target) + (uint64_t(r.row) + i) * a.target_stride;
  }
  __device__ inline const TD *draft_row(uint32_t i) const {
    return static_cast<const TD *>(a.draft) + (uint64_t(r.row) + i) * a.draft_stride;
  }
  __device__ inline double prob(const Stat &v, float x) const {
    return exp_down(double(x) - double(v.max), per_temp) * v.inv;
  }
  __device__ inline double random_of(uint32_t i) const {
    return double(fminf(fmaxf(tree.random[i], 0.0f), 0.99999994f));  // (NaN: 0)
  }
  __device__ inline bool outside(uint32_t i) const { return uint32_t(tree.token[i]) >= a.vocab; }

  __device__ inline void stand_at(uint32_t node) {
    st.cur = node, st.child = tree.link[node].first;
    st.t = 0.0, st.mass = 1.0, st.left = 1.0;
    st.out = 0, st.token = 0;
  }
  __device__ inline void go_down(uint32_t c) {
    if (writes && lane == 0) a.path[r.row + int32_t(st.kept)] = int32_t(c);
    ++st.kept;
    stand_at(c);
  }

  // 16 logits of the node's target and, where it counts, its draft
  __device__ __forceinline__ void load(uint32_t first, uint32_t step, bool cut, float (&p)[16],
                                       float (&q)[16]) const {
    const Raw<TT> rp = load16(target_row(st.cur), a.vocab, first, step);
    if constexpr (!POINTS) {
      if (st.t > 0.0) values(load16(draft_row(st.cur), a.vocab, first, step), a.vocab, first, step, cut, q);
    }
    values(rp, a.vocab, first, step, cut, p);
  }

  // The weights max(p - t q, 0) of 16 tokens, four at a time: put(i, w).
  template <typename F>
  __device__ inline void weights(float (&p)[16], float (&q)[16], F &&put) const {
    const Stat ps = tree.target[st.cur], qs = POINTS ? ps : tree.draft[st.cur];
    const bool less = !POINTS && st.t > 0.0;
#pragma unroll 1
    for (int i = 0; i < 4; ++i, next<4>(p), next<4>(q)) {
      double w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = prob(ps, p[e]);
      if (less) {
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = fmax(__builtin_fma(-st.t, prob(qs, q[e]), w[e]), 0.0);
      }
      put(i, w);
    }
  }

  // the sum of a chunk's weights without the tokens in tree.hidden
  __device__ __forceinline__ double chunk_sum(uint32_t chunk) const {
    float p[16], q[16] = {};
    load(chunk * kChunk + 4 * lane, 256, (chunk + 1) * kChunk > a.vocab, p, q);
    double sum = 0.0;
    weights(p, q, [&](int i, double (&w)[4]) {
      const uint32_t at = 256 * uint32_t(i) + 4 * lane, bits = tree.hidden[at / 32] >> (at % 32);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = bits >> e & 1 ? 0.0 : w[e];
      sum += (w[0] + w[1]) + (w[2] + w[3]);
    });
    return wave_sum(sum);
  }

  // Which of a lane's 16 tokens of a chunk (as load16's, with step 256) are rejected
  // children's.  One of them is known without the tree.
  __device__ inline uint32_t rejected(uint32_t chunk) const {
    const auto bit = [&](uint32_t token) {
      const uint32_t at = token % kChunk;
      return at % 256 / 4 == lane ? 1u << (at / 256 * 4 + at % 4) : 0u;
    };
    if (st.out == 1) return uint32_t(st.token) / kChunk == chunk ? bit(uint32_t(st.token)) : 0u;
    uint32_t bits = 0;
#pragma unroll 1
    for (uint32_t j0 = 0; j0 < st.child; j0 += 64) {
      const uint32_t j = j0 + lane;
      uint64_t m = __ballot(j < st.child && gone(j) && chunk_of(j) == chunk);
      for (; m; m &= m - 1) bits |= bit(uint32_t(tree.token[j0 + uint32_t(__ffsll((unsigned long long)m)) - 1]));
    }
    return bits;
  }

  // The sums that the walk waits for, of a chunk.
  __device__ __forceinline__ void pass(uint32_t chunk, double *out) const {
    const bool both = st.waits > 1;
    const uint32_t without = both ? rejected(chunk) : 0;
    float p[16], q[16] = {};
    load(chunk * kChunk + 4 * lane, 256, (chunk + 1) * kChunk > a.vocab, p, q);
    const Stat ps = tree.target[st.cur], qs = tree.draft[st.cur];
    double sum = 0.0, rest = 0.0;
#pragma unroll 1
    for (int i = 0; i < 4; ++i, next<4>(p), next<4>(q)) {
      double w[4], v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = prob(qs, q[e]);
        w[e] = fmax(__builtin_fma(-st.t, v[e], prob(ps, p[e])), 0.0);
        v[e] = without >> (4 * i + e) & 1 ? 0.0 : v[e];
      }
      sum += (w[0] + w[1]) + (w[2] + w[3]);
      rest += (v[0] + v[1]) + (v[2] + v[3]);
    }
    sum = wave_sum(sum);
    if (lane == 0) out[chunk] = sum;
    if (!both) return;
    rest = wave_sum(rest);
    if (lane == 0) out[a.chunks + chunk] = rest;
  }

  // Tests children and goes down until sums are needed (what st.waits says) or the walk
  // has ended at `next` (0).
  __device__ __forceinline__ uint32_t walk(int32_t &next) {
    next = -1;
#pragma unroll 1
    while (true) {
      const Stat here = tree.target[st.cur];
      if (here.best < 0) return 0;
      uint32_t c = st.child;
      if (greedy) {
        while (c != kNone && tree.token[c] != here.best) c = tree.link[c].next;
        if (c == kNone) {
          next = here.best;
          return 0;
        }
        go_down(c);
        continue;
      }
      if (!POINTS && c != kNone && tree.draft[st.cur].best < 0) return 0;
      bool down = false;
#pragma unroll 1
      while (c != kNone && st.mass >= kLeast && st.left >= kLeastDraft) {
        const Link link = tree.link[c];
        const double u = random_of(c), p = tree.px[c], q = POINTS ? 0.0 : tree.qx[c];
        st.child = link.next;
        if (!outside(c)) {
          const double rest = link.again ? 0.0 : fmax(__builtin_fma(-st.t, q, p), 0.0);
          if (POINTS ? u * st.mass < rest : u * st.mass * q < rest * st.left) {
            down = true;
            break;
          }
          if constexpr (POINTS) {
            st.mass = fmax(st.mass - rest, 0.0);
          } else {
            st.t += st.mass / st.left;
            if (link.again) return 1;
            ++st.out, st.token = tree.token[c];
            return !a.replace && st.child != kNone ? 2 : 1;
          }
        }
        c = link.next;
      }
      if (!down) {
        if (writes) next = pick(here);
        return 0;
      }
      go_down(c);
    }
  }

  // Of 256 chunks' sums from c0 on, a lane's four (0 behind the last), in one wait.
  __device__ __forceinline__ void load4(const double *from, uint32_t c0, double (&v)[4]) const {
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) v[j] = from[min(c0 + 64 * j + lane, a.chunks - 1)];
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) v[j] = c0 + 64 * j + lane < a.chunks ? v[j] : 0.0;
  }
  // Theirs and all others' sum; v: the first 256's.
  __device__ __forceinline__ double total_of(const double *from, const double (&v)[4]) const {
    double sum = ((v[0] + v[1]) + v[2]) + v[3];
#pragma unroll 1
    for (uint32_t c0 = 256; c0 < a.chunks; c0 += 256) {
      double x[4];
      load4(from, c0, x);
      sum += ((x[0] + x[1]) + x[2]) + x[3];
    }
    return wave_sum(sum);
  }

  // The token behind the path: from what is left of p, or from p where nothing is.
  __device__ __forceinline__ int32_t pick(const Stat &here) {
    const uint32_t chunks = a.chunks;
    bool hidden = POINTS && st.child != tree.link[st.cur].first;
    if (!(st.mass >= kLeast)) st.t = 0.0, hidden = false;
    double *left = sums;  // of each chunk
    if (!(st.t > 0.0)) {
      const Part *const part = a.part + (uint64_t(r.row) + st.cur) * chunks;
      left = chunks <= kLocalChunks ? &tree.weight[0][0] : a.rest + uint64_t(s) * chunks;
#pragma unroll 1
      for (uint32_t c0 = lane; c0 < chunks; c0 += 256) {
        Part v[4];
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) v[j] = part[min(c0 + 64 * j, chunks - 1)];
#pragma unroll 1
        for (uint32_t c = c0; c < min(c0 + 256, chunks); c += 64) {
          left[c] = v[0].sum * exp_down(double(v[0].max) - double(here.max), per_temp) * here.inv;
#pragma unroll
          for (uint32_t j = 0; j < 3; ++j) v[j].sum = v[j + 1].sum, v[j].max = v[j + 1].max;
        }
      }
      __threadfence_block();
      if (hidden) take_out(left);
    }
    double v[4];
    load4(left, 0, v);
    const double limit = random_of(0) * total_of(left, v);
    // the first chunk whose running sum passes the limit
    double before = 0.0;
    uint32_t at = chunks;
#pragma unroll 1
    for (uint32_t c0 = 0; c0 < chunks; c0 += 64) {
      if (c0 && c0 % 256 == 0) load4(left, c0, v);
      const double run = wave_scan(v[0]);
      const uint64_t m = __ballot(before + run > limit && v[0] > 0.0);
      if (m) {
        const int l = __ffsll((unsigned long long)m) - 1;
        at = c0 + uint32_t(l);
        before += lane_value(run - v[0], l);
        break;
      }
      before += lane_value(run, 63);
#pragma unroll
      for (int j = 0; j < 3; ++j) v[j] = v[j + 1];
    }
    if (at >= chunks) return here.best;
    if (hidden) hide(at);
    // its weights, 16 in a row for a lane, and the lane in which the sum passes it
    float p[16], q[16] = {};
    const uint32_t first = at * kChunk + 16 * lane;
    load(first, 4, (at + 1) * kChunk > a.vocab, p, q);
    double sum = 0.0;
    weights(p, q, [&](int i, double (&w)[4]) {
      const uint32_t bits = hidden ? tree.hidden[lane / 2] >> (16 * (lane & 1) + 4 * i) : 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        w[e] = bits >> e & 1 ? 0.0 : w[e];
        tree.weight[4 * i + e][lane] = w[e];
        sum += w[e];
      }
    });
    __threadfence_block();
    const double run = before + wave_scan(sum);
    // (a rounding may leave the sum at the chunk's end just below the limit: then its
    // last token with a weight)
    uint64_t lanes = __ballot(run > limit && sum > 0.0);
    const bool passes = lanes != 0;
    if (!passes) lanes = __ballot(sum > 0.0);
    if (!lanes) return here.best;
    const int l = passes ? __ffsll((unsigned long long)lanes) - 1 : 63 - __clzll((long long)lanes);
    const double w = lane < 16 ? tree.weight[lane][l] : 0.0;
    const double run16 = lane_value(run - sum, l) + wave_scan(w);
    const uint64_t some = __ballot(w > 0.0), over = __ballot(w > 0.0 && run16 > limit);
    const int e = passes && over ? __ffsll((unsigned long long)over) - 1 : 63 - __clzll((long long)some);
    return int32_t(at * kChunk) + 16 * l + e;
  }

  // A child of `cur` with a token, the first of that token: a rejected one, among those
  // that have been tested.
  __device__ inline bool gone(uint32_t j) const {
    return j < count && tree.up[j] == int32_t(st.cur) && !outside(j) && !tree.link[j].again;
  }
  __device__ inline uint32_t chunk_of(uint32_t j) const { return uint32_t(tree.token[j]) / kChunk; }

  // Takes the rejected points out of the chunks' sums.  Where little of a chunk is left
  // its tokens are summed up again: the difference would be the sum's rounding.
  __device__ inline void take_out(double *left) {
#pragma unroll 1
    for (uint32_t j0 = 0; j0 < count; j0 += 64) {
      uint64_t todo = __ballot(gone(j0 + lane));
#pragma unroll 1
      while (todo) {
        const uint32_t chunk = chunk_of(j0 + uint32_t(__ffsll((unsigned long long)todo)) - 1);
        double out = 0.0;
        bool earlier = false;  // done with a node of an earlier 64
#pragma unroll 1
        for (uint32_t i0 = 0; i0 < count; i0 += 64) {
          const uint32_t i = i0 + lane;
          const bool same = gone(i) && chunk_of(i) == chunk;
          out += same ? tree.px[i] : 0.0;
          const uint64_t m = __ballot(same);
          if (i0 < j0 && m) earlier = true;
          if (i0 == j0) todo &= ~m;
        }
        if (earlier) continue;
        const double all = left[chunk];
        double rest = all - wave_sum(out);
        if (!(rest > all * 0x1p-20)) {
          hide(chunk);
          rest = chunk_sum(chunk);
        }
        if (lane == 0) left[chunk] = rest;
      }
    }
    __threadfence_block();
  }

  // a chunk's tokens among the rejected points, as bits
  __device__ inline void hide(uint32_t chunk) {
    if (lane < kChunk / 32) tree.hidden[lane] = 0;
    __threadfence_block();
    for (uint32_t j = lane; j < count; j += 64)
      if (gone(j) && chunk_of(j) == chunk)
        atomicOr(&tree.hidden[uint32_t(tree.token[j]) % kChunk / 32], 1u << (tree.token[j] & 31));
    __threadfence_block();
  }

  __device__ inline void finish(int32_t next) {
    if (!writes) return;
    for (uint32_t i = st.kept + lane; i < count; i += 64) a.path[r.row + int32_t(i)] = -1;
    if (lane == 0) a.kept[s] = int32_t(st.kept), a.next[s] = next;
  }
};

// The rows' statistics and the tokens' probabilities, then the walk up to the first
// rejection of a drawn token, or to its end.  All latency: 6 us for a chain of 5 rows, 12
// for 32 chains that are accepted whole and end in a token, about 0.5 us a node and 4 for
// the token.
//
// Of few chunks it goes to the walk's end, with passes of its own in place of
// pass_kernel's launches (5 us each, an idle one 1 to 2).  us of a call with launches /
// so, sequences x nodes (most children), chunks, means of 6 inputs:
//   8 x 16 (4), 8: 41.4 / 27.0   32 x 24 (4), 8: 56.4 / 40.2   32 x 6 (1), 8: 30.4 / 22.5
//   8 x 16 (4), 16: 40.2 / 33.7  32 x 24 (4), 16: 71.9 / 66.5  32 x 6 (1), 16: 32.3 / 27.5
//   8 x 16 (4), 32: 44.3 / 49.3  32 x 24 (4), 32: 78.2 / 95.9  32 x 6 (1), 32: 38.6 / 40.0
constexpr uint32_t kWalkThreads = 2 * kMaxNodes, kFewChunks = 16;
static_assert(kFewChunks <= 64);

template <typename TT, typename TD, bool POINTS>
__global__ __launch_bounds__(kWalkThreads) void walk_kernel(VerifyArgs a) {
  __shared__ Tree tree;
  __shared__ State state;
  __shared__ double sums[2 * kFewChunks];
  const uint32_t s = blockIdx.x, tid = threadIdx.x;
  const Rows r = rows_of(a.b, s);
  if (r.count <= 0) {
    if (tid == 0) {
      a.kept[s] = 0, a.next[s] = -1;
      if constexpr (!POINTS) a.state[0][s].waits = 0;
    }
    return;
  }
  Walk<TT, TD, POINTS> w(a, tree, s, r, true, a.sums[0]);
  const uint32_t count = w.count;
  // a node's logits: the target's by one half of the block, the draft's by the other
  const uint32_t node = tid % kMaxNodes;
  const bool of_draft = tid >= kMaxNodes;
  const Node me = load_node(a, r, node);
  const bool drawn = me.up >= 0 && uint32_t(me.token) < a.vocab && !w.greedy && !(POINTS && of_draft);
  float x = 0.0f;
  if (drawn) {
    if (!of_draft) x = logit(w.target_row(uint32_t(me.up)), uint32_t(me.token));
    else if constexpr (!POINTS) x = logit(w.draft_row(uint32_t(me.up)), uint32_t(me.token));
  }
  // (of draft rows without children: statistics of anything, that nothing looks at)
  const uint32_t rows = (POINTS || w.greedy ? 1 : 2) * count;
  uint32_t lanes = 64;
  while (lanes > 8 && rows * lanes > kWalkThreads) lanes /= 2;
#pragma unroll 1
  for (uint32_t k = tid / lanes; k < rows; k += kWalkThreads / lanes) {
    const bool drafted = k >= count;
    const uint32_t i = drafted ? k - count : k;
    const Stat st = join_groups((drafted ? a.draft_group : a.target_group) + (uint64_t(r.row) + i) * a.groups,
                                a.groups, tid % lanes, lanes, w.per_temp);
    if (tid % lanes == 0) (drafted ? tree.draft : tree.target)[i] = st;
  }
  if (!of_draft) tree.put(tid, me);
  __syncthreads();
  link_tree(tree, count, eq_dev::uniform(tid >> 6), kWalkThreads / 64, tid & 63);
  if (drawn) (of_draft ? tree.qx : tree.px)[node] = w.prob((of_draft ? tree.draft : tree.target)[me.up], x);
  __syncthreads();
  const bool few = a.chunks <= kFewChunks;
  if (!POINTS && !few && tid < count) {
    const uint64_t row = uint64_t(r.row) + tid;
    a.px[row] = tree.px[tid], a.qx[row] = tree.qx[tid];
    a.target_stat[row] = tree.target[tid], a.draft_stat[row] = tree.draft[tid];
    a.link[row] = tree.link[tid];
  }
  if (tid == 0) a.path[r.row] = 0;
  w.st.kept = 1;
  w.stand_at(0);
  const uint32_t wave = eq_dev::uniform(tid >> 6);
  if constexpr (!POINTS) {
    if (few) w.sums = sums;
  }
#pragma unroll 1
  while (true) {
    if (wave == 0) {
      int32_t next;
      w.st.waits = w.walk(next);
      if (!w.st.waits) w.finish(next);
      if (!POINTS && w.lane == 0) {
        if (few) state = w.st;
        else a.state[0][s] = w.st;
      }
    }
    if (POINTS || !few) return;
    __syncthreads();
    w.st = state;
    if (!w.st.waits) return;
    if constexpr (!POINTS) {
#pragma unroll 1
      for (uint32_t c = wave; c < a.chunks; c += kWalkThreads / 64) w.pass(c, sums);
      __syncthreads();
      if (wave == 0) {
        w.st.mass = wave_sum(w.lane < a.chunks ? sums[w.lane] : 0.0);
        if (w.st.waits > 1) w.st.left = wave_sum(w.lane < a.chunks ? sums[a.chunks + w.lane] : 0.0);
      }
    }
  }
}

// The rest of a walk.  Pass n: every block of a sequence goes on with the walk by the
// sums of pass n - 1 (alike, and one of them writes), up to the next rejection, and takes
// its part of the sums of max(p - t q, 0) that it waits for then.  END: one block a
// sequence, to the walk's end, by passes of its own where it has to.
//
// Passes by all compute units take 6 us for 8 sequences of 100003 logits, 9 for 32 of
// 131072, of which both sums in place of one are up to 1; by one block about 13.  All
// latency: vector units 9% busy.  Launches of their own for 3 / 4 / 5 / 8 of them, means of
// 8 inputs: 8 trees of up to 32 nodes 53.7 / 55.6 / 57.7 / 64.8 us, with up to 8 children
// 73.9 / 70.9 / 72.7 / 78.6, 32 of 24 nodes 99.1 / 94.5 / 93.9 / 99.5; an idle one is 1 to
// 2.  A counter and the last block to arrive in place of the next launch took 36 us for
// 1024 blocks, with fences by every thread; calls of few blocks were not tried.
template <typename TT, typename TD, bool END>
__global__ __launch_bounds__(END ? kWalkThreads : 256) void pass_kernel(VerifyArgs a, uint32_t n) {
  __shared__ Tree tree;
  __shared__ State state;
  const uint32_t s = blockIdx.y, tid = threadIdx.x, wave = eq_dev::uniform(tid >> 6);
  const uint32_t before = n ? (n - 1) & 1 : 0;
  State *const to = a.state[n & 1] + s;
  const bool writer = blockIdx.x == 0;
  const State st = a.state[before][s];
  const Rows r = rows_of(a.b, s);
  if (!st.waits) {
    if (!END && n && writer && tid == 0) to->waits = 0;
    return;
  }
  Walk<TT, TD, false> w(a, tree, s, r, writer, a.sums[before]);
  w.st = st;
  double v[4], left[4];  // the first 256 chunks' sums of the pass before
  w.load4(w.sums, 0, v);
  w.load4(w.sums + a.chunks, 0, left);  // (of anything, if they were not wanted)
  double *const new_sums = a.sums[n & 1] + 2 * uint64_t(s) * a.chunks;
  auto load_rows = [&](uint32_t i) {
    const uint64_t row = uint64_t(r.row) + i;
    tree.target[i] = a.target_stat[row], tree.draft[i] = a.draft_stat[row];
  };
  auto pass = [&](uint32_t first, uint32_t step, double *out) {
#pragma unroll 1
    for (uint32_t c = first; c < a.chunks; c += step) w.pass(c, out);
  };
  if (n == 0) {  // (the walk waits already)
    if (tid == 0) load_rows(st.cur);
    __syncthreads();
  } else {
    if (tid < kMaxNodes) tree.put(tid, load_node(a, r, tid));
    if (tid < w.count) {
      const uint64_t row = uint64_t(r.row) + tid;
      tree.px[tid] = a.px[row], tree.qx[tid] = a.qx[row];
      load_rows(tid);
      tree.link[tid] = a.link[row];
    }
    __syncthreads();
  }
#pragma unroll 1
  while (true) {
    if (n) {
      if (wave == 0) {
        w.st.mass = w.total_of(w.sums, v);
        if (w.st.waits > 1) w.st.left = w.total_of(w.sums + a.chunks, left);
        int32_t next;
        w.st.waits = w.walk(next);
        if (!w.st.waits) w.finish(next);
        if (w.lane == 0) {
          state = w.st;
          if (!END && writer) *to = w.st;
        }
      }
      __syncthreads();
      w.st = state;
      if (!w.st.waits) return;
    }
    if constexpr (!END) {
      pass(blockIdx.x * 4 + wave, gridDim.x * 4, new_sums);
      return;
    }
    pass(wave, kWalkThreads / 64, w.sums);
    __syncthreads();
    w.load4(w.sums, 0, v);
    w.load4(w.sums + a.chunks, 0, left);
  }
}

// ----------------------------------------------------------------------- host

bool batch_ok(const eq_kv_batch *b) {
  return b && b->n_seqs <= 65535 && b->max_new <= b->n_tokens && b->max_new <= kMaxNodes &&
         b->n_tokens <= 1u << 30 && (b->n_seqs == 0 || b->seq_start);
}

BatchArgs batch_args(const eq_kv_batch *b) {
  return BatchArgs{b->seq_start, b->kv_len, b->n_seqs, b->n_tokens, b->max_new};
}

size_t round256(size_t v) { return (v + 255) / 256 * 256; }

int done() { return hipGetLastError() == hipSuccess ? EQ_OK : EQ_EHIP; }

}  // namespace

extern "C" int eq_tree_mask(const eq_kv_batch *batch, const int32_t *parents, uint32_t window,
                            uint32_t *mask, int32_t *positions, hipStream_t stream) {
  if (!batch_ok(batch)) return EQ_EINVAL;
  if (batch->n_seqs == 0 || batch->max_new == 0) return EQ_OK;
  if (!batch->kv_len || !parents || !mask || !positions) return EQ_EINVAL;
  const MaskArgs a{batch_args(batch), parents, mask, positions, window, (batch->max_new + 31) / 32};
  hipLaunchKernelGGL(tree_mask_kernel, dim3(batch->n_seqs), dim3(kMaxNodes), 0, stream, a);
  return done();
}

namespace {

// The parts of a workspace, one behind the other.
struct Room {
  uint8_t *at;
  size_t used = 0;
  template <typename T>
  T *take(size_t n) {
    T *const p = reinterpret_cast<T *>(at + used);
    used += round256(n * sizeof(T));
    return p;
  }
};

// Splits a batch's rows and a workspace for them; the bytes that it needs.  (`per` goes by
// the whole batch's size, so the order of a row's sums and its exponentials' references do
// too: statistics of the same row may differ by 2^-38 between batches.)
size_t lay_out(VerifyArgs &a, bool draft, void *ws) {
  a.chunks = (a.vocab + kChunk - 1) / kChunk;
  const uint64_t work = uint64_t(a.chunks) * a.b.n_tokens * (draft ? 2 : 1);
  a.per = uint32_t(std::min<uint64_t>(std::max<uint64_t>(work / kStatWaves, 1), kMostPer));
  a.groups = (a.chunks + 4 * a.per - 1) / (4 * a.per);
  Room room{static_cast<uint8_t *>(ws)};
  const size_t rows = a.b.n_tokens, seqs = a.b.n_seqs;
  a.part = room.take<Part>(rows * a.chunks);
  a.target_group = room.take<Part>(rows * a.groups);
  if (a.chunks > kLocalChunks) a.rest = room.take<double>(seqs * a.chunks);
  if (draft) {
    a.sums[0] = room.take<double>(2 * seqs * a.chunks);
    a.sums[1] = room.take<double>(2 * seqs * a.chunks);
    a.state[0] = room.take<State>(seqs);
    a.state[1] = room.take<State>(seqs);
    a.draft_group = room.take<Part>(rows * a.groups);
    a.px = room.take<double>(rows);
    a.qx = room.take<double>(rows);
    a.target_stat = room.take<Stat>(rows);
    a.draft_stat = room.take<Stat>(rows);
    a.link = room.take<Link>(rows);
  }
  return room.used;
}

template <typename TT, typename TD>
void launch_verify(const VerifyArgs &a, uint32_t max_children, hipStream_t stream) {
  const bool draft = a.draft != nullptr;
  if (a.b.max_new)
    hipLaunchKernelGGL((row_stats_kernel<TT, TD>), dim3((draft ? 2 : 1) * a.groups, a.b.max_new, a.b.n_seqs),
                       dim3(256), 0, stream, a);
  const dim3 seqs(a.b.n_seqs);
  if (!draft) {
    hipLaunchKernelGGL((walk_kernel<TT, TD, true>), seqs, dim3(kWalkThreads), 0, stream, a);
    return;
  }
  hipLaunchKernelGGL((walk_kernel<TT, TD, false>), seqs, dim3(kWalkThreads), 0, stream, a);
  if (a.b.max_new < 2 || a.chunks <= kFewChunks) return;
  // a chain's walk ends with its first rejection
  const uint32_t rounds = max_children == 1 ? 1 : std::min(kRounds, a.b.max_new - 1);
  const dim3 pass((a.chunks + 3) / 4, a.b.n_seqs);
  for (uint32_t n = 0; n < rounds; ++n)
    hipLaunchKernelGGL((pass_kernel<TT, TD, false>), pass, dim3(256), 0, stream, a, n);
  hipLaunchKernelGGL((pass_kernel<TT, TD, true>), dim3(1, a.b.n_seqs), dim3(kWalkThreads), 0, stream, a,
                     rounds);
}

}  // namespace

extern "C" size_t eq_tree_verify_workspace_bytes(const eq_kv_batch *batch, uint32_t vocab, int draft) {
  if (!batch_ok(batch) || vocab == 0 || vocab > kMaxVocab || batch->n_seqs == 0) return 0;
  VerifyArgs a{};
  a.b = batch_args(batch);
  a.vocab = vocab;
  return lay_out(a, draft != 0, nullptr);
}

extern "C" int eq_tree_verify(const eq_kv_batch *batch, const int32_t *parents, const int32_t *tokens,
                              const void *target, uint64_t target_stride, uint32_t target_dtype,
                              const void *draft, uint64_t draft_stride, uint32_t draft_dtype,
                              uint32_t vocab, const float *temperature, const float *random,
                              uint32_t replace, uint32_t max_children, int32_t *path, int32_t *kept,
                              int32_t *next, void *ws, size_t ws_bytes, hipStream_t stream) {
  if (!batch_ok(batch) || target_dtype > EQ_BF16 || (draft && draft_dtype > EQ_BF16) || vocab == 0 ||
      vocab > kMaxVocab || max_children == 0)
    return EQ_EINVAL;
  if (batch->n_seqs == 0) return EQ_OK;
  VerifyArgs a{batch_args(batch), parents, tokens, target, draft, target_stride, draft_stride,
               temperature, random, path, kept, next};
  a.vocab = vocab;
  a.replace = replace != 0;
  const size_t need = lay_out(a, draft != nullptr, ws);
  if (!kept || !next || !ws || ws_bytes < need || (reinterpret_cast<uintptr_t>(ws) & 15)) return EQ_EINVAL;
  const auto odd = [](const void *p, uint32_t dtype) {
    return reinterpret_cast<uintptr_t>(p) % (dtype == EQ_F32 ? 4 : 2) != 0;
  };
  if (odd(target, target_dtype) || odd(draft, draft_dtype)) return EQ_EINVAL;
  if (batch->max_new &&
      (!parents || !tokens || !target || !random || !path ||
       (batch->n_tokens > 1 && (target_stride < vocab || (draft && draft_stride < vocab)))))
    return EQ_EINVAL;
  const bool t16 = target_dtype == EQ_BF16, d16 = draft ? draft_dtype == EQ_BF16 : t16;
  if (t16 && d16) launch_verify<uint16_t, uint16_t>(a, max_children, stream);
  else if (t16) launch_verify<uint16_t, float>(a, max_children, stream);
  else if (d16) launch_verify<float, uint16_t>(a, max_children, stream);
  else launch_verify<float, float>(a, max_children, stream);
  return done();
}
