// Drafted trees (declared in include/eq.h): their masks and positions, and the
// verification of drafted tokens against the target's distributions.
//
// Verification.  p and q are the softmax of a target's and a draft's logits.  With
// r_0 = p, the children x_1, x_2, .. of a node are tested in order: x_j is accepted
// with probability min(1, r(x_j) / q(x_j)), else r becomes max(r - q, 0) and q loses
// x_j, both normalised again.  All of that is one family of functions,
//   r ~ max(p - t q, 0),  G(t) = sum max(p - t q, 0),  Q = 1 - sum of the rejected q,
// from t = 0 (G = 1, Q = 1), with t + G / Q in the place of t after a rejection:
//   max(p - t q, 0) / G - q / Q = (max(p - t q, 0) - (G / Q) q) / G.
// A rejected x has p(x) < t q(x) from then on, so that q need not be cut there.  x is
// accepted when u G q(x) < max(p(x) - t q(x), 0) Q.  A rejection thus costs one pass
// over the vocabulary for one number.
//
// Everything is in 64 bits.  A token is where a running sum of probabilities passes u
// times the whole: the sum's error, over the probabilities near it, is how often a
// rounding would decide, 2^-24 times thousands of tokens in 32 bits.  64-bit vector
// instructions issue at the rate of 32-bit ones here, and an exponential is 20.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "eq.h"
#include "eq_device.h"

namespace {

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
  const int32_t row = b.seq_start[s], end = b.seq_start[s + 1];
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
// LDS: as many steps as the node is deep.
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

// A chunk's largest logit, where it first is (-1: the chunk holds a NaN or +infinity),
// and the sum of exp((x - max) / T).
struct Part {
  double sum;
  float max;
  int32_t arg;
};

struct VerifyArgs {
  BatchArgs b;
  const int32_t *parents, *tokens;
  const void *target, *draft;
  uint64_t target_stride, draft_stride;
  const float *temperature, *random;
  int32_t *path, *kept, *next;
  Part *target_part, *draft_part;  // [n_tokens][chunks]
  double *sums;                    // [n_seqs][chunks]
  uint32_t vocab, chunks;
  bool replace;
};

// exp(x) for x <= 0, 0 where it is below 2^-1022 (and for NaN): x = k ln 2 + r, the
// series of exp(r) to its 12th power (|r| <= ln 2 / 2: the next term is 2^-52).
__device__ inline double exp_down(double x) {
  x = fmax(x, -800.0);
  const double k = __builtin_rint(x * 1.4426950408889634074);
  double r = __builtin_fma(k, -2977044471.0 / 4294967296.0, x);  // ln 2: its first 32 bits,
  r = __builtin_fma(k, -1.9082149292705877e-10, r);          // and the rest
  double y = 1.0 / 479001600.0;
  y = __builtin_fma(y, r, 1.0 / 39916800.0);
  y = __builtin_fma(y, r, 1.0 / 3628800.0);
  y = __builtin_fma(y, r, 1.0 / 362880.0);
  y = __builtin_fma(y, r, 1.0 / 40320.0);
  y = __builtin_fma(y, r, 1.0 / 5040.0);
  y = __builtin_fma(y, r, 1.0 / 720.0);
  y = __builtin_fma(y, r, 1.0 / 120.0);
  y = __builtin_fma(y, r, 1.0 / 24.0);
  y = __builtin_fma(y, r, 1.0 / 6.0);
  y = __builtin_fma(y, r, 0.5);
  y = __builtin_fma(y, r, 1.0);
  y = __builtin_fma(y, r, 1.0);
  return __builtin_ldexp(y, int(k));
}

template <typename T>
__device__ inline float logit(const T *row, uint32_t i) {
  if constexpr (sizeof(T) == 4) return row[i];
  else return eq_dev::bf16_to_f32(row[i]);
}

// A lane's 16 logits of a chunk, four in a row: element 4 i + e is number 256 i + 4
// lane + e.  -infinity behind the vocabulary.  Rows start at any element.
template <typename T>
__device__ inline void load_chunk(const T *row, uint32_t vocab, uint32_t first, uint32_t lane,
                                  float (&x)[16]) {
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    const uint32_t at = first + 256 * i + 4 * lane;
    if (at + 4 <= vocab) {
      T v[4];
      __builtin_memcpy(v, row + at, sizeof(v));
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) x[4 * i + e] = logit(v, e);
    } else {
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) x[4 * i + e] = at + e < vocab ? logit(row, at + e) : -INFINITY;
    }
  }
}

__device__ inline double wave_sum64(double v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  return v;
}

__device__ inline float temperature_of(const VerifyArgs &a, uint32_t s) {
  return a.temperature ? a.temperature[s] : 1.0f;
}

// The statistics of a row's chunks, a wavefront each.  Draft rows of nodes without
// children are left out.
template <typename TT, typename TD>
__global__ __launch_bounds__(256) void row_stats_kernel(VerifyArgs a) {
  const uint32_t s = blockIdx.z, i = blockIdx.y;
  const uint32_t groups = (a.chunks + 3) / 4;
  const bool drafted = blockIdx.x >= groups;
  const Rows r = rows_of(a.b, s);
  if (int32_t(i) >= r.count) return;
  const float temp = temperature_of(a, s);
  const bool greedy = !(temp > 0.0f);
  if (drafted) {
    if (greedy) return;
    const int32_t j = int32_t(threadIdx.x);
    if (!__syncthreads_or(j > int32_t(i) && j < r.count && a.parents[r.row + j] == int32_t(i))) return;
  }
  const uint32_t lane = threadIdx.x & 63, wave = eq_dev::uniform(threadIdx.x >> 6);
  const uint32_t chunk = (blockIdx.x - (drafted ? groups : 0)) * 4 + wave;
  if (chunk >= a.chunks) return;
  const uint64_t row = uint64_t(r.row) + i;
  float x[16];
  if (drafted)
    load_chunk(static_cast<const TD *>(a.draft) + row * a.draft_stride, a.vocab, chunk * kChunk, lane, x);
  else
    load_chunk(static_cast<const TT *>(a.target) + row * a.target_stride, a.vocab, chunk * kChunk, lane,
               x);
  float top = x[0];
  bool bad = false;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    top = fmaxf(top, x[e]);
    bad = bad || !(x[e] < INFINITY);
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
  int32_t arg = 0x7FFFFFFF;
#pragma unroll
  for (int e = 15; e >= 0; --e)
    if (x[e] == top) arg = int32_t(chunk * kChunk + 256 * (e / 4) + 4 * lane + e % 4);
#pragma unroll
  for (int d = 1; d < 64; d *= 2) arg = min(arg, __shfl_xor(arg, d));
  double sum = 0.0;
  if (!greedy && top > -INFINITY) {
    const double inv = 1.0 / double(temp), m = double(top);
#pragma unroll
    for (int e = 0; e < 16; ++e) sum += exp_down((double(x[e]) - m) * inv);
    sum = wave_sum64(sum);
  }
  if (__any(bad)) arg = -1;
  if (lane == 0) (drafted ? a.draft_part : a.target_part)[row * a.chunks + chunk] = Part{sum, top, arg};
}

// A row's distribution: exp((x - max) / T) inv; best: its first largest logit, or -1
// where the row has no distribution.
struct Stat {
  double inv;
  float max;
  int32_t best;
};

// A row's statistics from its chunks', by 16 lanes: the same in all of them.
__device__ inline Stat join_parts(const Part *part, uint32_t chunks, uint32_t lane16, double inv_temp) {
  float top = -INFINITY;
  int32_t arg = 0x7FFFFFFF;
  bool bad = false;
  for (uint32_t c = lane16; c < chunks; c += 16) {
    const Part p = part[c];
    bad = bad || p.arg < 0;
    if (p.max > top || arg == 0x7FFFFFFF) top = p.max, arg = p.arg;
  }
#pragma unroll
  for (int d = 1; d < 16; d *= 2) {
    const float m = __shfl_xor(top, d);
    const int32_t j = __shfl_xor(arg, d);
    const int b = __shfl_xor(int(bad), d);
    bad = bad || b;
    if (m > top || (m == top && j < arg)) top = m, arg = j;
  }
  double sum = 0.0;
  for (uint32_t c = lane16; c < chunks; c += 16) {
    const Part p = part[c];
    sum += p.max > -INFINITY ? p.sum * exp_down((double(p.max) - double(top)) * inv_temp) : 0.0;
  }
#pragma unroll
  for (int d = 1; d < 16; d *= 2) sum += __shfl_xor(sum, d);
  return Stat{1.0 / sum, top, bad || top == -INFINITY ? -1 : arg};
}

// One block walks a sequence's tree.  Every wavefront takes the same decisions.
template <typename TT, typename TD, bool POINTS>
__global__ __launch_bounds__(1024) void walk_kernel(VerifyArgs a) {
  __shared__ Stat target_stat[kMaxNodes], draft_stat[kMaxNodes];
  __shared__ double px[kMaxNodes], qx[kMaxNodes];  // p and q of a node's token at its parent
  __shared__ int32_t up[kMaxNodes], token[kMaxNodes];
  __shared__ uint32_t inner[kMaxNodes], hidden[kChunk / 32];
  const uint32_t s = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const uint32_t wave = eq_dev::uniform(tid >> 6), waves = blockDim.x >> 6;
  const Rows r = rows_of(a.b, s);
  if (r.count <= 0) {
    if (tid == 0) a.kept[s] = 0, a.next[s] = -1;
    return;
  }
  const uint32_t count = uint32_t(r.count);
  const float temp = temperature_of(a, s);
  const bool greedy = !(temp > 0.0f);
  const double inv_temp = greedy ? 1.0 : 1.0 / double(temp);
  auto target_row = [&](uint32_t i) {
    return static_cast<const TT *>(a.target) + (uint64_t(r.row) + i) * a.target_stride;
  };
  auto draft_row = [&](uint32_t i) {
    return static_cast<const TD *>(a.draft) + (uint64_t(r.row) + i) * a.draft_stride;
  };

  if (tid < count) {
    const int32_t p = a.parents[r.row + int32_t(tid)];
    up[tid] = tid > 0 && p >= 0 && p < int32_t(tid) ? p : -1;
    token[tid] = a.tokens[r.row + int32_t(tid)];
    inner[tid] = 0;
  }
  __syncthreads();
  if (tid < count && up[tid] >= 0) inner[up[tid]] = 1;
  __syncthreads();
  for (uint32_t k = tid / 16; k < (POINTS ? 1 : 2) * count; k += blockDim.x / 16) {
    const bool drafted = k >= count;
    const uint32_t i = drafted ? k - count : k;
    if (drafted && (greedy || !inner[i])) continue;
    const Stat st = join_parts((drafted ? a.draft_part : a.target_part) + (uint64_t(r.row) + i) * a.chunks,
                               a.chunks, tid & 15, inv_temp);
    if ((tid & 15) == 0) (drafted ? draft_stat : target_stat)[i] = st;
  }
  __syncthreads();
  auto prob = [&](const Stat &st, float x) {
    return exp_down((double(x) - double(st.max)) * inv_temp) * st.inv;
  };
  if (tid < count && up[tid] >= 0 && uint32_t(token[tid]) < a.vocab && !greedy) {
    const uint32_t p = uint32_t(up[tid]), x = uint32_t(token[tid]);
    px[tid] = prob(target_stat[p], logit(target_row(p), x));
    if constexpr (POINTS) qx[tid] = 1.0;
    else qx[tid] = prob(draft_stat[p], logit(draft_row(p), x));
  }
  __syncthreads();

  auto random_of = [&](uint32_t i) {
    const float u = a.random[r.row + int32_t(i)];
    return double(fminf(fmaxf(u, 0.0f), 0.99999994f));  // (NaN: 0)
  };
  // the node's next child behind node `last`, or `count`
  auto child = [&](uint32_t node, uint32_t last) {
    for (uint32_t c = (last + 1) / 64 * 64; c < count; c += 64) {
      const uint32_t j = c + lane;
      const uint64_t m = __ballot(j > last && j < count && up[j] == int32_t(node));
      if (m) return c + uint32_t(__ffsll((unsigned long long)m)) - 1;
    }
    return count;
  };

  uint32_t cur = 0, last = 0, kept = 1;
  double t = 0.0, mass = 1.0, left = 1.0;
  if (tid == 0) a.path[r.row] = 0;
  int32_t next = -1;
  double *const sums = a.sums + uint64_t(s) * a.chunks;
  const uint32_t chunks = a.chunks;
  // weights of a chunk at the node where the walk stands; POINTS: without the tokens
  // in `hidden`, where any are
  auto weights = [&](uint32_t chunk, double tt, bool cut, double (&w)[16]) {
    float x[16];
    load_chunk(target_row(cur), a.vocab, chunk * kChunk, lane, x);
    const Stat ps = target_stat[cur];
#pragma unroll
    for (int e = 0; e < 16; ++e) w[e] = prob(ps, x[e]);
    if constexpr (!POINTS) {
      if (tt > 0.0) {
        load_chunk(draft_row(cur), a.vocab, chunk * kChunk, lane, x);
        const Stat qs = draft_stat[cur];
#pragma unroll
        for (int e = 0; e < 16; ++e) w[e] = fmax(w[e] - tt * prob(qs, x[e]), 0.0);
      }
    } else if (cut) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const uint32_t at = 256 * (e / 4) + 4 * lane + e % 4;
        if (hidden[at / 32] >> (at % 32) & 1) w[e] = 0.0;
      }
    }
  };
  auto chunk_sum = [&](const double (&w)[16]) {
    double v = 0.0;
#pragma unroll
    for (int e = 0; e < 16; ++e) v += w[e];
    return wave_sum64(v);
  };
  // the whole of sums, in a fixed order
  auto whole = [&]() {
    double v = 0.0;
    for (uint32_t c = lane; c < chunks; c += 64) v += sums[c];
    return wave_sum64(v);
  };
  // the chunk's tokens among the node's children before `end`, as bits
  auto hide = [&](uint32_t chunk, uint32_t end) {
    __syncthreads();
    if (tid < kChunk / 32) hidden[tid] = 0;
    __syncthreads();
    if (tid < end && up[tid] == int32_t(cur) && uint32_t(token[tid]) / kChunk == chunk)
      atomicOr(&hidden[uint32_t(token[tid]) % kChunk / 32], 1u << (token[tid] & 31));
    __syncthreads();
  };

  while (true) {
    const Stat here = target_stat[cur];
    if (here.best < 0) break;
    uint32_t c = child(cur, last);
    if (greedy) {
      while (c < count && token[c] != here.best) c = child(cur, c);
      if (c >= count) {
        next = here.best;
        break;
      }
      cur = last = c;
      if (tid == 0) a.path[r.row + int32_t(kept)] = int32_t(c);
      ++kept;
      continue;
    }
    if (!POINTS && c < count && draft_stat[cur].best < 0) break;
    bool down = false;
    for (; c < count; c = child(cur, c)) {
      last = c;
      if (uint32_t(token[c]) >= a.vocab) continue;
      const double q = qx[c];
      bool again = false;  // an earlier child of the same token was rejected
      for (uint32_t j = lane; j < c; j += 64)
        again = again || (up[j] == int32_t(cur) && token[j] == token[c]);
      again = __any(again);
      const double rest = again ? 0.0 : fmax(px[c] - t * q, 0.0);
      if (random_of(c) * mass * q < rest * left) {
        down = true;
        break;
      }
      if constexpr (POINTS) {
        mass = fmax(mass - rest, 0.0);
      } else {
        if (left > 0.0) t += mass / left;
        if (!a.replace && !again) left = fmax(left - q, 0.0);
        __syncthreads();
        for (uint32_t k = wave; k < chunks; k += waves) {
          double w[16];
          weights(k, t, false, w);
          const double v = chunk_sum(w);
          if (lane == 0) sums[k] = v;
        }
        __syncthreads();
        mass = whole();
      }
    }
    if (down) {
      cur = last = c;
      if (tid == 0) a.path[r.row + int32_t(kept)] = int32_t(c);
      ++kept;
      t = 0.0, mass = 1.0, left = 1.0;
      continue;
    }
    // no child is left: the next token from what remains, or from p where nothing does
    const bool rejected = last != cur;
    bool rest = rejected;
    if (POINTS || t == 0.0 || mass <= 0.0) {
      if (!POINTS) t = 0.0, rest = false;
      const Part *const part = a.target_part + (uint64_t(r.row) + cur) * chunks;
      auto from_parts = [&]() {
        __syncthreads();
        for (uint32_t k = tid; k < chunks; k += blockDim.x) {
          const Part p = part[k];
          sums[k] = p.max > -INFINITY
                        ? p.sum * exp_down((double(p.max) - double(here.max)) * inv_temp) * here.inv
                        : 0.0;
        }
        __syncthreads();
      };
      from_parts();
      if (POINTS && rest) {
        for (uint32_t c2 = child(cur, cur); c2 < count; c2 = child(cur, c2)) {
          if (uint32_t(token[c2]) >= a.vocab) continue;
          const uint32_t k = uint32_t(token[c2]) / kChunk;
          hide(k, count);
          if (wave == 0) {
            double w[16];
            weights(k, 0.0, true, w);
            const double v = chunk_sum(w);
            if (lane == 0) sums[k] = v;
          }
        }
        __syncthreads();
        if (!(whole() > 0.0)) {
          rest = false;
          from_parts();
        }
      }
    }
    const double limit = random_of(0) * whole();
    // the first chunk whose running sum passes the limit
    double before = 0.0;
    uint32_t at = chunks;
    for (uint32_t c0 = 0; c0 < chunks; c0 += 64) {
      const double v = c0 + lane < chunks ? sums[c0 + lane] : 0.0;
      double run = v;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const double o = __shfl_up(run, d);
        if (int(lane) >= d) run += o;
      }
      const uint64_t m = __ballot(before + run > limit && v > 0.0);
      if (m) {
        const int l = __ffsll((unsigned long long)m) - 1;
        at = c0 + uint32_t(l);
        before += __shfl(run - v, l);
        break;
      }
      before += __shfl(run, 63);
    }
    if (POINTS && rest && at < chunks) hide(at, count);
    next = here.best;
    if (at < chunks) {
      double w[16];
      weights(at, t, rest, w);
      int32_t found = 0x7FFFFFFF, any = -1;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const double v = (w[4 * i] + w[4 * i + 1]) + (w[4 * i + 2] + w[4 * i + 3]);
        double run = v;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
          const double o = __shfl_up(run, d);
          if (int(lane) >= d) run += o;
        }
        double sum = before + (run - v);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int32_t id = int32_t(at * kChunk + 256 * i + 4 * lane + e);
          sum += w[4 * i + e];
          if (w[4 * i + e] > 0.0) {
            any = id;
            if (sum > limit) found = min(found, id);
          }
        }
        before += __shfl(run, 63);
      }
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        found = min(found, __shfl_xor(found, d));
        any = max(any, __shfl_xor(any, d));
      }
      // (a rounding may leave the sum at the chunk's end just below the limit)
      if (found != 0x7FFFFFFF) next = found;
      else if (any >= 0) next = any;
    }
    break;
  }
  if (tid >= kept && tid < count) a.path[r.row + int32_t(tid)] = -1;
  if (tid == 0) a.kept[s] = int32_t(kept), a.next[s] = next;
}

// ----------------------------------------------------------------------- host

bool batch_ok(const eq_kv_batch *b) {
  return b && b->n_seqs <= 65535 && b->max_new <= b->n_tokens && b->max_new <= kMaxNodes &&
         b->n_tokens <= 1u << 30 && (b->n_seqs == 0 || b->seq_start);
}

BatchArgs batch_args(const eq_kv_batch *b) {
  return BatchArgs{b->seq_start, b->kv_len, b->n_seqs, b->n_tokens, b->max_new};
}

uint32_t chunks_of(uint32_t vocab) { return (vocab + kChunk - 1) / kChunk; }

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

extern "C" size_t eq_tree_verify_workspace_bytes(const eq_kv_batch *batch, uint32_t vocab, int draft) {
  if (!batch_ok(batch) || vocab == 0 || vocab > kMaxVocab || batch->n_seqs == 0 || batch->max_new == 0)
    return 0;
  const size_t rows = round256(size_t(batch->n_tokens) * chunks_of(vocab) * sizeof(Part));
  return rows * (draft ? 2 : 1) + round256(size_t(batch->n_seqs) * chunks_of(vocab) * sizeof(double));
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
  if (!kept || !next) return EQ_EINVAL;
  const size_t need = eq_tree_verify_workspace_bytes(batch, vocab, draft != nullptr);
  if (batch->max_new && (!parents || !tokens || !target || !random || !path || !ws || ws_bytes < need ||
                         (reinterpret_cast<uintptr_t>(ws) & 15) ||
                         (batch->n_tokens > 1 && (target_stride < vocab || (draft && draft_stride < vocab)))))
    return EQ_EINVAL;
  VerifyArgs a{batch_args(batch), parents, tokens, target, draft, target_stride, draft_stride,
               temperature, random, path, kept, next, nullptr, nullptr, nullptr, vocab,
               chunks_of(vocab), replace != 0};
  const size_t rows = round256(size_t(batch->n_tokens) * a.chunks * sizeof(Part));
  uint8_t *at = static_cast<uint8_t *>(ws);
  a.target_part = reinterpret_cast<Part *>(at);
  if (draft) a.draft_part = reinterpret_cast<Part *>(at += rows);
  a.sums = reinterpret_cast<double *>(at + rows);
  const dim3 stats((draft ? 2 : 1) * ((a.chunks + 3) / 4), batch->max_new, batch->n_seqs);
  const dim3 walk(batch->n_seqs), many(1024);
  auto go = [&](auto tt, auto td) {
    using TT = decltype(tt);
    using TD = decltype(td);
    if (batch->max_new) hipLaunchKernelGGL((row_stats_kernel<TT, TD>), stats, dim3(256), 0, stream, a);
    if (draft) hipLaunchKernelGGL((walk_kernel<TT, TD, false>), walk, many, 0, stream, a);
    else hipLaunchKernelGGL((walk_kernel<TT, TT, true>), walk, many, 0, stream, a);
  };
  const bool t16 = target_dtype == EQ_BF16, d16 = draft ? draft_dtype == EQ_BF16 : t16;
  if (t16) d16 ? go(uint16_t{}, uint16_t{}) : go(uint16_t{}, float{});
  else d16 ? go(float{}, uint16_t{}) : go(float{}, float{});
  return done();
}
