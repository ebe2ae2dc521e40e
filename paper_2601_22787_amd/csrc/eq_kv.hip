// Query and key heads between the projections and attention, and the 4-bit
// key/value cache (declared in include/eq.h): the norm of each head with its
// rotation, appending to the cache with the keys' rotation on the way, and
// reading the cache back.  All of these move bytes: what bounds them is memory
// for prompts and the launch for single tokens.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "eq.h"
#include "eq_device.h"
#include "eq_kv.h"

namespace {

using namespace eq_kv;
using eq_dev::bf16_to_f32;
using eq_dev::pack_bf16;

struct Rope {
  const float *cos, *sin;
  uint32_t rows, half, pairs;  // half = 0: no rotation
};

// N consecutive elements (of 8 or 16) as fp32; VEC: 16-byte aligned.
template <typename T, int N, bool VEC>
__device__ inline void load_row(const T *p, float *x) {
  if constexpr (!VEC) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (sizeof(T) == 4) x[i] = p[i];
      else x[i] = bf16_to_f32(p[i]);
    }
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const float4 v = *reinterpret_cast<const float4 *>(p + i);
      x[i] = v.x, x[i + 1] = v.y, x[i + 2] = v.z, x[i + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 8) {
      const uint4 v = *reinterpret_cast<const uint4 *>(p + i);
      const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[i + 2 * j] = __uint_as_float(u[j] << 16);
        x[i + 2 * j + 1] = __uint_as_float(u[j] & 0xFFFF0000u);
      }
    }
  }
}

__device__ inline uint32_t table_row(const Rope &r, int32_t p) {
  return min(uint32_t(max(p, 0)), r.rows - 1);
}

// ------------------------------------------------------------ norm + rotation

struct NormArgs {
  const void *q, *k;
  uint64_t q_stride, k_stride;
  const uint16_t *q_weight, *k_weight;
  uint16_t *q_out, *k_out;
  const int32_t *positions;
  Rope rope;
  uint32_t tokens, q_heads, k_heads, dim;
  float eps;
  bool wide_weights;  // 16-byte aligned
  uint32_t parts;     // blocks of a token
};

// A head is held by L lanes (a power of two, dim/8 rounded up), 8 consecutive
// channels a lane: the mean is log2 L exchanges, a rotation by halves one more
// (channels c and c + half are half/8 lanes apart, half being a multiple of 8),
// and every load and store is 16 bytes a lane.  A block takes heads of one token,
// 256/L side by side, so that they share what its position reads.  A lane has all
// of a head before it stores any of it, and a head is one wavefront's, so BF16
// rows may be rewritten in place.
//
// Bound by memory: 8192 tokens of 72 heads of 128, BF16: 306 MB in 61.7 us, 4.96
// TB/s (a 1 GiB device copy: 5.07).  Heads in no order of tokens, each with its
// own table rows, took 79 us; two or three heads in flight for a lane 65 and 70,
// fewer wavefronts being resident then.
template <typename T, int L, bool VEC>
__global__ __launch_bounds__(256) void norm_rope_kernel(NormArgs a) {
  constexpr uint32_t kSide = 256 / L;
  const uint32_t heads = a.q_heads + a.k_heads;
  const uint32_t t = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
  const uint32_t c0 = 8 * (threadIdx.x % L), half = a.rope.half;
  const bool turned = c0 < 2 * half, upper = c0 >= half && !a.rope.pairs;
  float cs[8] = {}, sn[8] = {};
  if (turned) {
    const uint64_t at = uint64_t(table_row(a.rope, a.positions[t])) * half;
    if (a.rope.pairs) {
      load_row<float, 4, true>(a.rope.cos + at + c0 / 2, cs);
      load_row<float, 4, true>(a.rope.sin + at + c0 / 2, sn);
    } else {
      load_row<float, 8, true>(a.rope.cos + at + (upper ? c0 - half : c0), cs);
      load_row<float, 8, true>(a.rope.sin + at + (upper ? c0 - half : c0), sn);
    }
  }
  for (uint32_t h0 = part * kSide; h0 < heads; h0 += a.parts * kSide) {
    const uint32_t h = h0 + threadIdx.x / L;
    const bool on = h < heads && c0 < a.dim, is_k = h >= a.q_heads;
    const uint16_t *const weight = is_k ? a.k_weight : a.q_weight;
    float x[8] = {};
    if (on)
      load_row<T, 8, VEC>(is_k ? static_cast<const T *>(a.k) + t * a.k_stride +
                                     uint64_t(h - a.q_heads) * a.dim + c0
                               : static_cast<const T *>(a.q) + t * a.q_stride + uint64_t(h) * a.dim + c0,
                          x);
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) ss += x[i] * x[i];
#pragma unroll
    for (int d = 1; d < L; d *= 2) ss += __shfl_xor(ss, d);
    if (weight && on) {
      const float r = rsqrtf(ss / float(a.dim) + a.eps);
      float wt[8];
      if (a.wide_weights) load_row<uint16_t, 8, true>(weight + c0, wt);
      else load_row<uint16_t, 8, false>(weight + c0, wt);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = x[i] * r * wt[i];
    }
    if (half && a.rope.pairs) {
      if (turned) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float u = x[2 * i], v = x[2 * i + 1];
          x[2 * i] = u * cs[i] - v * sn[i];
          x[2 * i + 1] = v * cs[i] + u * sn[i];
        }
      }
    } else if (half) {
      const uint32_t step = half / 8, lane = threadIdx.x & 63;
      const uint32_t other = turned ? (upper ? lane - step : lane + step) : lane;
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = __shfl(x[i], int(other));
      if (turned) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = x[i] * cs[i] + (upper ? y[i] : -y[i]) * sn[i];
      }
    }
    if (on) {
      uint16_t *const out = is_k ? a.k_out + (uint64_t(t) * a.k_heads + h - a.q_heads) * a.dim + c0
                                 : a.q_out + (uint64_t(t) * a.q_heads + h) * a.dim + c0;
      *reinterpret_cast<uint4 *>(out) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]),
                                                   pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
    }
  }
}

// Few tokens: a block for each 256/L heads, so that no head waits for another's;
// many: one for a token.  A launch has fewer than 2^32 threads along x, so more
// tokens than kMostTokens are several launches.
constexpr uint32_t kMostTokens = 1u << 23;

template <typename T, bool VEC>
void launch_norm(const NormArgs &a, hipStream_t stream) {
  auto go = [&](auto kernel, uint32_t lanes) {
    const uint32_t per = 256 / lanes;
    for (uint64_t t = 0; t < a.tokens; t += kMostTokens) {
      NormArgs b = a;
      b.tokens = uint32_t(std::min<uint64_t>(a.tokens - t, kMostTokens));
      b.parts = b.tokens < 256 ? (a.q_heads + a.k_heads + per - 1) / per : 1;
      if (a.q_heads) {
        b.q = static_cast<const T *>(a.q) + t * a.q_stride;
        b.q_out = a.q_out + t * a.q_heads * a.dim;
      }
      if (a.k_heads) {
        b.k = static_cast<const T *>(a.k) + t * a.k_stride;
        b.k_out = a.k_out + t * a.k_heads * a.dim;
      }
      if (a.positions) b.positions = a.positions + t;
      hipLaunchKernelGGL(kernel, dim3(b.tokens * b.parts), dim3(256), 0, stream, b);
    }
  };
  const uint32_t need = a.dim / 8;
  if (need <= 2) go(norm_rope_kernel<T, 2, VEC>, 2);
  else if (need <= 4) go(norm_rope_kernel<T, 4, VEC>, 4);
  else if (need <= 8) go(norm_rope_kernel<T, 8, VEC>, 8);
  else if (need <= 16) go(norm_rope_kernel<T, 16, VEC>, 16);
  else go(norm_rope_kernel<T, 32, VEC>, 32);
}

// --------------------------------------------------------------------- append

struct AppendArgs {
  View w;
  const void *k, *v;
  uint64_t k_stride, v_stride;
  const int32_t *positions;
  Rope rope;
};

// Largest magnitude bits of x over the lanes of a group of G (a power of two)
// and this lane's N values; infinities and NaN sort above every number.
template <int N, int G>
__device__ inline uint32_t group_top(const float *x) {
  float top = 0.0f;  // (the maximum passes over NaN)
  bool nan = false;
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    top = fmaxf(top, fmaxf(fabsf(x[i]), fabsf(x[i + 1])));
    nan = nan || __builtin_isunordered(x[i], x[i + 1]);
  }
  uint32_t m = nan ? 0x7FC00000u : __float_as_uint(top);
#pragma unroll
  for (int d = 1; d < G; d *= 2) m = max(m, uint32_t(__shfl_xor(int(m), d)));
  return m;
}

// Scale byte of a group whose largest magnitude has the bits `top`: adding a
// quarter of the significand carries into the exponent from 1.75 on.
__device__ inline uint32_t scale_byte(uint32_t top) {
  if (top >= 0x7F800000u) return 255;
  return uint32_t(min(max(int32_t((top + 0x200000u) >> 23) - 2, 24), 252));
}

__device__ inline float scale_value(uint32_t b) { return __uint_as_float(b << 23); }

// Eight values over 2^(b - 127) as E2M1 codes, the first in the low bits.
__device__ inline uint32_t codes8(const float *x, uint32_t b) {
  const float s = scale_value(b == 255 ? 127 : b);
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], s, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], s, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], s, 2);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], s, 3);
  return r;
}

// The key's channels e0 .. e0 + N - 1 rotated.  Every product and the sum are
// rounded apart (no fused multiply-add), so that a code does not depend on how
// a compiler contracts them.  VEC: chunks of N do not straddle a half.
template <typename T, int N, bool VEC>
__device__ inline void rotate_key(const Rope &r, const T *row, uint32_t e0, int32_t pos, float *x) {
#pragma clang fp contract(off)
  const uint32_t half = r.half;
  if (e0 >= 2 * half) return;
  const uint64_t at = uint64_t(table_row(r, pos)) * half;
  if (r.pairs) {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      if (e0 + i >= 2 * half) break;
      const float c = r.cos[at + (e0 + i) / 2], s = r.sin[at + (e0 + i) / 2];
      const float u = x[i], v = x[i + 1];
      x[i] = u * c - v * s;
      x[i + 1] = v * c + u * s;
    }
  } else if (VEC && half % N == 0) {
    const bool upper = e0 >= half;
    const uint64_t o = at + (upper ? e0 - half : e0);
    float y[N], c[N], s[N];
    load_row<T, N, true>(row + (upper ? e0 - half : e0 + half), y);
    load_row<float, N, true>(r.cos + o, c);
    load_row<float, N, true>(r.sin + o, s);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float p = x[i] * c[i], q = y[i] * s[i];
      x[i] = upper ? p + q : p - q;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t e = e0 + i;
      if (e >= 2 * half) break;
      const bool upper = e >= half;
      float y;
      load_row<T, 1, false>(row + (upper ? e - half : e + half), &y);
      const uint64_t o = at + (upper ? e - half : e);
      const float p = x[i] * r.cos[o], q = y * r.sin[o];
      x[i] = upper ? p + q : p - q;
    }
  }
}

// A wavefront takes 8 positions (aligned to 8) of one head: those are the
// tokens of one dword of a channel's value codes, so no two wavefronts write
// the same dword, and one that writes only some of its tokens can keep the
// others'.  A token has 8 lanes of D/8 channels: its keys' scales are one or
// two exchanges, its value scale three.  Value codes go through LDS, a row of
// D/2 bytes a token, and come back as a column of bytes, two channels of eight
// tokens, that is repacked into the two channels' dwords.
//
// Between memory and vector instructions (rotation, the groups' maxima, packing:
// the vector units are half busy): 5729 positions of 32 heads of 128, BF16, with
// rotation, 121 MB in 30 us, 4.0 TB/s.  Whole units of 32 positions for a
// wavefront hold 175 registers and took 2 to 8 us more.  A token for each of 8
// sequences takes 4.6 us, all of it the chain from the lengths over the page
// number to the stores.
template <typename TK, typename TV, int D, bool VEC>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a, uint32_t groups) {
  constexpr int N = D / 8;           // channels a lane
  __shared__ __attribute__((aligned(16))) uint8_t lds[4][8][D / 2 + 4];
  const View &w = a.w;
  const uint32_t lane = threadIdx.x & 63, wave = eq_dev::uniform(threadIdx.x >> 6);
  const uint32_t s = blockIdx.y;
  const uint32_t item = blockIdx.x * 4 + wave;  // (group, head), heads within groups
  const Seq q = sequence(w, s);
  const uint32_t h = item % w.kv_heads;
  const int32_t start = max(q.base, 0), end = min(q.base + q.count, int32_t(w.max_len));
  int32_t first = 0, page = -1;
  if (item < groups * w.kv_heads && q.count > 0 && start < end) {
    first = (start & ~7) + 8 * int32_t(item / w.kv_heads);  // (below 2^31: both are at most 2^30)
    if (first < end) page = page_of(w, s, first);
  }
  const uint32_t t = lane >> 3, sub = lane & 7, e0 = sub * N;
  const int32_t pos = first + int32_t(t);
  const bool on = page >= 0 && pos >= q.base && pos < end;
  const uint32_t slot = uint32_t(pos) & ((1u << w.page_shift) - 1);
  uint8_t *const part = w.pages + uint64_t(max(page, 0)) * w.page_bytes + uint64_t(h) * w.head_bytes;
  const uint64_t row = on ? uint64_t(q.row) + (pos - q.base) : 0;
  float x[N] = {}, v[N] = {};
  if (on) {
    const TK *const kr = static_cast<const TK *>(a.k) + row * a.k_stride + uint64_t(h) * D;
    load_row<TK, N, VEC>(kr + e0, x);
    load_row<TV, N, VEC>(static_cast<const TV *>(a.v) + row * a.v_stride + uint64_t(h) * D + e0, v);
    if (a.rope.half) rotate_key<TK, N, VEC>(a.rope, kr, e0, a.positions ? a.positions[row] : pos, x);
  }
  constexpr int kPerBlock = 32 / N;  // lanes of a key group
  uint32_t b = scale_byte(group_top<N, kPerBlock>(x));
  if (on) {
    uint32_t *const kc = reinterpret_cast<uint32_t *>(part + slot * (D / 2) + e0 / 2);
    if constexpr (N == 16) *reinterpret_cast<uint2 *>(kc) = make_uint2(codes8(x, b), codes8(x + 8, b));
    else *kc = codes8(x, b);
    if (sub % kPerBlock == 0)
      part[w.ks_off + slot / 16 * (D / 2) + (slot % 4 * (D / 32) + sub / kPerBlock) * 4 +
           slot % 16 / 4] = uint8_t(b);
  }
  b = scale_byte(group_top<N, 8>(v));
  if (on && sub == 0) part[w.vs_off + slot] = uint8_t(b);
#pragma unroll
  for (int i = 0; i < N / 8; ++i)
    *reinterpret_cast<uint32_t *>(&lds[wave][t][e0 / 2 + 4 * i]) = codes8(v + 8 * i, b);
  const uint64_t mask = __ballot(on);
  __syncthreads();
  if (page < 0 || lane >= D / 2) return;
  uint32_t lo = 0, hi = 0, keep = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t c = lds[wave][i][lane];
    lo |= (c & 15) << (4 * i);
    hi |= (c >> 4) << (4 * i);
    if (!(mask >> (8 * i) & 1)) keep |= 15u << (4 * i);
  }
  const uint32_t slot0 = uint32_t(first) & ((1u << w.page_shift) - 1);
  uint32_t *const vc = reinterpret_cast<uint32_t *>(part + w.v_off +
                                                    (slot0 / 32 * D + 2 * lane) * 16 +
                                                    slot0 % 32 / 2);
  if (keep) {
    lo = (lo & ~keep) | (vc[0] & keep);
    hi = (hi & ~keep) | (vc[4] & keep);
  }
  vc[0] = lo;
  vc[4] = hi;
}

// ----------------------------------------------------------------------- read

// Two codes (a byte's) at 2^(b - 127) as BF16; every one is a BF16 value.
__device__ inline uint32_t bf16_pair(uint32_t byte, uint32_t b) {
  const uint32_t v = __builtin_bit_cast(
      uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(byte, scale_value(b), 0));
  return b == 255 ? 0x7FC07FC0u : v;
}

// A unit of 32 positions of a head for each wavefront, its loads in flight
// together (8 positions, a quarter of the bytes for the same chain of loads, took
// 47 us where this takes 42): of keys a lane has D/8 channels of four tokens, of
// values two channels of all 32, which leave as whole rows.
//
// Bound by memory, by its writes above all: 8 x 4096 positions of 8 heads of 128,
// 169 MB (134 of them written) in 41.7 us, 4.05 TB/s; streaming stores took 50.
// 1001 positions: 5.0 us, the chain of loads.
template <int D>
__global__ __launch_bounds__(256) void read_kernel(View w, uint16_t *k, uint16_t *v,
                                                   uint32_t units) {
  constexpr int N = D / 8;
  const uint32_t lane = threadIdx.x & 63, wave = eq_dev::uniform(threadIdx.x >> 6);
  const uint32_t s = blockIdx.y;
  const uint32_t item = blockIdx.x * 4 + wave;
  if (item >= units * w.kv_heads) return;
  const Seq q = sequence(w, s);
  const uint32_t h = item % w.kv_heads;
  const int32_t start = max(q.base, 0), end = min(q.base + q.count, int32_t(w.max_len));
  if (q.count <= 0 || start >= end) return;
  const int32_t first = (start & ~31) + 32 * int32_t(item / w.kv_heads);
  if (first >= end) return;
  const int32_t page = page_of(w, s, first);
  if (page < 0) return;
  const uint32_t slot0 = uint32_t(first) & ((1u << w.page_shift) - 1);
  const uint8_t *const part = w.pages + uint64_t(page) * w.page_bytes + uint64_t(h) * w.head_bytes;
  const uint32_t t = lane >> 3, sub = lane & 7, e0 = sub * N;
  uint4 vc[2], vs[2];
  uint32_t kc[4][N / 8], kb[4];
  // (what is read of tokens that are not asked for is in the unit all the same)
  const uint32_t pair = min(lane, uint32_t(D / 2 - 1));
#pragma unroll
  for (int i = 0; i < 2; ++i)
    vc[i] = *reinterpret_cast<const uint4 *>(part + w.v_off + (slot0 / 32 * D + 2 * pair + i) * 16);
#pragma unroll
  for (int i = 0; i < 2; ++i)
    vs[i] = *reinterpret_cast<const uint4 *>(part + w.vs_off + slot0 + 16 * i);
#pragma unroll
  for (uint32_t g = 0; g < 4; ++g) {
    const uint32_t slot = slot0 + 8 * g + t;
    const uint32_t *const p = reinterpret_cast<const uint32_t *>(part + slot * (D / 2) + e0 / 2);
#pragma unroll
    for (int i = 0; i < N / 8; ++i) kc[g][i] = p[i];
    kb[g] = part[w.ks_off + slot / 16 * (D / 2) + (slot % 4 * (D / 32) + e0 / 32) * 4 + slot % 16 / 4];
  }
  const uint64_t step = uint64_t(w.kv_heads) * D;  // elements between the rows of two tokens
  const int64_t row0 = (int64_t(q.row) + (first - q.base)) * int64_t(step) + int64_t(h) * D;
#pragma unroll
  for (uint32_t g = 0; g < 4; ++g) {
    const int32_t pos = first + int32_t(8 * g + t);
    if (pos < q.base || pos >= end) continue;
    uint16_t *const out = k + row0 + int64_t(8 * g + t) * int64_t(step) + e0;
#pragma unroll
    for (int i = 0; i < N / 8; ++i) {
      const uint32_t c = kc[g][i], b = kb[g];
      *reinterpret_cast<uint4 *>(out + 8 * i) =
          make_uint4(bf16_pair(c & 255, b), bf16_pair(c >> 8 & 255, b), bf16_pair(c >> 16 & 255, b),
                     bf16_pair(c >> 24, b));
    }
  }
  if (lane >= D / 2) return;
  const uint32_t lo[4] = {vc[0].x, vc[0].y, vc[0].z, vc[0].w};
  const uint32_t hi[4] = {vc[1].x, vc[1].y, vc[1].z, vc[1].w};
  const uint32_t sc[8] = {vs[0].x, vs[0].y, vs[0].z, vs[0].w, vs[1].x, vs[1].y, vs[1].z, vs[1].w};
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    if (first + i < q.base || first + i >= end) continue;
    const uint32_t byte = (lo[i / 8] >> (4 * (i % 8)) & 15) | (hi[i / 8] >> (4 * (i % 8)) & 15) << 4;
    *reinterpret_cast<uint32_t *>(v + row0 + int64_t(i) * int64_t(step) + 2 * lane) =
        bf16_pair(byte, sc[i / 4] >> (8 * (i % 4)) & 255);
  }
}

// ----------------------------------------------------------------------- host

bool rope_ok(const eq_rope *r, uint32_t head_dim) {
  return !r || (r->cos && r->sin && r->rows >= 1 && r->dims >= 16 && r->dims % 16 == 0 &&
                r->dims <= head_dim &&
                ((reinterpret_cast<uintptr_t>(r->cos) | reinterpret_cast<uintptr_t>(r->sin)) & 15) ==
                    0);
}

Rope device_rope(const eq_rope *r) {
  return r ? Rope{r->cos, r->sin, r->rows, r->dims / 2, r->pairs} : Rope{nullptr, nullptr, 1, 0, 0};
}

bool aligned16(const void *p, uint64_t stride_bytes) {
  return ((reinterpret_cast<uintptr_t>(p) | stride_bytes) & 15) == 0;
}

int done() { return hipGetLastError() == hipSuccess ? EQ_OK : EQ_EHIP; }

// Aligned runs of `run` positions that `max_new` consecutive ones can touch.
uint32_t position_runs(uint32_t max_new, uint32_t run) { return (max_new + run - 2) / run + 1; }

}  // namespace

extern "C" int eq_qk_norm_rope(const void *q, uint64_t q_stride, uint32_t q_heads,
                               const uint16_t *q_weight, uint16_t *q_out, const void *k,
                               uint64_t k_stride, uint32_t k_heads, const uint16_t *k_weight,
                               uint16_t *k_out, uint32_t dtype, uint32_t tokens, uint32_t head_dim,
                               float eps, const int32_t *positions, const eq_rope *rope,
                               hipStream_t stream) {
  const uint64_t heads = uint64_t(q_heads) + k_heads;
  if (dtype > EQ_BF16 || head_dim == 0 || head_dim % 16 || head_dim > 256 || q_heads > 4096 ||
      k_heads > 4096 || !rope_ok(rope, head_dim) || !(eps >= 0.0f))
    return EQ_EINVAL;
  if (tokens == 0 || heads == 0) return EQ_OK;  // (a tensor of no tokens has no address)
  if (rope && !positions) return EQ_EINVAL;
  if ((q_heads && (!q || !q_out || (reinterpret_cast<uintptr_t>(q_out) & 15) ||
                   (tokens > 1 && q_stride < uint64_t(q_heads) * head_dim))) ||
      (k_heads && (!k || !k_out || (reinterpret_cast<uintptr_t>(k_out) & 15) ||
                   (tokens > 1 && k_stride < uint64_t(k_heads) * head_dim))))
    return EQ_EINVAL;
  const uint64_t item = dtype == EQ_F32 ? 4 : 2;
  NormArgs a{q, k, q_stride, k_stride, q_weight, k_weight, q_out, k_out, positions,
             device_rope(rope), tokens, q_heads, k_heads, head_dim, eps,
             ((reinterpret_cast<uintptr_t>(q_weight) | reinterpret_cast<uintptr_t>(k_weight)) & 15) == 0,
             0};
  const bool vec = (!q_heads || aligned16(q, q_stride * item)) &&
                   (!k_heads || aligned16(k, k_stride * item));
  if (dtype == EQ_F32) vec ? launch_norm<float, true>(a, stream) : launch_norm<float, false>(a, stream);
  else vec ? launch_norm<uint16_t, true>(a, stream) : launch_norm<uint16_t, false>(a, stream);
  return done();
}

extern "C" size_t eq_kv_page_bytes(uint32_t kv_heads, uint32_t head_dim, uint32_t page_tokens) {
  if (!sizes_ok(kv_heads, head_dim, page_tokens)) return 0;
  return size_t(head_bytes(head_dim, page_tokens)) * kv_heads;
}

namespace {

template <typename TK, typename TV>
void launch_append(const AppendArgs &a, uint32_t head_dim, bool vec, uint32_t groups, dim3 grid,
                   hipStream_t stream) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a, groups); };
  if (head_dim == 128) vec ? go(append_kernel<TK, TV, 128, true>) : go(append_kernel<TK, TV, 128, false>);
  else vec ? go(append_kernel<TK, TV, 64, true>) : go(append_kernel<TK, TV, 64, false>);
}

}  // namespace

extern "C" int eq_kv_append(const eq_kv_cache *cache, const eq_kv_batch *batch, const void *k,
                            uint64_t k_stride, uint32_t k_dtype, const void *v, uint64_t v_stride,
                            uint32_t v_dtype, const int32_t *positions, const eq_rope *rope,
                            hipStream_t stream) {
  if (!batch_ok(cache, batch) || k_dtype > EQ_BF16 || v_dtype > EQ_BF16 ||
      !rope_ok(rope, cache->head_dim))
    return EQ_EINVAL;
  if (batch->n_seqs == 0 || batch->max_new == 0 || batch->max_len == 0) return EQ_OK;
  const uint64_t width = uint64_t(cache->kv_heads) * cache->head_dim;
  if (!k || !v || (batch->n_tokens > 1 && (k_stride < width || v_stride < width))) return EQ_EINVAL;
  AppendArgs a{view(cache, batch), k, v, k_stride, v_stride, positions, device_rope(rope)};
  const bool vec = aligned16(k, k_stride * (k_dtype == EQ_F32 ? 4 : 2)) &&
                   aligned16(v, v_stride * (v_dtype == EQ_F32 ? 4 : 2));
  const uint32_t groups = position_runs(batch->max_new, 8);
  const uint64_t blocks = (uint64_t(groups) * cache->kv_heads + 3) / 4;
  if (blocks > kMaxBlocks) return EQ_EINVAL;
  const dim3 grid(uint32_t(blocks), batch->n_seqs);
  const uint32_t d = cache->head_dim;
  if (k_dtype == EQ_F32)
    v_dtype == EQ_F32 ? launch_append<float, float>(a, d, vec, groups, grid, stream)
                      : launch_append<float, uint16_t>(a, d, vec, groups, grid, stream);
  else
    v_dtype == EQ_F32 ? launch_append<uint16_t, float>(a, d, vec, groups, grid, stream)
                      : launch_append<uint16_t, uint16_t>(a, d, vec, groups, grid, stream);
  return done();
}

extern "C" int eq_kv_read(const eq_kv_cache *cache, const eq_kv_batch *batch, uint16_t *k,
                          uint16_t *v, hipStream_t stream) {
  if (!batch_ok(cache, batch)) return EQ_EINVAL;
  if (batch->n_seqs == 0 || batch->max_new == 0 || batch->max_len == 0) return EQ_OK;
  if (!k || !v || ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 15))
    return EQ_EINVAL;
  const uint32_t units = position_runs(batch->max_new, 32);
  const uint64_t blocks = (uint64_t(units) * cache->kv_heads + 3) / 4;
  if (blocks > kMaxBlocks) return EQ_EINVAL;
  const dim3 grid(uint32_t(blocks), batch->n_seqs);
  if (cache->head_dim == 128)
    hipLaunchKernelGGL((read_kernel<128>), grid, dim3(256), 0, stream, view(cache, batch), k, v,
                       units);
  else
    hipLaunchKernelGGL((read_kernel<64>), grid, dim3(256), 0, stream, view(cache, batch), k, v,
                       units);
  return done();
}
