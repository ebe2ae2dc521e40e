// Query and key heads between the projections and attention, and the 4-bit
// key/value cache (declared in include/eq.h): the norm of each head with its
// rotation, appending to the cache with the keys' rotation on the way, and
// reading the cache back.  All of these move bytes: what bounds them is memory
// for prompts and the launch for single tokens.
#include <hip/hip_runtime.h>

#include "eq.h"
#include "eq_device.h"
#include "eq_kv.h"

namespace {

using namespace eq_kv;
using eq_dev::bf16_to_f32;
using eq_dev::pack_bf16;

typedef short short2v __attribute__((ext_vector_type(2)));

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
};

// A head is held by L lanes (a power of two, dim/8 rounded up), 8 consecutive
// channels a lane, so a wavefront normalises 64/L heads at once: the mean is
// log2 L exchanges, a rotation by halves one more (channels c and c + half are
// half/8 lanes apart, half being a multiple of 8), and every load and store
// is 16 bytes a lane.  A lane has all of its inputs before its first store, and
// a head is one wavefront's, so BF16 rows may be rewritten in place.
template <typename T, int L, bool VEC>
__global__ __launch_bounds__(256) void norm_rope_kernel(NormArgs a) {
  const uint32_t heads = a.q_heads + a.k_heads;
  const uint64_t item = (uint64_t(blockIdx.x) * 256 + threadIdx.x) / L;
  const uint32_t l = threadIdx.x % L, c0 = 8 * l;
  const bool on = item < uint64_t(a.tokens) * heads && c0 < a.dim;
  const uint32_t t = on ? uint32_t(item / heads) : 0, h = on ? uint32_t(item % heads) : 0;
  const bool is_k = h >= a.q_heads;
  const uint32_t hh = is_k ? h - a.q_heads : h;
  const uint16_t *const weight = is_k ? a.k_weight : a.q_weight;
  float x[8] = {};
  if (on)
    load_row<T, 8, VEC>(static_cast<const T *>(is_k ? a.k : a.q) +
                            t * (is_k ? a.k_stride : a.q_stride) + uint64_t(hh) * a.dim + c0, x);
  float ss = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) ss += x[i] * x[i];
#pragma unroll
  for (int d = 1; d < L; d *= 2) ss += __shfl_xor(ss, d);
  if (weight && on) {
    const float r = rsqrtf(ss / float(a.dim) + a.eps);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = x[i] * r * bf16_to_f32(weight[c0 + i]);
  }
  const uint32_t half = a.rope.half;
  if (half) {
    const bool turned = on && c0 < 2 * half;
    const uint64_t at = uint64_t(turned ? table_row(a.rope, a.positions[t]) : 0) * half;
    if (a.rope.pairs) {
      if (turned) {
        float c[4], s[4];
        *reinterpret_cast<float4 *>(c) = *reinterpret_cast<const float4 *>(a.rope.cos + at + c0 / 2);
        *reinterpret_cast<float4 *>(s) = *reinterpret_cast<const float4 *>(a.rope.sin + at + c0 / 2);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float u = x[2 * i], v = x[2 * i + 1];
          x[2 * i] = u * c[i] - v * s[i];
          x[2 * i + 1] = v * c[i] + u * s[i];
        }
      }
    } else {
      const bool upper = c0 >= half;
      const uint32_t step = half / 8, lane = threadIdx.x & 63;
      const uint32_t other = turned ? (upper ? lane - step : lane + step) : lane;
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = __shfl(x[i], int(other));
      if (turned) {
        float c[8], s[8];
        const uint64_t o = at + (upper ? c0 - half : c0);
        load_row<float, 8, true>(a.rope.cos + o, c);
        load_row<float, 8, true>(a.rope.sin + o, s);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = x[i] * c[i] + (upper ? y[i] : -y[i]) * s[i];
      }
    }
  }
  if (on) {
    uint16_t *const out = (is_k ? a.k_out : a.q_out) +
                          (uint64_t(t) * (is_k ? a.k_heads : a.q_heads) + hh) * a.dim + c0;
    *reinterpret_cast<uint4 *>(out) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]),
                                                 pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
  }
}

template <typename T, bool VEC>
void launch_norm(const NormArgs &a, hipStream_t stream) {
  const uint64_t items = uint64_t(a.tokens) * (a.q_heads + a.k_heads);
  auto go = [&](auto kernel, uint32_t lanes) {
    hipLaunchKernelGGL(kernel, dim3(uint32_t((items * lanes + 255) / 256)), dim3(256), 0, stream,
                       a);
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
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) m = max(m, __float_as_uint(x[i]) & 0x7FFFFFFFu);
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
template <typename T, int D, bool VEC>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a, uint32_t groups) {
  constexpr int N = D / 8;           // channels a lane
  __shared__ __attribute__((aligned(16))) uint8_t lds[4][8][D / 2 + 4];
  const View &w = a.w;
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t s = blockIdx.y;
  const uint32_t item = blockIdx.x * 4 + wave;  // (group, head), heads within groups
  const Seq q = sequence(w, s);
  const uint32_t h = item % w.kv_heads;
  const int32_t first = (max(q.base, 0) & ~7) + 8 * int32_t(item / w.kv_heads);
  const int32_t end = min(q.base + q.count, int32_t(w.max_len));
  int32_t page = -1;
  if (item < groups * w.kv_heads && q.count > 0 && first < end)
    page = eq_dev::uniform(page_of(w, s, first));
  const uint32_t t = lane >> 3, sub = lane & 7, e0 = sub * N;
  const int32_t pos = first + int32_t(t);
  const bool on = page >= 0 && pos >= q.base && pos < end;
  const uint32_t slot = uint32_t(pos) & ((1u << w.page_shift) - 1);
  uint8_t *const part = w.pages + uint64_t(max(page, 0)) * w.page_bytes + uint64_t(h) * w.head_bytes;
  const uint64_t row = on ? uint64_t(q.row) + (pos - q.base) : 0;
  float x[N] = {};
  if (on) {
    const T *const kr = static_cast<const T *>(a.k) + row * a.k_stride + uint64_t(h) * D;
    load_row<T, N, VEC>(kr + e0, x);
    if (a.rope.half) rotate_key<T, N, VEC>(a.rope, kr, e0, a.positions ? a.positions[row] : pos, x);
  }
  constexpr int kPerBlock = 32 / N;  // lanes of a key group
  uint32_t b = scale_byte(group_top<N, kPerBlock>(x));
  if (on) {
    uint32_t *const kc = reinterpret_cast<uint32_t *>(part + slot * (D / 2) + e0 / 2);
#pragma unroll
    for (int i = 0; i < N / 8; ++i) kc[i] = codes8(x + 8 * i, b);
    if (sub % kPerBlock == 0)
      part[w.ks_off + slot / 16 * (D / 2) + (slot % 4 * (D / 32) + sub / kPerBlock) * 4 +
           slot % 16 / 4] = uint8_t(b);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = 0.0f;
    load_row<T, N, VEC>(static_cast<const T *>(a.v) + row * a.v_stride + uint64_t(h) * D + e0, x);
  }
  b = scale_byte(group_top<N, 8>(x));
  if (on && sub == 0) part[w.vs_off + slot] = uint8_t(b);
#pragma unroll
  for (int i = 0; i < N / 8; ++i)
    *reinterpret_cast<uint32_t *>(&lds[wave][t][e0 / 2 + 4 * i]) = codes8(x + 8 * i, b);
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

// The same 8 positions of a head for each wavefront as in append_kernel: keys
// a lane's D/8 channels of one token, values two channels of eight tokens (a
// dword each), which leave as whole rows.
template <int D>
__global__ __launch_bounds__(256) void read_kernel(View w, uint16_t *k, uint16_t *v,
                                                   uint32_t groups) {
  constexpr int N = D / 8;
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t s = blockIdx.y;
  const uint32_t item = blockIdx.x * 4 + wave;
  if (item >= groups * w.kv_heads) return;
  const Seq q = sequence(w, s);
  const uint32_t h = item % w.kv_heads;
  const int32_t first = (max(q.base, 0) & ~7) + 8 * int32_t(item / w.kv_heads);
  const int32_t end = min(q.base + q.count, int32_t(w.max_len));
  if (q.count <= 0 || first >= end) return;
  const int32_t page = eq_dev::uniform(page_of(w, s, first));
  if (page < 0) return;
  const uint32_t slot0 = uint32_t(first) & ((1u << w.page_shift) - 1);
  const uint8_t *const part = w.pages + uint64_t(page) * w.page_bytes + uint64_t(h) * w.head_bytes;
  auto out_row = [&](int32_t pos) {
    return ((uint64_t(q.row) + (pos - q.base)) * w.kv_heads + h) * D;
  };
  const uint32_t t = lane >> 3, sub = lane & 7, e0 = sub * N;
  const int32_t pos = first + int32_t(t);
  uint2 vc = make_uint2(0, 0);
  if (lane < D / 2) {
    const uint32_t *const p = reinterpret_cast<const uint32_t *>(
        part + w.v_off + (slot0 / 32 * D + 2 * lane) * 16 + slot0 % 32 / 2);
    vc = make_uint2(p[0], p[4]);
  }
  const uint2 vs = *reinterpret_cast<const uint2 *>(part + w.vs_off + slot0);
  if (pos >= q.base && pos < end) {
    const uint32_t slot = slot0 + t;
    const uint32_t *const kc = reinterpret_cast<const uint32_t *>(part + slot * (D / 2) + e0 / 2);
    const uint32_t b = part[w.ks_off + slot / 16 * (D / 2) + (slot % 4 * (D / 32) + e0 / 32) * 4 +
                            slot % 16 / 4];
    uint32_t *const out = reinterpret_cast<uint32_t *>(k + out_row(pos) + e0);
#pragma unroll
    for (int i = 0; i < N / 8; ++i) {
      const uint32_t c = kc[i];
      *reinterpret_cast<uint4 *>(out + 4 * i) =
          make_uint4(bf16_pair(c & 255, b), bf16_pair(c >> 8 & 255, b), bf16_pair(c >> 16 & 255, b),
                     bf16_pair(c >> 24, b));
    }
  }
  if (lane >= D / 2) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int32_t p = first + i;
    if (p < q.base || p >= end) continue;
    const uint32_t byte = (vc.x >> (4 * i) & 15) | (vc.y >> (4 * i) & 15) << 4;
    const uint32_t b = (i < 4 ? vs.x : vs.y) >> (8 * (i & 3)) & 255;
    *reinterpret_cast<uint32_t *>(v + out_row(p) + 2 * lane) = bf16_pair(byte, b);
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

// Groups of 8 aligned positions that `max_new` consecutive ones can touch.
uint32_t position_groups(uint32_t max_new) { return (max_new + 6) / 8 + 1; }

}  // namespace

extern "C" int eq_qk_norm_rope(const void *q, uint64_t q_stride, uint32_t q_heads,
                               const uint16_t *q_weight, uint16_t *q_out, const void *k,
                               uint64_t k_stride, uint32_t k_heads, const uint16_t *k_weight,
                               uint16_t *k_out, uint32_t dtype, uint32_t tokens, uint32_t head_dim,
                               float eps, const int32_t *positions, const eq_rope *rope,
                               hipStream_t stream) {
  const uint64_t heads = uint64_t(q_heads) + k_heads;
  if (dtype > EQ_BF16 || head_dim == 0 || head_dim % 16 || head_dim > 256 || q_heads > 4096 ||
      k_heads > 4096 || !rope_ok(rope, head_dim) || (rope && !positions) || !(eps >= 0.0f))
    return EQ_EINVAL;
  if ((q_heads && (!q || !q_out || (reinterpret_cast<uintptr_t>(q_out) & 15) ||
                   (tokens > 1 && q_stride < uint64_t(q_heads) * head_dim))) ||
      (k_heads && (!k || !k_out || (reinterpret_cast<uintptr_t>(k_out) & 15) ||
                   (tokens > 1 && k_stride < uint64_t(k_heads) * head_dim))))
    return EQ_EINVAL;
  if (tokens == 0 || heads == 0) return EQ_OK;
  if (uint64_t(tokens) * heads > (uint64_t(1) << 33)) return EQ_EINVAL;  // grid below 2^31
  const uint64_t item = dtype == EQ_F32 ? 4 : 2;
  NormArgs a{q, k, q_stride, k_stride, q_weight, k_weight, q_out, k_out, positions,
             device_rope(rope), tokens, q_heads, k_heads, head_dim, eps};
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

extern "C" int eq_kv_append(const eq_kv_cache *cache, const eq_kv_batch *batch, const void *k,
                            uint64_t k_stride, const void *v, uint64_t v_stride, uint32_t dtype,
                            const int32_t *positions, const eq_rope *rope, hipStream_t stream) {
  if (!batch_ok(cache, batch) || dtype > EQ_BF16 || !rope_ok(rope, cache->head_dim))
    return EQ_EINVAL;
  if (batch->n_seqs == 0 || batch->max_new == 0 || batch->max_len == 0) return EQ_OK;
  const uint64_t width = uint64_t(cache->kv_heads) * cache->head_dim;
  if (!k || !v || (batch->n_tokens > 1 && (k_stride < width || v_stride < width))) return EQ_EINVAL;
  AppendArgs a{view(cache, batch), k, v, k_stride, v_stride, positions, device_rope(rope)};
  const uint64_t item = dtype == EQ_F32 ? 4 : 2;
  const bool vec = aligned16(k, k_stride * item) && aligned16(v, v_stride * item);
  const uint32_t groups = position_groups(batch->max_new);
  const uint64_t blocks = (uint64_t(groups) * cache->kv_heads + 3) / 4;
  if (blocks > 0x7FFFFFFFu) return EQ_EINVAL;
  const dim3 grid(uint32_t(blocks), batch->n_seqs);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a, groups);
  };
  if (cache->head_dim == 128) {
    if (dtype == EQ_F32) vec ? go(append_kernel<float, 128, true>) : go(append_kernel<float, 128, false>);
    else vec ? go(append_kernel<uint16_t, 128, true>) : go(append_kernel<uint16_t, 128, false>);
  } else {
    if (dtype == EQ_F32) vec ? go(append_kernel<float, 64, true>) : go(append_kernel<float, 64, false>);
    else vec ? go(append_kernel<uint16_t, 64, true>) : go(append_kernel<uint16_t, 64, false>);
  }
  return done();
}

extern "C" int eq_kv_read(const eq_kv_cache *cache, const eq_kv_batch *batch, uint16_t *k,
                          uint16_t *v, hipStream_t stream) {
  if (!batch_ok(cache, batch)) return EQ_EINVAL;
  if (batch->n_seqs == 0 || batch->max_new == 0 || batch->max_len == 0) return EQ_OK;
  if (!k || !v || ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 15))
    return EQ_EINVAL;
  const uint32_t groups = position_groups(batch->max_new);
  const uint64_t blocks = (uint64_t(groups) * cache->kv_heads + 3) / 4;
  if (blocks > 0x7FFFFFFFu) return EQ_EINVAL;
  const dim3 grid(uint32_t(blocks), batch->n_seqs);
  if (cache->head_dim == 128)
    hipLaunchKernelGGL((read_kernel<128>), grid, dim3(256), 0, stream, view(cache, batch), k, v,
                       groups);
  else
    hipLaunchKernelGGL((read_kernel<64>), grid, dim3(256), 0, stream, view(cache, batch), k, v,
                       groups);
  return done();
}
