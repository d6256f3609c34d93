// Rotary positions on rows of heads: half or interleaved pairs, part of the head, scaled frequencies, forward and
// transposed.
//
// (y_a, y_b) = gain * (a cos - b sin, b cos + a sin) with the angle p * theta_j.  The angle is formed in TURNS,
// p * (theta_j / 2 pi), in fp64 and reduced to [-1/2, 1/2] there; the remainder goes to fp32 sincospi.  That costs three
// fp64 operations instead of an fp64 sine and cosine and, with theta_j <= 1, is exact to 2^-24 of a turn for every int32
// position (2^31 / 2 pi turns are less than 2^29, where fp64 has steps of 2^-24).
//
// HBM-bound: 2 * rows * head_dim elements move (3 fma per element).  A token's cosines and sines are needed by all its
// heads, so a CTA takes one or two whole tokens, its threads form each (token, pair) once into shared memory, and the heads
// are then streamed: one thread owns 2 x 16 bytes of a head (both members of its pairs), neighbouring threads
// neighbouring vectors.  Measured in a graph / call after call in a stream: 16,384 tokens of 72 heads of 128, bf16, 604 MB:
// 98 / 100 us, 6.2 / 6.0 TB/s (94 / 92 % of a copy's rate; 102 to 108 us after seconds of it, when the power cap has taken the
// clock from 1.97 to 1.8 GHz); 1,003 tokens of 40 heads, fp32, 41 MB: 8.6 / 10.2 us; one token 2.5 / 6.7 us.
#include <float.h>

#include <cmath>
#include <new>

#include "rope.cuh"

namespace kvr {
namespace {

constexpr int kRopeThreads = 128;
constexpr int kRopeMaxTokens = 2;   // tokens of a CTA (16,384 tokens of 72 heads: 97.7 us with two, 102 us with four)
constexpr int kRopeAhead = 3;       // heads of a thread whose loads are in flight together

struct RopeParams {
  const void *x;
  void *out;
  long long x_ts, x_hs, o_ts, o_hs;   // strides, elements
  const int *positions;
  int n_tokens, n_heads, head_dim, rotary, interleaved;
  int tokens_per_cta, heads_per_cta;
  float gain, sign;                   // sign = -1: transposed
  double turns[kRopeMaxPairs];
};

template <typename T>
struct Vec;   // 16 bytes as floats
template <>
struct Vec<float> {
  static constexpr int n = 4;
  static __device__ __forceinline__ void unpack(uint4 r, float (&f)[4]) {
    f[0] = __uint_as_float(r.x); f[1] = __uint_as_float(r.y); f[2] = __uint_as_float(r.z); f[3] = __uint_as_float(r.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
};
template <>
struct Vec<bf16> {
  static constexpr int n = 8;
  static __device__ __forceinline__ void unpack(uint4 r, float (&f)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t *>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// cosines and sines (times gain) of the CTA's tokens: cs[token][pair]
__device__ __forceinline__ void rope_table_of(const RopeParams &p, int t0, int nt, float2 (*cs)[kRopeMaxPairs]) {
  const int half = p.rotary >> 1;
  for (int i = threadIdx.x; i < nt * half; i += kRopeThreads) {
    const int t = i / half, j = i - t * half;
    cs[t][j] = rope_turn(p.positions[t0 + t], p.turns[j], p.gain, p.sign);
  }
}

// Rows that can be read as 16-byte vectors whose members are whole pairs: interleaved pairs always (the vector at the end
// of the rotated part is rotated pair by pair), halves if rotary / 2 is a multiple of the vector length.
template <typename T, bool INTERLEAVED>
__global__ void __launch_bounds__(kRopeThreads) rope_vec_kernel(const __grid_constant__ RopeParams p) {
  constexpr int VE = Vec<T>::n;
  __shared__ __align__(16) float2 cs[kRopeMaxTokens][kRopeMaxPairs];
  const int t0 = blockIdx.x * p.tokens_per_cta, nt = min(p.tokens_per_cta, p.n_tokens - t0);
  const int h0 = blockIdx.y * p.heads_per_cta, nh = min(p.heads_per_cta, p.n_heads - h0);
  const int half = p.rotary >> 1;
  const int turned = (p.rotary + 2 * VE - 1) / (2 * VE);                   // threads of a head that rotate
  const int rest = turned * 2 * VE;                                        // first element that is only copied
  const int units = turned + (p.head_dim > rest ? (p.head_dim - rest + 2 * VE - 1) / (2 * VE) : 0);
  const int lanes = kRopeThreads / units;                                  // heads in flight
  const int u = threadIdx.x % units, slot = threadIdx.x / units;
  const bool idle = slot >= lanes;
  const bool in_place = p.x == p.out;
  const T *x = static_cast<const T *>(p.x);
  T *out = static_cast<T *>(p.out);
  // elements of the two vectors inside the head
  const int e0 = u < turned ? (INTERLEAVED ? u * 2 * VE : u * VE) : rest + (u - turned) * 2 * VE;
  const int e1 = u < turned && !INTERLEAVED ? e0 + half : e0 + VE;
  const bool two = e1 < p.head_dim;
  const bool copies = u >= turned;
  const int items = idle || (copies && in_place) ? 0 : nt * nh;

  uint4 a[kRopeAhead], b[kRopeAhead] = {};
  auto load = [&](int first) {
#pragma unroll
    for (int i = 0; i < kRopeAhead; ++i) {
      const int it = first + i * lanes;
      if (it >= items) break;
      const int t = it / nh, h = it - t * nh;
      const T *row = x + (t0 + t) * p.x_ts + (h0 + h) * p.x_hs;
      a[i] = *reinterpret_cast<const uint4 *>(row + e0);
      if (two) b[i] = *reinterpret_cast<const uint4 *>(row + e1);
    }
  };
  auto turn = [&](int it, const uint4 &ca, const uint4 &cb) {
    const int t = it / nh, h = it - t * nh;
    T *row = out + (t0 + t) * p.o_ts + (h0 + h) * p.o_hs;
    if (copies) {
      *reinterpret_cast<uint4 *>(row + e0) = ca;
      if (two) *reinterpret_cast<uint4 *>(row + e1) = cb;
      return;
    }
    float fa[VE], fb[VE];
    Vec<T>::unpack(ca, fa);
    Vec<T>::unpack(cb, fb);
    const float2 *w = cs[t] + u * VE;
    if (INTERLEAVED) {
#pragma unroll
      for (int i = 0; i < VE; i += 2) {
        const float2 w0 = w[i / 2], w1 = w[VE / 2 + i / 2];
        const float x0 = fa[i], y0 = fa[i + 1], x1 = fb[i], y1 = fb[i + 1];
        if (u * VE + i / 2 < half) {
          fa[i] = turned_first(x0, y0, w0);
          fa[i + 1] = turned_neighbour(x0, y0, w0);
        }
        if (u * VE + VE / 2 + i / 2 < half) {
          fb[i] = turned_first(x1, y1, w1);
          fb[i + 1] = turned_second(x1, y1, w1);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        const float2 wi = w[i];
        const float xa = fa[i], xb = fb[i];
        fa[i] = turned_first(xa, xb, wi);
        fb[i] = turned_second(xa, xb, wi);
      }
    }
    *reinterpret_cast<uint4 *>(row + e0) = Vec<T>::pack(fa);
    if (two) *reinterpret_cast<uint4 *>(row + e1) = Vec<T>::pack(fb);
  };
  load(slot);      // under the trigonometry
  rope_table_of(p, t0, nt, cs);
  __syncthreads();
  for (int first = slot; first < items; first += kRopeAhead * lanes) {
    if (first > slot) load(first);
#pragma unroll
    for (int i = 0; i < kRopeAhead; ++i)
      if (first + i * lanes < items) turn(first + i * lanes, a[i], b[i]);
  }
}

// Halves whose members do not start on the same place of a vector (rotary / 2 no multiple of its length), in rows that can
// be read as vectors all the same: a warp takes up to eight heads of a token through shared memory, vectors in and out, pairs
// in between (8,000 tokens of 72 heads of 128, 102 rotated: 70 us, against 255 us with a thread per pair straight from
// global memory; 45 us of bytes, 53 us where all 128 are rotated: a warp's loads, turns and stores follow one another with
// nothing in flight meanwhile, and its pairs are read from shared memory two bytes at a time).
constexpr int kRopeRowBytes = 4096;      // of a warp
template <typename T>
__global__ void __launch_bounds__(kRopeThreads) rope_row_kernel(const __grid_constant__ RopeParams p) {
  constexpr int VE = Vec<T>::n;
  __shared__ __align__(16) float2 cs[kRopeMaxTokens][kRopeMaxPairs];
  __shared__ __align__(16) uint4 rows_s[kRopeThreads / 32][kRopeRowBytes / 16];
  const int t0 = blockIdx.x * p.tokens_per_cta, nt = min(p.tokens_per_cta, p.n_tokens - t0);
  const int h0 = blockIdx.y * p.heads_per_cta, nh = min(p.heads_per_cta, p.n_heads - h0);
  const int half = p.rotary >> 1, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int vecs = p.head_dim / VE;
  const int at_once = min(8, kRopeRowBytes / (p.head_dim * (int)sizeof(T)));
  const int groups = (nh + at_once - 1) / at_once;
  const T *x = static_cast<const T *>(p.x);
  T *out = static_cast<T *>(p.out);
  uint4 *buf = rows_s[warp];
  T *vals = reinterpret_cast<T *>(buf);
  rope_table_of(p, t0, nt, cs);
  __syncthreads();
  for (int it = warp; it < nt * groups; it += kRopeThreads / 32) {
    const int t = it / groups, first = (it - t * groups) * at_once, n = min(at_once, nh - first);
    const T *src = x + (t0 + t) * p.x_ts + (h0 + first) * p.x_hs;
    T *dst = out + (t0 + t) * p.o_ts + (h0 + first) * p.o_hs;
#pragma unroll 4
    for (int v = lane; v < n * vecs; v += 32) {
      const int r = v / vecs;
      buf[v] = *reinterpret_cast<const uint4 *>(src + r * p.x_hs + (v - r * vecs) * VE);
    }
    __syncwarp();
    for (int j = lane; j < half; j += 32) {
      const float2 w = cs[t][j];
#pragma unroll 4
      for (int r = 0; r < n; ++r) {
        T *row = vals + r * p.head_dim;
        const float a = (float)row[j], b = (float)row[j + half];
        row[j] = (T)turned_first(a, b, w);
        row[j + half] = (T)turned_second(a, b, w);
      }
    }
    __syncwarp();
#pragma unroll 4
    for (int v = lane; v < n * vecs; v += 32) {
      const int r = v / vecs;
      *reinterpret_cast<uint4 *>(dst + r * p.o_hs + (v - r * vecs) * VE) = buf[v];
    }
    __syncwarp();
  }
}

// Any alignment: a thread per pair or per copied element.
template <typename T, bool INTERLEAVED>
__global__ void __launch_bounds__(kRopeThreads) rope_any_kernel(const __grid_constant__ RopeParams p) {
  __shared__ float2 cs[kRopeMaxTokens][kRopeMaxPairs];
  const int t0 = blockIdx.x * p.tokens_per_cta, nt = min(p.tokens_per_cta, p.n_tokens - t0);
  const int h0 = blockIdx.y * p.heads_per_cta, nh = min(p.heads_per_cta, p.n_heads - h0);
  rope_table_of(p, t0, nt, cs);
  __syncthreads();
  const int half = p.rotary >> 1, units = half + p.head_dim - p.rotary;
  const T *x = static_cast<const T *>(p.x);
  T *out = static_cast<T *>(p.out);
  for (int it = threadIdx.x; it < nt * nh * units; it += kRopeThreads) {
    const int u = it % units, th = it / units;
    const int t = th / nh, h = th - t * nh;
    const T *src = x + (t0 + t) * p.x_ts + (h0 + h) * p.x_hs;
    T *dst = out + (t0 + t) * p.o_ts + (h0 + h) * p.o_hs;
    if (u >= half) {
      const int e = p.rotary + u - half;
      dst[e] = src[e];
      continue;
    }
    const int ea = INTERLEAVED ? 2 * u : u, eb = INTERLEAVED ? 2 * u + 1 : u + half;
    const float2 w = cs[t][u];
    const float a = (float)src[ea], b = (float)src[eb];
    dst[ea] = (T)turned_first(a, b, w);
    dst[eb] = (T)turned_second(a, b, w);
  }
}

template <typename T>
int launch_rope(RopeParams &p, cudaStream_t st) {
  constexpr int VE = Vec<T>::n;
  const int half = p.rotary / 2;
  const bool aligned = (((uintptr_t)p.x | (uintptr_t)p.out) & 15) == 0 &&
                       ((p.x_ts | p.x_hs | p.o_ts | p.o_hs) % VE) == 0 && p.head_dim % VE == 0;
  const bool vec = aligned && (p.interleaved || half % VE == 0);
  const int device = current_device();
  if (device < 0) return KV_ERR_CUDA;
  const int sms = sm_count(device);
  // whole tokens per CTA while there are at least four CTAs per SM of them; fewer tokens than that: the heads of a token
  // are split as well, 32 to a CTA, and 16 when there are hardly any tokens (one token of 72 heads 2.5 us against 2.65 us)
  p.tokens_per_cta = kRopeMaxTokens;
  while (p.tokens_per_cta > 1 && (p.n_tokens + p.tokens_per_cta - 1) / p.tokens_per_cta < 4 * sms) p.tokens_per_cta >>= 1;
  const int heads = p.n_tokens >= 4 * sms ? 1024 : (p.n_tokens >= 64 ? 32 : 16);
  p.heads_per_cta = p.n_heads < heads ? p.n_heads : heads;
  const dim3 grid((p.n_tokens + p.tokens_per_cta - 1) / p.tokens_per_cta,
                  (p.n_heads + p.heads_per_cta - 1) / p.heads_per_cta);
  if (grid.y > 65535) return KV_ERR_SHAPE;
  if (vec && p.interleaved)
    rope_vec_kernel<T, true><<<grid, kRopeThreads, 0, st>>>(p);
  else if (vec)
    rope_vec_kernel<T, false><<<grid, kRopeThreads, 0, st>>>(p);
  else if (aligned)
    rope_row_kernel<T><<<grid, kRopeThreads, 0, st>>>(p);
  else if (p.interleaved)
    rope_any_kernel<T, true><<<grid, kRopeThreads, 0, st>>>(p);
  else
    rope_any_kernel<T, false><<<grid, kRopeThreads, 0, st>>>(p);
  KV_COUNT_LAUNCH();
  KV_CUDA(cudaGetLastError());
  return KV_OK;
}

bool positive(double v) { return std::isfinite(v) && v > 0.0; }

}  // namespace
}  // namespace kvr

extern "C" {

int32_t kv_rope_create(const kv_rope_desc *desc, kv_rope **out) {
  using namespace kvr;
  if (desc == nullptr || out == nullptr) return KV_ERR_ARG;
  const kv_rope_desc &d = *desc;
  if (d.rotary_dim <= 0 || d.rotary_dim % 2 != 0 || d.rotary_dim > 2 * kRopeMaxPairs) return KV_ERR_SHAPE;
  if (d.layout != KV_ROPE_HALF && d.layout != KV_ROPE_INTERLEAVED) return KV_ERR_ARG;
  if (d.scaling < KV_ROPE_SCALE_NONE || d.scaling > KV_ROPE_SCALE_PARTS) return KV_ERR_ARG;
  if (!positive(d.base) || !(d.gain >= FLT_MIN && d.gain <= FLT_MAX)) return KV_ERR_ARG;      // the kernels' gain is fp32
  if (d.scaling != KV_ROPE_SCALE_NONE && !positive(d.factor)) return KV_ERR_ARG;
  if (d.scaling == KV_ROPE_SCALE_NTK && d.rotary_dim <= 2) return KV_ERR_SHAPE;
  if (d.scaling == KV_ROPE_SCALE_PARTS &&
      (!positive(d.original_ctx) || !std::isfinite(d.low) || !std::isfinite(d.high) || !(d.high > d.low)))
    return KV_ERR_ARG;
  const int half = d.rotary_dim / 2;
  const double two_pi = 6.283185307179586476925;
  double base = d.base;
  if (d.scaling == KV_ROPE_SCALE_NTK) base *= std::pow(d.factor, (double)d.rotary_dim / (d.rotary_dim - 2));
  if (!positive(base)) return KV_ERR_ARG;
  kv_rope *r = new (std::nothrow) kv_rope();
  if (r == nullptr) return KV_ERR_ARG;
  r->d = d;
  for (int j = 0; j < half; ++j) {
    double theta = std::pow(base, -(double)j / half);
    if (d.scaling == KV_ROPE_SCALE_LINEAR) theta /= d.factor;
    if (d.scaling == KV_ROPE_SCALE_PARTS) {
      double g = (d.original_ctx * theta / two_pi - d.low) / (d.high - d.low);
      g = g < 0.0 ? 0.0 : (g > 1.0 ? 1.0 : g);
      theta = (1.0 - g) * theta / d.factor + g * theta;
    }
    if (!(theta <= 1.0)) {      // what the reduction of the angle in turns counts on
      delete r;
      return KV_ERR_ARG;
    }
    r->theta[j] = theta;
    r->turns[j] = theta / two_pi;
  }
  *out = r;
  return KV_OK;
}

int32_t kv_rope_destroy(kv_rope *r) {
  delete r;
  return KV_OK;
}

int32_t kv_rope_frequencies(const kv_rope *r, double *theta_host, int32_t n) {
  if (r == nullptr || theta_host == nullptr || n < r->d.rotary_dim / 2) return KV_ERR_ARG;
  for (int j = 0; j < r->d.rotary_dim / 2; ++j) theta_host[j] = r->theta[j];
  return KV_OK;
}

int32_t kv_op_rope(const kv_rope *rope, const void *x_dev, int64_t x_token_stride, int64_t x_head_stride, int32_t dtype,
                   int32_t n_tokens, int32_t n_heads, int32_t head_dim, const int32_t *positions_dev, int32_t backward,
                   void *out_dev, int64_t out_token_stride, int64_t out_head_stride, void *stream) {
  using namespace kvr;
  if (rope == nullptr || n_tokens < 0 || n_heads <= 0 || head_dim <= 0) return KV_ERR_ARG;
  if (dtype != KV_DTYPE_BF16 && dtype != KV_DTYPE_F32) return KV_ERR_ARG;
  if (head_dim < rope->d.rotary_dim || head_dim > 1024) return KV_ERR_SHAPE;
  if (n_tokens == 0) return KV_OK;
  if (x_dev == nullptr || out_dev == nullptr || positions_dev == nullptr) return KV_ERR_ARG;
  const uintptr_t elem = dtype == KV_DTYPE_BF16 ? 1 : 3;
  if (((uintptr_t)x_dev & elem) || ((uintptr_t)out_dev & elem) || ((uintptr_t)positions_dev & 3)) return KV_ERR_ARG;
  if (x_token_stride < 0 || x_head_stride < 0) return KV_ERR_ARG;
  if (!rows_disjoint(out_token_stride, out_head_stride, n_tokens, n_heads, head_dim)) return KV_ERR_ARG;
  if (x_dev == out_dev && (x_token_stride != out_token_stride || x_head_stride != out_head_stride)) return KV_ERR_ARG;
  RopeParams p;
  p.x = x_dev;
  p.out = out_dev;
  p.x_ts = x_token_stride;
  p.x_hs = x_head_stride;
  p.o_ts = out_token_stride;
  p.o_hs = out_head_stride;
  p.positions = positions_dev;
  p.n_tokens = n_tokens;
  p.n_heads = n_heads;
  p.head_dim = head_dim;
  p.rotary = rope->d.rotary_dim;
  p.interleaved = rope->d.layout == KV_ROPE_INTERLEAVED;
  p.gain = (float)rope->d.gain;
  p.sign = backward ? -1.f : 1.f;
  for (int j = 0; j < kRopeMaxPairs; ++j) p.turns[j] = j < p.rotary / 2 ? rope->turns[j] : 0.0;
  if (dtype == KV_DTYPE_BF16) return launch_rope<bf16>(p, (cudaStream_t)stream);
  return launch_rope<float>(p, (cudaStream_t)stream);
}

}  // extern "C"
