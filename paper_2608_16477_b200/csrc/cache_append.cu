// Keys and values of new tokens into the pages of a cache with the rotary position applied on the way, and the queries beside
// them turned into rows: what a decode step, or a chunk of a prefill, does between its projection and its attention.
//
// The same bits as the rotary operator on Q and K followed by the write of the rows (a turned key is rounded to the rows' type
// before it is quantised), with K read once and written once, and one launch.  HBM-bound: q twice, k and v once, the pages once.
//
// head_dim / 16 lanes own a row, two pieces of 8 values each, so placed that where pairs lie in halves a lane holds both members of
// its own.  A CTA takes all rows of a few tokens, or 16 (32) rows of one where there are few tokens; its threads form each (token,
// pair)'s sine and cosine once into shared memory while their first rows are on the way.  Small CTAs of few registers with one row to a
// lane in flight, ten to an SM, were better than more rows in flight or CTAs that stay (16,384 tokens of 32 query and 8 KV heads of 128,
// bf16 into e2m1 pages, 355 MB: 68 us against 73 to 104; 5.2 TB/s, 79 % of a copy's rate; the sines and cosines take 7 us of it, the
// conversion to e2m1 most of the rest).  One token of 64 / 8 heads 2.4 us, 64 tokens 3.0 us.
#include "cache_format.cuh"
#include "rope.cuh"

namespace kvr {
namespace {

constexpr int kAppendThreads = 128;
constexpr int kAppendTokens = 4;      // most tokens of a CTA
constexpr int kAppendMaxTokens = 1 << 30;

struct AppendParams {
  RowLayout layout;
  SlotMap map;
  int n_tokens, n_q, n_kv;
  int rotary, interleaved, tokens_per_cta, rows_per_cta;
  float gain;
  const int *positions;
  const long long *slots;
  const char *q, *k, *v;
  char *q_out;
  long long q_ts, q_hs, k_ts, k_hs, v_ts, v_hs, o_ts, o_hs;      // bytes
  double turns[kRopeMaxPairs];
};

// How the pairs of a head lie to the lanes' pieces.  Halves whose members begin at multiples of 16 dims, the head's rest as well
// (rotary_dim 32, 64, 96 or all of it): a lane's pieces are the two members of its pairs, or two pieces of the rest.  Interleaved pairs: a
// piece holds its pairs.  Other halves: a lane loads the other members from global memory.
enum { kHalves = 0, kInterleaved = 1, kAnyHalves = 2 };

// Turns a lane's pieces, which begin at dims `first` and `first` + `apart`.  cs: the token's (cos, sin), by pair (kHalves: by place_of).
template <typename T, int D, int MODE>
__device__ __forceinline__ void turn(Raw<T> &raw, const char *row, int first, int apart, int sub, int rotary, unsigned group, const float2 *cs) {
  const int half = rotary >> 1;
  float f[2][8];
  if (MODE == kHalves) {
    if (first >= half) return;      // the rest of the head
    raw.unpack(0, f[0]);
    raw.unpack(1, f[1]);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float4 w = *reinterpret_cast<const float4 *>(cs + (k * (D / 16) + sub) * 2);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float2 wi = i ? make_float2(w.z, w.w) : make_float2(w.x, w.y);
        const float a = f[0][2 * k + i], b = f[1][2 * k + i];
        f[0][2 * k + i] = turned_first(a, b, wi);
        f[1][2 * k + i] = turned_second(a, b, wi);
      }
    }
    raw.pack(0, f[0]);
    raw.pack(1, f[1]);
  } else if (MODE == kInterleaved) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int e0 = first + h * apart;
      if (e0 >= rotary) continue;
      raw.unpack(h, f[h]);
#pragma unroll
      for (int i = 0; i < 8; i += 4) {
        const float4 w = *reinterpret_cast<const float4 *>(cs + (e0 + i) / 2);      // two pairs; past the last one: not used
        const bool front = (e0 + i) * (int)sizeof(T) % 32 < 16;
        const float a0 = f[h][i], b0 = f[h][i + 1], a1 = f[h][i + 2], b1 = f[h][i + 3];
        if (e0 + i < rotary) {
          f[h][i] = turned_first(a0, b0, make_float2(w.x, w.y));
          f[h][i + 1] = front ? turned_neighbour(a0, b0, make_float2(w.x, w.y)) : turned_second(a0, b0, make_float2(w.x, w.y));
        }
        if (e0 + i + 2 < rotary) {
          f[h][i + 2] = turned_first(a1, b1, make_float2(w.z, w.w));
          f[h][i + 3] = front ? turned_neighbour(a1, b1, make_float2(w.z, w.w)) : turned_second(a1, b1, make_float2(w.z, w.w));
        }
      }
      raw.pack(h, f[h]);
    }
  } else {
    float other[2][8];
    raw.unpack(0, f[0]);
    raw.unpack(1, f[1]);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int e = first + h * apart + i;
        other[h][i] = e < rotary ? (float)reinterpret_cast<const T *>(row)[e < half ? e + half : e - half] : 0.f;
      }
    __syncwarp(group);      // the row may be overwritten in place from here on
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int e = first + h * apart + i;
        if (e < half)
          f[h][i] = turned_first(f[h][i], other[h][i], cs[e]);
        else if (e < rotary)
          f[h][i] = turned_second(other[h][i], f[h][i], cs[e - half]);
      }
    raw.pack(0, f[0]);
    raw.pack(1, f[1]);
  }
}

// Place of pair j of a head turned in halves, so that the 16-byte loads of a row's lanes (pairs 8 sub, ... + 7) follow one another.
template <int D>
__device__ __forceinline__ int place_of(int j) {
  return ((((j & 7) >> 1) * (D / 16) + (j >> 3)) << 1) + (j & 1);
}

template <typename T, int D, int FMT, int MODE>
__global__ void __launch_bounds__(kAppendThreads, sizeof(T) == 2 ? 10 : 8) cache_append_kernel(const __grid_constant__ AppendParams p) {
  constexpr int LPR = D / 16, ROWS = kAppendThreads / LPR;
  __shared__ __align__(16) float2 cs[kAppendTokens][kRopeMaxPairs];
  __shared__ long long block_s[kAppendTokens];      // of a token's slot: the block's place (-1: outside the pool), and the offset in it
  __shared__ int offset_s[kAppendTokens];
  const int t0 = blockIdx.x * p.tokens_per_cta, nt = min(p.tokens_per_cta, p.n_tokens - t0);
  const int rows = p.n_q + 2 * p.n_kv, r0 = blockIdx.y * p.rows_per_cta, nr = min(p.rows_per_cta, rows - r0);
  const int sub = threadIdx.x % LPR, half = p.rotary >> 1;
  const int first = MODE != kHalves || sub < half / 8 ? sub * 8 : p.rotary + sub * 8 - half;      // dims of the lane's pieces
  const int apart = MODE != kHalves ? D / 2 : sub < half / 8 ? half : (D - p.rotary) / 2;
  const unsigned group = ((1u << LPR) - 1u) << (threadIdx.x & 31 & ~(LPR - 1));

  // Row `at` of a token: K's heads come first, then V's, then the queries'.
  int token = 0, at = threadIdx.x / LPR;
  auto settle = [&]() {
    while (at >= nr) {
      at -= nr;
      ++token;
    }
  };
  settle();
  Raw<T> x;
  const char *src = nullptr;
  auto load = [&]() {
    const int row = r0 + at;
    const long long t = t0 + token;
    src = row < p.n_kv ? p.k + t * p.k_ts + row * p.k_hs
                       : row < 2 * p.n_kv ? p.v + t * p.v_ts + (row - p.n_kv) * p.v_hs : p.q + t * p.q_ts + (row - 2 * p.n_kv) * p.q_hs;
    x.load(src + first * (int)sizeof(T), apart * (int)sizeof(T));
  };
  if (token < nt) load();      // under the trigonometry
  for (int i = threadIdx.x; i < nt * half; i += kAppendThreads) {
    const int t = i / half, j = i - t * half;
    cs[t][MODE == kHalves ? place_of<D>(j) : j] = rope_turn(p.positions[t0 + t], p.turns[j], p.gain, 1.f);
  }
  if (threadIdx.x < nt) {
    int block, offset;
    const bool live = p.map.split(p.slots[t0 + threadIdx.x], block, offset);
    block_s[threadIdx.x] = live ? block * p.layout.block_stride : -1;
    offset_s[threadIdx.x] = offset;
  }
  __syncthreads();
  while (token < nt) {
    const int row = r0 + at, kind = row < p.n_kv ? 0 : row < 2 * p.n_kv ? 1 : 2;      // K, V, Q
    if (kind != 1) turn<T, D, MODE>(x, src, first, apart, sub, p.rotary, group, cs[token]);
    if (kind == 2) {
      char *to = p.q_out + (long long)(t0 + token) * p.o_ts + (row - 2 * p.n_kv) * p.o_hs + first * (int)sizeof(T);
      float f[8];
      x.unpack(0, f);
      store8(to, f, T());
      x.unpack(1, f);
      store8(to + apart * (int)sizeof(T), f, T());
    } else {
      const long long block = block_s[token];
      const Pieces<D, FMT> to(p.layout, kind, row - kind * p.n_kv, first);
      put_row<T, D, FMT>(x, to, p.layout.slot_stride, apart, block, offset_s[token], sub, group, block >= 0);
    }
    at += ROWS;
    settle();
    if (token < nt) load();
  }
}

template <typename T, int D, int FMT>
int launch_append(AppendParams &p, cudaStream_t st) {
  constexpr int ROWS = kAppendThreads / (D / 16);
  const int device = current_device();
  if (device < 0) return KV_ERR_CUDA;
  const int sms = sm_count(device), rows = p.n_q + 2 * p.n_kv;
  // Whole tokens to a CTA once there are four for each SM, as many as give a lane three rows; below that a token's rows are
  // spread over CTAs.
  const bool whole_tokens = p.n_tokens >= 4 * sms;
  p.rows_per_cta = whole_tokens || rows < ROWS ? rows : ROWS;
  p.tokens_per_cta = 1;
  if (whole_tokens)
    while (p.tokens_per_cta < kAppendTokens && p.tokens_per_cta * rows < 3 * ROWS &&
           (p.n_tokens + 2 * p.tokens_per_cta - 1) / (2 * p.tokens_per_cta) >= 4 * sms)
      p.tokens_per_cta *= 2;
  const dim3 grid((p.n_tokens + p.tokens_per_cta - 1) / p.tokens_per_cta, (rows + p.rows_per_cta - 1) / p.rows_per_cta);
  if (grid.y > 65535) return KV_ERR_SHAPE;
  if (p.interleaved)
    cache_append_kernel<T, D, FMT, kInterleaved><<<grid, kAppendThreads, 0, st>>>(p);
  else if (p.rotary % 32 == 0 && (D - p.rotary) % 32 == 0)
    cache_append_kernel<T, D, FMT, kHalves><<<grid, kAppendThreads, 0, st>>>(p);
  else
    cache_append_kernel<T, D, FMT, kAnyHalves><<<grid, kAppendThreads, 0, st>>>(p);
  KV_COUNT_LAUNCH();
  KV_CUDA(cudaGetLastError());
  return KV_OK;
}

template <int FMT>
int append_format(AppendParams &p, int d, bool f32, cudaStream_t st) {
  if (d == 128) return f32 ? launch_append<float, 128, FMT>(p, st) : launch_append<bf16, 128, FMT>(p, st);
  return f32 ? launch_append<float, 64, FMT>(p, st) : launch_append<bf16, 64, FMT>(p, st);
}

}  // namespace
}  // namespace kvr

extern "C" {

int32_t kv_op_cache_append(const kv_rope *rope, const kv_cache_desc *cache, int32_t layer, const void *q_dev, int64_t q_token_stride,
                           int64_t q_head_stride, int32_t n_q_heads, void *q_out_dev, int64_t q_out_token_stride,
                           int64_t q_out_head_stride, const void *k_dev, int64_t k_token_stride, int64_t k_head_stride,
                           const void *v_dev, int64_t v_token_stride, int64_t v_head_stride, int32_t dtype, int32_t n_tokens,
                           const int32_t *positions_dev, const int64_t *slots_dev, void *stream) {
  using namespace kvr;
  if (rope == nullptr || n_tokens < 0 || n_q_heads < 0 || (dtype != KV_DTYPE_BF16 && dtype != KV_DTYPE_F32)) return KV_ERR_ARG;
  int rc = check_cache_desc(cache, true);
  if (rc != KV_OK) return rc;
  const int d = cache->head_dim;
  if (d != 64 && d != 128) return KV_ERR_SHAPE;
  if (layer < 0 || layer >= cache->n_layers || rope->d.rotary_dim > d || n_tokens > kAppendMaxTokens) return KV_ERR_SHAPE;
  if ((long long)n_q_heads + 2ll * cache->n_kv_heads > 1 << 20) return KV_ERR_SHAPE;      // rows of a token are counted in 32 bits
  if (n_tokens == 0) return KV_OK;
  if (k_dev == nullptr || v_dev == nullptr || positions_dev == nullptr || slots_dev == nullptr) return KV_ERR_ARG;
  if (n_q_heads > 0 && (q_dev == nullptr || q_out_dev == nullptr)) return KV_ERR_ARG;
  const int size = dtype == KV_DTYPE_BF16 ? 2 : 4;
  if (n_q_heads == 0) q_token_stride = q_head_stride = q_out_token_stride = q_out_head_stride = 0;
  const int64_t strides[8] = {k_token_stride, k_head_stride, v_token_stride, v_head_stride,
                              q_token_stride, q_head_stride, q_out_token_stride, q_out_head_stride};
  for (int64_t s : strides)
    if (s < 0 || s * size % 16 != 0) return KV_ERR_ARG;
  if (((uintptr_t)k_dev & 15) || ((uintptr_t)v_dev & 15) || ((uintptr_t)slots_dev & 7) || ((uintptr_t)positions_dev & 3)) return KV_ERR_ARG;
  if (n_q_heads > 0) {
    if (((uintptr_t)q_dev & 15) || ((uintptr_t)q_out_dev & 15)) return KV_ERR_ARG;
    if (!rows_disjoint(q_out_token_stride, q_out_head_stride, n_tokens, n_q_heads, d)) return KV_ERR_ARG;
    if (q_dev == q_out_dev && (q_token_stride != q_out_token_stride || q_head_stride != q_out_head_stride)) return KV_ERR_ARG;
  }
  AppendParams p;
  p.layout = row_layout(make_view(cache), layer);
  p.map = slot_map(cache);
  p.n_tokens = n_tokens;
  p.n_q = n_q_heads;
  p.n_kv = cache->n_kv_heads;
  p.rotary = rope->d.rotary_dim;
  p.interleaved = rope->d.layout == KV_ROPE_INTERLEAVED;
  p.gain = (float)rope->d.gain;
  p.positions = positions_dev;
  p.slots = reinterpret_cast<const long long *>(slots_dev);
  p.q = (const char *)q_dev;
  p.k = (const char *)k_dev;
  p.v = (const char *)v_dev;
  p.q_out = (char *)q_out_dev;
  p.q_ts = q_token_stride * size;
  p.q_hs = q_head_stride * size;
  p.k_ts = k_token_stride * size;
  p.k_hs = k_head_stride * size;
  p.v_ts = v_token_stride * size;
  p.v_hs = v_head_stride * size;
  p.o_ts = q_out_token_stride * size;
  p.o_hs = q_out_head_stride * size;
  for (int j = 0; j < kRopeMaxPairs; ++j) p.turns[j] = j < p.rotary / 2 ? rope->turns[j] : 0.0;
  const bool f32 = dtype == KV_DTYPE_F32;
  cudaStream_t st = (cudaStream_t)stream;
  switch (format_of(cache->elem_bytes)) {
    case kBf16: return append_format<kBf16>(p, d, f32, st);
    case kE4m3: return append_format<kE4m3>(p, d, f32, st);
    default: return append_format<kE2m1>(p, d, f32, st);
  }
}

}  // extern "C"
