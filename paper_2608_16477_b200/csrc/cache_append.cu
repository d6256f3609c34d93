// Keys and values of new tokens into the pages of a cache with the rotary position applied on the way, and the queries beside
// them turned into rows: what a decode step, or a chunk of a prefill, does between its projection and its attention.
//
// The same bits as the rotary operator on Q and K followed by the write of the rows (a turned key is rounded to the rows' type
// before it is quantised), with K read once and written once, and one launch.  HBM-bound: q twice, k and v once, the pages once.
//
// head_dim / 16 lanes own a row, two pieces of 8 values each half a row apart, as in the write of rows; where the whole head turns in
// halves both members of a pair are the lane's own.  Other pairs have their partner loaded once more (from L1, mostly).  A CTA takes
// all rows of a few tokens, or 32 (64) rows of one where there are few tokens; its threads form each (token, pair)'s sine and cosine
// once into shared memory while their first rows are on the way.
#include "cache_format.cuh"
#include "rope.cuh"

namespace kvr {
namespace {

constexpr int kAppendThreads = 256;
constexpr int kAppendTokens = 8;      // most tokens of a CTA
constexpr int kAppendAhead = 2;       // rows of a lane whose loads are in flight together
constexpr int kAppendMaxTokens = 1 << 30;

struct AppendParams {
  CacheView cache;
  SlotMap map;
  int layer, n_tokens, n_q, n_kv;
  int rotary, interleaved, tokens_per_cta, rows_per_cta;
  float gain;
  const int *positions;
  const long long *slots;
  const char *q, *k, *v;
  char *q_out;
  long long q_ts, q_hs, k_ts, k_hs, v_ts, v_hs, o_ts, o_hs;      // bytes
  double turns[kRopeMaxPairs];
};

// One row that a group of lanes has in hand.
template <typename T>
struct Row {
  Raw<T> raw;
  int kind, head, token;      // 0 K, 1 V, 2 Q, 3 none
  const char *src;            // the row
  long long slot;
};

// Turns a lane's pieces; cs: the token's (cos, sin) by pair.
template <typename T, int D>
__device__ __forceinline__ void turn_any(const AppendParams &p, Raw<T> &raw, const char *src, int sub, unsigned group, const float2 *cs) {
  const int half = p.rotary >> 1;
  float f[2][8], other[2][8];
  raw.unpack(0, f[0]);
  raw.unpack(1, f[1]);
  if (p.interleaved) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const int pair = (h * (D / 2) + sub * 8 + i) >> 1;
        if (pair < half) {
          const float2 w = cs[pair];
          const float a = f[h][i], b = f[h][i + 1];
          f[h][i] = turned_first(a, b, w);
          f[h][i + 1] = turned_second(a, b, w);
        }
      }
  } else {
    const T *row = reinterpret_cast<const T *>(src);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int e0 = h * (D / 2) + sub * 8;
      if (half % 8 == 0) {
        if (e0 < p.rotary) {
          Raw<T> partner;
          partner.load(src + (e0 < half ? e0 + half : e0 - half) * (int)sizeof(T), 0);
          partner.unpack(0, other[h]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int e = e0 + i;
          other[h][i] = e < p.rotary ? (float)row[e < half ? e + half : e - half] : 0.f;
        }
      }
    }
    __syncwarp(group);      // the row may be overwritten in place from here on
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int e = h * (D / 2) + sub * 8 + i;
        if (e < half)
          f[h][i] = turned_first(f[h][i], other[h][i], cs[e]);
        else if (e < p.rotary)
          f[h][i] = turned_second(other[h][i], f[h][i], cs[e - half]);
      }
  }
  raw.pack(0, f[0]);
  raw.pack(1, f[1]);
}

// Place of pair j of a whole head turned in halves, so that the 16-byte loads of a row's lanes (pairs 8 sub, ... + 7) follow one another.
template <int D>
__device__ __forceinline__ int place_of(int j) {
  return ((((j & 7) >> 1) * (D / 16) + (j >> 3)) << 1) + (j & 1);
}

template <typename T, int D, int FMT, bool WHOLE>      // WHOLE: the whole head turns in halves
__global__ void __launch_bounds__(kAppendThreads) cache_append_kernel(const __grid_constant__ AppendParams p) {
  constexpr int LPR = D / 16, ROWS = kAppendThreads / LPR, PIECE = 8 * (int)sizeof(T);
  __shared__ __align__(16) float2 cs[kAppendTokens][kRopeMaxPairs];
  const int t0 = blockIdx.x * p.tokens_per_cta, nt = min(p.tokens_per_cta, p.n_tokens - t0);
  const int rows = p.n_q + 2 * p.n_kv, r0 = blockIdx.y * p.rows_per_cta, nr = min(p.rows_per_cta, rows - r0);
  const int sub = threadIdx.x % LPR, items = nt * nr, half = p.rotary >> 1;
  const unsigned group = ((1u << LPR) - 1u) << (threadIdx.x & 31 & ~(LPR - 1));

  Row<T> r[kAppendAhead];
  auto load = [&](int first) {
#pragma unroll
    for (int i = 0; i < kAppendAhead; ++i) {
      const int it = first + i * ROWS;
      r[i].kind = 3;
      if (it >= items) continue;
      const int t = it / nr, row = r0 + it - t * nr;
      r[i].token = t;
      r[i].slot = -1;
      if (row < p.n_kv) {
        r[i].kind = 0;
        r[i].head = row;
        r[i].src = p.k + (t0 + t) * p.k_ts + row * p.k_hs;
      } else if (row < 2 * p.n_kv) {
        r[i].kind = 1;
        r[i].head = row - p.n_kv;
        r[i].src = p.v + (t0 + t) * p.v_ts + r[i].head * p.v_hs;
      } else {
        r[i].kind = 2;
        r[i].head = row - 2 * p.n_kv;
        r[i].src = p.q + (t0 + t) * p.q_ts + r[i].head * p.q_hs;
      }
      if (r[i].kind < 2) r[i].slot = __ldg(p.slots + t0 + t);
      r[i].raw.load(r[i].src + sub * PIECE, D / 2 * (int)sizeof(T));
    }
  };
  load(threadIdx.x / LPR);      // under the trigonometry
  for (int i = threadIdx.x; i < nt * half; i += kAppendThreads) {
    const int t = i / half, j = i - t * half;
    cs[t][WHOLE ? place_of<D>(j) : j] = rope_turn(p.positions[t0 + t], p.turns[j], p.gain, 1.f);
  }
  __syncthreads();
  for (int first = threadIdx.x / LPR; first < items; first += kAppendAhead * ROWS) {
    if (first >= ROWS) load(first);
#pragma unroll
    for (int i = 0; i < kAppendAhead; ++i) {
      Row<T> &x = r[i];
      if (x.kind == 3) continue;
      if (x.kind != 1) {
        if (WHOLE) {
          float a[8], b[8];
          x.raw.unpack(0, a);
          x.raw.unpack(1, b);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float4 w = *reinterpret_cast<const float4 *>(&cs[x.token][(k * LPR + sub) * 2]);
            const float2 w0 = make_float2(w.x, w.y), w1 = make_float2(w.z, w.w);
            const float a0 = a[2 * k], b0 = b[2 * k], a1 = a[2 * k + 1], b1 = b[2 * k + 1];
            a[2 * k] = turned_first(a0, b0, w0);
            b[2 * k] = turned_second(a0, b0, w0);
            a[2 * k + 1] = turned_first(a1, b1, w1);
            b[2 * k + 1] = turned_second(a1, b1, w1);
          }
          x.raw.pack(0, a);
          x.raw.pack(1, b);
        } else {
          turn_any<T, D>(p, x.raw, x.src, sub, group, cs[x.token]);
        }
      }
      if (x.kind == 2) {
        char *row = p.q_out + (t0 + x.token) * p.o_ts + x.head * p.o_hs + sub * PIECE;
        float f[8];
        x.raw.unpack(0, f);
        store8(row, f, T());
        x.raw.unpack(1, f);
        store8(row + D / 2 * (int)sizeof(T), f, T());
      } else {
        int block, offset;
        const bool live = p.map.split(x.slot, block, offset);
        const Pieces<D, FMT> to(p.cache, p.layer, x.kind, x.head, sub);
        put_row<T, D, FMT>(x.raw, to, block * p.cache.block_stride, offset, sub, group, live);
      }
    }
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
  if (p.rotary == D && !p.interleaved)
    cache_append_kernel<T, D, FMT, true><<<grid, kAppendThreads, 0, st>>>(p);
  else
    cache_append_kernel<T, D, FMT, false><<<grid, kAppendThreads, 0, st>>>(p);
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
  p.cache = make_view(cache);
  p.map = slot_map(cache);
  p.layer = layer;
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
