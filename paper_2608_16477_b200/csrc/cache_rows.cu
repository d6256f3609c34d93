// K and V rows into the pages of a cache, and back, through a list of slots: bf16, e4m3 and e2m1 pages.
//
// e4m3 pages: one scale 2^e per (token, KV head) of K and of V, e the least integer with max |x| <= 448 * 2^e.  A power
// of two instead of max / 448: x * 2^-e and code * 2^e are exact, so a stored value is x rounded once to four significant
// bits, the two directions need no division, and reading back into bf16 is exact.  The price is up to one binade of the
// range: codes keep their four bits down to 2^-6, which is 2^-13.8 of the row's maximum at the worst and 2^-14.8 at best.
//
// HBM-bound: every value is read once and written once; instructions are what has to be saved beside that.  head_dim / 16
// lanes own a row, the row maximum is a shuffle over them; a lane has two pieces of 8 values, half a row apart, so that
// consecutive lanes move consecutive 16-byte (bf16) or 8-byte (codes) pieces.  A thread keeps its place in the token (K or
// V, head, piece) for all its tokens, so that only the slot's page has to be worked out for each; once there are tokens
// enough it takes two at a time, with their slots, then all their loads, in flight together.  The maximum runs over the raw
// bits (an infinity or NaN shows in it, and only then the row is gone through value by value).  Measured in a graph / call after
// call, 16,384 tokens of 8 heads of 128: bf16 to e4m3 and back, 101 MB each way, 18.4 / 20.5 and 18.8 / 20.5 us (5.4 / 4.9 TB/s,
// 82 / 75 % of a copy's rate with the launch in it); bf16 to bf16 pages and back, 134 MB, 24.3 / 26.6 and 23.0 / 24.9 us (5.5 and 5.8
// TB/s), fp32, 201 MB, 33.9 / 36.1 and 38.3 / 40.7 us.  64 tokens 1.9 to 2.5 us.  A piece of 8 to a lane and index arithmetic for
// every row: 161 instructions a warp and row, 27 us.
// e2m1 pages (16,384 tokens of 8 heads of 128; floor): from bf16 20.4 us (13.1), into bf16 19.2 (13.1), from fp32 37.1 (23.4; 49 with
// three comparisons for every value), into fp32 39.0 (23.4).  Writing from bf16 and reading into bf16 are busy with conversions (issue slots 68 and 75 %,
// ALU pipe 62 and 58 %); fp32 rows wait for their loads (issue slots 53 %), or for the path to memory (30 %).
#include "cache_format.cuh"

namespace kvr {
namespace {

constexpr int kRowThreads = 256;
constexpr int kMaxTokens = 1 << 30;   // tokens are counted in 32 bits, a CTA's ahead

struct RowsParams {
  RowLayout layout;
  SlotMap map;
  int n_kv_heads;
  int n_tokens, heads;                            // heads of K, and of V, that a CTA takes
  const long long *slots;
  char *k, *v;                                    // rows
  long long k_ts, k_hs, v_ts, v_hs;               // strides, bytes
};

// A thread's place: the piece `sub` of head `head` of K or V, for tokens first, first + step, ...
template <int D>
struct Place {
  static constexpr int LPR = D / 16;              // lanes of a row
  int sub, first, step, kv, head;
  bool idle;
  unsigned group;                                 // the row's lanes
  char *row;                                      // of token 0
  long long row_step;
  __device__ __forceinline__ Place(const RowsParams &p, int u, int bytes) {      // bytes: of a piece of the row
    const int per = 2 * p.heads * LPR, tokens = kRowThreads / per;      // threads of a token, tokens of a CTA at a time
    const int at = (int)threadIdx.x / per, in = (int)threadIdx.x - at * per;
    const int line = in / LPR;
    kv = line >= p.heads;
    head = blockIdx.y * p.heads + line - kv * p.heads;
    sub = in % LPR;
    idle = at >= tokens || head >= p.n_kv_heads;
    step = tokens;
    first = blockIdx.x * tokens * u + at;
    group = (LPR == 32 ? 0xffffffffu : ((1u << LPR) - 1u)) << (threadIdx.x & 31 & ~(LPR - 1));
    row = (kv ? p.v + head * p.v_hs : p.k + head * p.k_hs) + sub * bytes;
    row_step = kv ? p.v_ts : p.k_ts;
  }
};

template <typename T, int D, int FMT, int U>      // U: tokens of a thread at a time
__global__ void __launch_bounds__(kRowThreads) cache_write_kernel(const __grid_constant__ RowsParams p) {
  const Place<D> me(p, U, 8 * (int)sizeof(T));
  if (me.idle) return;                                        // whole rows at a time: the shuffles are the row's own
  const Pieces<D, FMT> to(p.layout, me.kv, me.head, me.sub * 8);
  for (int t0 = me.first; t0 < p.n_tokens; t0 += gridDim.x * me.step * U) {
    Raw<T> raw[U];
    long long slot[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int t = t0 + i * me.step;
      const bool is = t < p.n_tokens;
      slot[i] = is ? __ldg(p.slots + t) : -1;
      raw[i].load(me.row + (is ? t : 0) * me.row_step, D / 2 * (int)sizeof(T));
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      int block, offset;
      const bool live = p.map.split(slot[i], block, offset);
      put_row<T, D, FMT>(raw[i], to, p.layout.slot_stride, D / 2, block * p.layout.block_stride, offset, me.sub, me.group, live);
    }
  }
}

template <typename T, int D, int FMT, int U>
__global__ void __launch_bounds__(kRowThreads) cache_read_kernel(const __grid_constant__ RowsParams p) {
  const Place<D> me(p, U, 8 * (int)sizeof(T));
  if (me.idle) return;
  const Pieces<D, FMT> from(p.layout, me.kv, me.head, me.sub * 8);
  constexpr int APART = FMT == kE2m1 ? D / 4 : D / 2 * FMT;
  uint4 raw[U][FMT == kBf16 ? 2 : 1];                         // e4m3, e2m1: both pieces in one
  uint32_t scale[U];
  long long slot[U];
  bool live[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int t = me.first + i * me.step;
    slot[i] = t < p.n_tokens ? __ldg(p.slots + t) : -1;
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    int block, offset;
    live[i] = p.map.split(slot[i], block, offset);            // block 0, offset 0 if not: read, but not written anywhere
    const long long at = block * p.layout.block_stride;
    const char *values = from.values + at + offset * p.layout.slot_stride;
    if (FMT == kE4m3) {
      const uint2 a = *reinterpret_cast<const uint2 *>(values), b = *reinterpret_cast<const uint2 *>(values + APART);
      raw[i][0] = make_uint4(a.x, a.y, b.x, b.y);
      scale[i] = *reinterpret_cast<const uint8_t *>(from.scale + at + offset);
    } else if (FMT == kE2m1) {
      const uint8_t *g = reinterpret_cast<const uint8_t *>(from.groups + at + (long long)offset * (D / 16));
      raw[i][0] = make_uint4(*reinterpret_cast<const uint32_t *>(values), *reinterpret_cast<const uint32_t *>(values + APART), g[0], g[D / 32]);
      scale[i] = *reinterpret_cast<const uint8_t *>(from.scale + at + offset);
    } else {
      raw[i][0] = *reinterpret_cast<const uint4 *>(values);
      raw[i][FMT == kBf16] = *reinterpret_cast<const uint4 *>(values + APART);
    }
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    if (!live[i]) continue;
    char *row = me.row + (me.first + i * me.step) * me.row_step;
    float f[2][8];
    if (FMT == kE4m3) {
      const float s = __uint_as_float(scale[i] << 23);
      const uint32_t w[4] = {raw[i][0].x, raw[i][0].y, raw[i][0].z, raw[i][0].w};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float2 c = floats_of_half2(half2_of_e4m3x2(w[j >> 1] >> ((j & 1) * 16)));
        f[j >> 2][(2 * j) & 7] = c.x * s;
        f[j >> 2][(2 * j + 1) & 7] = c.y * s;
      }
    } else if (FMT == kE2m1) {
      const float s = __uint_as_float(scale[i] << 23);
      const uint32_t w[2] = {raw[i][0].x, raw[i][0].y}, g[2] = {raw[i][0].z, raw[i][0].w};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t both = half2_of_e4m3x2(g[h] * 0x101u);
        uint32_t v[4];
        halves_of_e2m1(w[h], v);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 c = floats_of_half2(mul_half2(v[j], both));
          f[h][2 * j] = c.x * s;
          f[h][2 * j + 1] = c.y * s;
        }
      }
    } else {
      Raw<bf16> b;
      b.a[0] = raw[i][0];
      b.a[1] = raw[i][FMT == kBf16];
      b.unpack(0, f[0]);
      b.unpack(1, f[1]);
    }
    store8(row, f[0], T());
    store8(row + D / 2 * (int)sizeof(T), f[1], T());
  }
}

template <typename T, int D, int FMT, int U>
int launch_rows_u(const RowsParams &p, bool write, int sms, cudaStream_t st) {
  const int tokens = kRowThreads / (2 * p.heads * Place<D>::LPR) * U;
  dim3 grid((p.n_tokens + tokens - 1) / tokens, (p.n_kv_heads + p.heads - 1) / p.heads);
  if (grid.y > 65535) return KV_ERR_SHAPE;
  // Writing stays in place with four CTAs per SM (16,384 tokens of 8 heads of 128: 18.4 us against 20.7 us with a CTA for
  // every two tokens); reading, whose loads wait for the slots, is better off with new CTAs (18.8 us against 19.2 us).
  const unsigned stay = (unsigned)(4 * sms / (int)grid.y > 1 ? 4 * sms / (int)grid.y : 1);
  if (write && grid.x > stay) grid.x = stay;
  if (write)
    cache_write_kernel<T, D, FMT, U><<<grid, kRowThreads, 0, st>>>(p);
  else
    cache_read_kernel<T, D, FMT, U><<<grid, kRowThreads, 0, st>>>(p);
  KV_COUNT_LAUNCH();
  KV_CUDA(cudaGetLastError());
  return KV_OK;
}

// Two tokens to a thread once that still gives every SM eight CTAs (16,384 tokens: write 20.7 us against 23.1 us with one,
// read 18.8 us against 23.3 us; four are no better), one below that (few rows: the chain slot -> row ->
// store is all there is, and more CTAs share it).
template <typename T, int D, int FMT>
int launch_rows(RowsParams &p, bool write, cudaStream_t st) {
  const int device = current_device();
  if (device < 0) return KV_ERR_CUDA;
  const int most = kRowThreads / (2 * Place<D>::LPR);          // heads that fit a CTA with their K and V
  p.heads = p.n_kv_heads < most ? p.n_kv_heads : most;
  const long long threads = (long long)p.n_tokens * 2 * p.n_kv_heads * Place<D>::LPR;
  const int sms = sm_count(device);
  return threads >= 16ll * kRowThreads * sms ? launch_rows_u<T, D, FMT, 2>(p, write, sms, st)
                                             : launch_rows_u<T, D, FMT, 1>(p, write, sms, st);
}

template <int FMT>
int rows_format(RowsParams &p, int d, bool f32, bool write, cudaStream_t st) {
  if (d == 128) return f32 ? launch_rows<float, 128, FMT>(p, write, st) : launch_rows<bf16, 128, FMT>(p, write, st);
  return f32 ? launch_rows<float, 64, FMT>(p, write, st) : launch_rows<bf16, 64, FMT>(p, write, st);
}

// strides are in elements of dtype
int rows_call(const kv_cache_desc *cache, int layer, const void *k, int64_t k_ts, int64_t k_hs, const void *v,
              int64_t v_ts, int64_t v_hs, int dtype, int n_tokens, const int64_t *slots, bool write, void *stream) {
  if (n_tokens < 0 || (dtype != KV_DTYPE_BF16 && dtype != KV_DTYPE_F32)) return KV_ERR_ARG;
  int rc = check_cache_desc(cache, true);
  if (rc != KV_OK) return rc;
  if (cache->head_dim != 64 && cache->head_dim != 128) return KV_ERR_SHAPE;
  if (layer < 0 || layer >= cache->n_layers || n_tokens > kMaxTokens) return KV_ERR_SHAPE;
  if (n_tokens == 0) return KV_OK;
  if (k == nullptr || v == nullptr || slots == nullptr) return KV_ERR_ARG;
  const int size = dtype == KV_DTYPE_BF16 ? 2 : 4, d = cache->head_dim;
  const int64_t strides[4] = {k_ts, k_hs, v_ts, v_hs};
  for (int64_t s : strides)
    if (s < 0 || s * size % 16 != 0) return KV_ERR_ARG;
  if (((uintptr_t)k & 15) || ((uintptr_t)v & 15) || ((uintptr_t)slots & 7)) return KV_ERR_ARG;
  if (!write) {   // rows that are written must not overlap one another
    if (!rows_disjoint(k_ts, k_hs, n_tokens, cache->n_kv_heads, d) ||
        !rows_disjoint(v_ts, v_hs, n_tokens, cache->n_kv_heads, d))
      return KV_ERR_ARG;
  }
  RowsParams p;
  p.layout = row_layout(make_view(cache), layer);
  p.map = slot_map(cache);
  p.n_kv_heads = cache->n_kv_heads;
  p.n_tokens = n_tokens;
  p.slots = reinterpret_cast<const long long *>(slots);
  p.k = (char *)const_cast<void *>(k);
  p.v = (char *)const_cast<void *>(v);
  p.k_ts = k_ts * size;
  p.k_hs = k_hs * size;
  p.v_ts = v_ts * size;
  p.v_hs = v_hs * size;
  const bool f32 = dtype == KV_DTYPE_F32;
  cudaStream_t st = (cudaStream_t)stream;
  switch (format_of(cache->elem_bytes)) {
    case kBf16: return rows_format<kBf16>(p, d, f32, write, st);
    case kE4m3: return rows_format<kE4m3>(p, d, f32, write, st);
    default: return rows_format<kE2m1>(p, d, f32, write, st);
  }
}

}  // namespace
}  // namespace kvr

extern "C" {

int32_t kv_op_cache_write(const kv_cache_desc *cache, int32_t layer, const void *k_dev, int64_t k_token_stride,
                          int64_t k_head_stride, const void *v_dev, int64_t v_token_stride, int64_t v_head_stride,
                          int32_t dtype, int32_t n_tokens, const int64_t *slots_dev, void *stream) {
  return kvr::rows_call(cache, layer, k_dev, k_token_stride, k_head_stride, v_dev, v_token_stride, v_head_stride, dtype,
                        n_tokens, slots_dev, true, stream);
}

int32_t kv_op_cache_read(const kv_cache_desc *cache, int32_t layer, const int64_t *slots_dev, int32_t n_tokens,
                         void *k_out_dev, int64_t k_token_stride, int64_t k_head_stride, void *v_out_dev,
                         int64_t v_token_stride, int64_t v_head_stride, int32_t dtype, void *stream) {
  return kvr::rows_call(cache, layer, k_out_dev, k_token_stride, k_head_stride, v_out_dev, v_token_stride,
                        v_head_stride, dtype, n_tokens, slots_dev, false, stream);
}

}  // extern "C"
