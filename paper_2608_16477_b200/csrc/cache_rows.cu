// K and V rows into the pages of a cache, and back, through a list of slots: bf16 pages and e4m3 pages.
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
#include <float.h>

#include "common.cuh"

namespace kvr {
namespace {

constexpr int kRowThreads = 256;
constexpr int kMaxTokens = 1 << 30;   // tokens are counted in 32 bits, a CTA's ahead
constexpr int kMinExp = -110, kMaxExp = 119;
// largest page pool for which slots fit 32 bits: the division by the block size is then a 32-bit one
constexpr long long kSlots32 = 0x7fffffffll;

struct RowsParams {
  CacheView cache;
  int layer, block_shift;                         // block_shift: log2(block_size), -1 if it is no power of two
  int n_tokens, heads;                            // heads of K, and of V, that a CTA takes
  long long n_slots;
  const long long *slots;
  char *k, *v;                                    // rows
  long long k_ts, k_hs, v_ts, v_hs;               // strides, bytes
};

// A thread's place: the piece `sub` of head `head` of K or V, for tokens first, first + step, ...
template <int D>
struct Place {
  static constexpr int LPR = D / 16;              // lanes of a row
  int sub, first, step;
  bool idle;
  unsigned group;                                 // the row's lanes
  char *row, *values, *scale;                     // of token 0; of slot 0 of block 0
  long long row_step, slot_bytes;
  __device__ __forceinline__ Place(const RowsParams &p, int elem, int u, int bytes) {      // bytes: of a piece of the row
    const int per = 2 * p.heads * LPR, tokens = kRowThreads / per;      // threads of a token, tokens of a CTA at a time
    const int at = (int)threadIdx.x / per, in = (int)threadIdx.x - at * per;
    const int line = in / LPR, kv = line >= p.heads, head = blockIdx.y * p.heads + line - kv * p.heads;
    sub = in % LPR;
    idle = at >= tokens || head >= p.cache.n_kv_heads;
    step = tokens;
    first = blockIdx.x * tokens * u + at;
    group = (LPR == 32 ? 0xffffffffu : ((1u << LPR) - 1u)) << (threadIdx.x & 31 & ~(LPR - 1));
    row = (kv ? p.v + head * p.v_hs : p.k + head * p.k_hs) + sub * bytes;
    row_step = kv ? p.v_ts : p.k_ts;
    slot_bytes = (long long)p.cache.n_kv_heads * D * elem;
    char *page = p.cache.page(p.layer, kv, 0);
    values = page + head * D * elem + sub * 8 * elem;
    scale = page + p.cache.value_bytes() + head * p.cache.block_size;
  }
};
// Block and offset of a slot; false if it lies outside the pool.
__device__ __forceinline__ bool split_slot(const RowsParams &p, long long slot, int &block, int &offset) {
  block = offset = 0;
  if ((unsigned long long)slot >= (unsigned long long)p.n_slots) return false;
  if (p.block_shift >= 0)
    block = (int)(slot >> p.block_shift);
  else if (p.n_slots <= kSlots32)
    block = (int)((uint32_t)slot / (uint32_t)p.cache.block_size);
  else
    block = (int)(slot / p.cache.block_size);
  offset = (int)(slot - (long long)block * p.cache.block_size);
  return true;
}

// Two pieces of 8 values of a row: the raw registers are loaded first and unpacked later.
template <typename T>
struct Raw;
template <>
struct Raw<bf16> {
  uint4 a[2];
  __device__ __forceinline__ void load(const char *p, int apart) {
    a[0] = *reinterpret_cast<const uint4 *>(p);
    a[1] = *reinterpret_cast<const uint4 *>(p + apart);
  }
  __device__ __forceinline__ void unpack(int h, float (&f)[8]) const {
    const uint32_t w[4] = {a[h].x, a[h].y, a[h].z, a[h].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint32_t max2(uint32_t x, uint32_t y) {
    uint32_t r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(y));
    return r;
  }
  // The largest |x| over the row's lanes, as an fp32 pattern: above 0x7f7fffff if one is no finite number.
  template <int LANES>
  __device__ __forceinline__ uint32_t top(unsigned group) const {
    const uint32_t s = 0x7fff7fffu;
    uint32_t m = max2(max2(max2(a[0].x & s, a[0].y & s), max2(a[0].z & s, a[0].w & s)),
                      max2(max2(a[1].x & s, a[1].y & s), max2(a[1].z & s, a[1].w & s)));
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) m = max2(m, __shfl_xor_sync(group, m, o));
    return max(m & 0xffff0000u, m << 16);
  }
};
template <>
struct Raw<float> {
  float4 a[2][2];
  __device__ __forceinline__ void load(const char *p, int apart) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      a[h][0] = reinterpret_cast<const float4 *>(p + h * apart)[0];
      a[h][1] = reinterpret_cast<const float4 *>(p + h * apart)[1];
    }
  }
  __device__ __forceinline__ void unpack(int h, float (&f)[8]) const {
    f[0] = a[h][0].x; f[1] = a[h][0].y; f[2] = a[h][0].z; f[3] = a[h][0].w;
    f[4] = a[h][1].x; f[5] = a[h][1].y; f[6] = a[h][1].z; f[7] = a[h][1].w;
  }
  static __device__ __forceinline__ float larger(float x, float y) {      // of the magnitudes, NaN if one is NaN
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(fabsf(x)), "f"(fabsf(y)));
    return r;
  }
  template <int LANES>
  __device__ __forceinline__ uint32_t top(unsigned group) const {
    float m = 0.f;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 2; ++i) m = larger(m, larger(larger(a[h][i].x, a[h][i].y), larger(a[h][i].z, a[h][i].w)));
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) m = larger(m, __shfl_xor_sync(group, m, o));
    return __float_as_uint(m) & 0x7fffffffu;
  }
};

__device__ __forceinline__ uint4 pack_bf16(const float (&f)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t *>(&h);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(char *p, const float (&f)[8], bf16) { *reinterpret_cast<uint4 *>(p) = pack_bf16(f); }
__device__ __forceinline__ void store8(char *p, const float (&f)[8], float) {
  reinterpret_cast<float4 *>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
  reinterpret_cast<float4 *>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}

__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float2 from_e4m3x2(uint16_t c) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(c));
  float2 f;
  asm("{\n\t.reg .b16 l, u;\n\tmov.b32 {l, u}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, u;\n\t}"
      : "=f"(f.x), "=f"(f.y) : "r"(h));
  return f;
}

template <typename T, int D, bool E4M3, int U>      // U: tokens of a thread at a time
__global__ void __launch_bounds__(kRowThreads) cache_write_kernel(const __grid_constant__ RowsParams p) {
  const Place<D> me(p, E4M3 ? 1 : 2, U, 8 * (int)sizeof(T));
  if (me.idle) return;                                        // whole rows at a time: the shuffles are the row's own
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
      const bool live = split_slot(p, slot[i], block, offset);
      char *values = me.values + block * p.cache.block_stride + offset * me.slot_bytes;
      float f[2][8];
      raw[i].unpack(0, f[0]);
      raw[i].unpack(1, f[1]);
      if (!E4M3) {
        if (live) {
          *reinterpret_cast<uint4 *>(values) = pack_bf16(f[0]);
          *reinterpret_cast<uint4 *>(values + D) = pack_bf16(f[1]);
        }
        continue;
      }
      uint32_t bits = raw[i].template top<Place<D>::LPR>(me.group);
      if (bits > 0x7f7fffffu) {                                 // infinities and NaN do not set the scale and become NaN
        float most = 0.f;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            if (!(fabsf(f[h][j]) <= FLT_MAX)) f[h][j] = __uint_as_float(0x7fc00000u);
            most = fmaxf(most, fabsf(f[h][j]));                 // ignores NaN
          }
#pragma unroll
        for (int o = Place<D>::LPR / 2; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(me.group, most, o));
        bits = __float_as_uint(most);
      }
      // |x| <= m * 2^x with 1 <= m < 2; 448 = 1.75 * 2^8, so e = x - 8, one more if m > 1.75
      int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u);
      e = min(max(e, kMinExp), kMaxExp);
      const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
      uint2 c[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        c[h].x = e4m3x2(f[h][0] * inv, f[h][1] * inv) | (e4m3x2(f[h][2] * inv, f[h][3] * inv) << 16);
        c[h].y = e4m3x2(f[h][4] * inv, f[h][5] * inv) | (e4m3x2(f[h][6] * inv, f[h][7] * inv) << 16);
      }
      if (live) {
        *reinterpret_cast<uint2 *>(values) = c[0];
        *reinterpret_cast<uint2 *>(values + D / 2) = c[1];
        if (me.sub == 0) me.scale[block * p.cache.block_stride + offset] = (char)(e + 127);
      }
    }
  }
}

template <typename T, int D, bool E4M3, int U>
__global__ void __launch_bounds__(kRowThreads) cache_read_kernel(const __grid_constant__ RowsParams p) {
  const Place<D> me(p, E4M3 ? 1 : 2, U, 8 * (int)sizeof(T));
  if (me.idle) return;
  uint4 raw[U][E4M3 ? 1 : 2];                                 // e4m3: both pieces in one
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
    live[i] = split_slot(p, slot[i], block, offset);          // block 0, offset 0 if not: read, but not written anywhere
    const char *values = me.values + block * p.cache.block_stride + offset * me.slot_bytes;
    if (E4M3) {
      const uint2 a = *reinterpret_cast<const uint2 *>(values), b = *reinterpret_cast<const uint2 *>(values + D / 2);
      raw[i][0] = make_uint4(a.x, a.y, b.x, b.y);
      scale[i] = *reinterpret_cast<const uint8_t *>(me.scale + block * p.cache.block_stride + offset);
    } else {
      raw[i][0] = *reinterpret_cast<const uint4 *>(values);
      raw[i][E4M3 ? 0 : 1] = *reinterpret_cast<const uint4 *>(values + D);
    }
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    if (!live[i]) continue;
    char *row = me.row + (me.first + i * me.step) * me.row_step;
    float f[2][8];
    if (E4M3) {
      const float s = __uint_as_float(scale[i] << 23);
      const uint32_t w[4] = {raw[i][0].x, raw[i][0].y, raw[i][0].z, raw[i][0].w};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float2 c = from_e4m3x2((uint16_t)(w[j >> 1] >> ((j & 1) * 16)));
        f[j >> 2][(2 * j) & 7] = c.x * s;
        f[j >> 2][(2 * j + 1) & 7] = c.y * s;
      }
    } else {
      Raw<bf16> b;
      b.a[0] = raw[i][0];
      b.a[1] = raw[i][E4M3 ? 0 : 1];
      b.unpack(0, f[0]);
      b.unpack(1, f[1]);
    }
    store8(row, f[0], T());
    store8(row + D / 2 * (int)sizeof(T), f[1], T());
  }
}

template <typename T, int D, bool E4M3, int U>
int launch_rows_u(const RowsParams &p, bool write, int sms, cudaStream_t st) {
  const int tokens = kRowThreads / (2 * p.heads * Place<D>::LPR) * U;
  dim3 grid((p.n_tokens + tokens - 1) / tokens, (p.cache.n_kv_heads + p.heads - 1) / p.heads);
  if (grid.y > 65535) return KV_ERR_SHAPE;
  // Writing stays in place with four CTAs per SM (16,384 tokens of 8 heads of 128: 18.4 us against 20.7 us with a CTA for
  // every two tokens); reading, whose loads wait for the slots, is better off with new CTAs (18.8 us against 19.2 us).
  const unsigned stay = (unsigned)(4 * sms / (int)grid.y > 1 ? 4 * sms / (int)grid.y : 1);
  if (write && grid.x > stay) grid.x = stay;
  if (write)
    cache_write_kernel<T, D, E4M3, U><<<grid, kRowThreads, 0, st>>>(p);
  else
    cache_read_kernel<T, D, E4M3, U><<<grid, kRowThreads, 0, st>>>(p);
  KV_COUNT_LAUNCH();
  KV_CUDA(cudaGetLastError());
  return KV_OK;
}

// Two tokens to a thread once that still gives every SM eight CTAs (16,384 tokens: write 20.7 us against 23.1 us with one,
// read 18.8 us against 23.3 us; four are no better), one below that (few rows: the chain slot -> row ->
// store is all there is, and more CTAs share it).
template <typename T, int D, bool E4M3>
int launch_rows(RowsParams &p, bool write, cudaStream_t st) {
  const int device = current_device();
  if (device < 0) return KV_ERR_CUDA;
  const int most = kRowThreads / (2 * Place<D>::LPR);          // heads that fit a CTA with their K and V
  p.heads = p.cache.n_kv_heads < most ? p.cache.n_kv_heads : most;
  const long long threads = (long long)p.n_tokens * 2 * p.cache.n_kv_heads * Place<D>::LPR;
  const int sms = sm_count(device);
  return threads >= 16ll * kRowThreads * sms ? launch_rows_u<T, D, E4M3, 2>(p, write, sms, st)
                                             : launch_rows_u<T, D, E4M3, 1>(p, write, sms, st);
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
  p.cache = make_view(cache);
  p.layer = layer;
  p.n_slots = (long long)cache->num_blocks * cache->block_size;
  p.block_shift = -1;
  for (int b = 0; b < 31; ++b)
    if ((1 << b) == cache->block_size) p.block_shift = b;
  p.n_tokens = n_tokens;
  p.slots = reinterpret_cast<const long long *>(slots);
  p.k = (char *)const_cast<void *>(k);
  p.v = (char *)const_cast<void *>(v);
  p.k_ts = k_ts * size;
  p.k_hs = k_hs * size;
  p.v_ts = v_ts * size;
  p.v_hs = v_hs * size;
  cudaStream_t st = (cudaStream_t)stream;
  const bool e4m3 = cache->elem_bytes == 1, f32 = dtype == KV_DTYPE_F32;
  if (d == 128) {
    if (e4m3) return f32 ? launch_rows<float, 128, true>(p, write, st) : launch_rows<bf16, 128, true>(p, write, st);
    return f32 ? launch_rows<float, 128, false>(p, write, st) : launch_rows<bf16, 128, false>(p, write, st);
  }
  if (e4m3) return f32 ? launch_rows<float, 64, true>(p, write, st) : launch_rows<bf16, 64, true>(p, write, st);
  return f32 ? launch_rows<float, 64, false>(p, write, st) : launch_rows<bf16, 64, false>(p, write, st);
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
