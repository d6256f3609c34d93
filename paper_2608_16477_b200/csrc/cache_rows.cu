// K and V rows into the pages of a cache, and back, through a list of slots: bf16 pages and e4m3 pages.
//
// e4m3 pages: one scale 2^e per (token, KV head) of K and of V, e the least integer with max |x| <= 448 * 2^e.  A power
// of two instead of max / 448: x * 2^-e and code * 2^e are exact, so a stored value is x rounded once to four significant
// bits (the e4m3 format itself has 2^-9 .. 448 to spread over, so the up to one binade that the power of two gives away
// costs only values below 2^-15 of the row's maximum), the two directions need no division, and reading back into bf16
// is exact.
//
// HBM-bound: every value is read once and written once.  head_dim / 8 lanes own a row (8 values each), the row maximum
// is a shuffle over them; consecutive lanes move consecutive 16-byte (bf16) or 8-byte (codes) pieces.  Once there are rows
// enough, a thread takes four of them and has their slots, then all their loads, in flight together.
#include <float.h>

#include "common.cuh"

namespace kvr {
namespace {

constexpr int kRowThreads = 256;
constexpr int kMinExp = -110, kMaxExp = 119;
// largest page pool for which slots fit 32 bits: the division by the block size is then a 32-bit one
constexpr long long kSlots32 = 0x7fffffffll;

struct RowsParams {
  CacheView cache;
  int layer, block_shift, token_shift;            // log2 of block_size and of 2 * n_kv_heads, -1 if no power of two
  long long n_slots;
  const long long *slots;
  char *k, *v;                                    // rows
  long long k_ts, k_hs, v_ts, v_hs;               // strides, bytes
  long long n_rows;                               // n_tokens * 2 * n_kv_heads
};

// Row r of the call: token, K or V, KV head; its strided side; and, from the token's slot, its page.
struct RowAt {
  char *row, *page;
  int token, kv, head, offset;   // offset: slot inside the page
  bool live;                     // the slot lies inside the pool
  __device__ __forceinline__ void find(const RowsParams &p, long long r) {
    const int per = 2 * p.cache.n_kv_heads;
    if (p.token_shift >= 0)
      token = (int)(r >> p.token_shift);
    else
      token = p.n_rows <= 0xffffffffll ? (int)((uint32_t)r / (uint32_t)per) : (int)(r / per);
    const int rem = (int)(r - (long long)token * per);
    kv = rem >= p.cache.n_kv_heads;
    head = rem - kv * p.cache.n_kv_heads;
    row = kv ? p.v + token * p.v_ts + head * p.v_hs : p.k + token * p.k_ts + head * p.k_hs;
  }
  __device__ __forceinline__ void place(const RowsParams &p, long long slot) {
    live = slot >= 0 && slot < p.n_slots;
    if (!live) slot = 0;
    long long block;
    if (p.block_shift >= 0)
      block = slot >> p.block_shift;
    else if (p.n_slots <= kSlots32)
      block = (uint32_t)slot / (uint32_t)p.cache.block_size;
    else
      block = slot / p.cache.block_size;
    offset = (int)(slot - block * p.cache.block_size);
    page = p.cache.page(p.layer, kv, (int)block);
  }
  __device__ __forceinline__ char *values(const RowsParams &p, int bytes) const {
    return page + ((long long)offset * p.cache.n_kv_heads + head) * bytes;
  }
  __device__ __forceinline__ char *scale(const RowsParams &p) const {
    return page + p.cache.value_bytes() + head * p.cache.block_size + offset;
  }
};

// 8 values of a row as floats; the raw registers are loaded first and unpacked later
template <typename T>
struct Raw8;
template <>
struct Raw8<bf16> {
  uint4 a;
  __device__ __forceinline__ void load(const char *p) { a = *reinterpret_cast<const uint4 *>(p); }
  __device__ __forceinline__ void unpack(float (&f)[8]) const {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
};
template <>
struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const char *p) {
    a = reinterpret_cast<const float4 *>(p)[0];
    b = reinterpret_cast<const float4 *>(p)[1];
  }
  __device__ __forceinline__ void unpack(float (&f)[8]) const {
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
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

template <typename T, int D, bool E4M3, int U>      // U: rows of a thread
__global__ void __launch_bounds__(kRowThreads) cache_write_kernel(const __grid_constant__ RowsParams p) {
  constexpr int LPR = D / 8;                 // lanes of a row
  constexpr int RPC = kRowThreads / LPR;     // rows of a CTA at a time
  const int sub = threadIdx.x % LPR;
  const long long r0 = (long long)blockIdx.x * RPC * U + threadIdx.x / LPR;
  RowAt at[U];
  Raw8<T> raw[U];
  long long slot[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const long long r = r0 + i * RPC;
    at[i].find(p, r < p.n_rows ? r : p.n_rows - 1);           // every lane stays for the shuffles
    slot[i] = r < p.n_rows ? __ldg(p.slots + at[i].token) : -1;
    raw[i].load(at[i].row + sub * 8 * (int)sizeof(T));
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    float f[8];
    raw[i].unpack(f);
    at[i].place(p, slot[i]);
    if (E4M3) {
      float most = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float a = fabsf(f[j]);
        most = fmaxf(most, a <= FLT_MAX ? a : 0.f);           // infinities and NaN do not set the scale
      }
#pragma unroll
      for (int o = LPR / 2; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
      // most = m * 2^x with 1 <= m < 2; 448 = 1.75 * 2^8, so e = x - 8, one more if m > 1.75
      const uint32_t bits = __float_as_uint(most);
      int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u);
      e = min(max(e, kMinExp), kMaxExp);
      const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = fabsf(f[j]) <= FLT_MAX ? f[j] * inv : __uint_as_float(0x7fc00000u);
      if (at[i].live) {
        uint2 c;
        c.x = e4m3x2(f[0], f[1]) | (e4m3x2(f[2], f[3]) << 16);
        c.y = e4m3x2(f[4], f[5]) | (e4m3x2(f[6], f[7]) << 16);
        *reinterpret_cast<uint2 *>(at[i].values(p, D) + sub * 8) = c;
        if (sub == 0) *at[i].scale(p) = (char)(e + 127);
      }
    } else if (at[i].live) {
      *reinterpret_cast<uint4 *>(at[i].values(p, 2 * D) + sub * 16) = pack_bf16(f);
    }
  }
}

template <typename T, int D, bool E4M3, int U>
__global__ void __launch_bounds__(kRowThreads) cache_read_kernel(const __grid_constant__ RowsParams p) {
  constexpr int LPR = D / 8, RPC = kRowThreads / LPR;
  const int sub = threadIdx.x % LPR;
  const long long r0 = (long long)blockIdx.x * RPC * U + threadIdx.x / LPR;
  RowAt at[U];
  uint4 raw[U];
  uint32_t scale[U];
  long long slot[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const long long r = r0 + i * RPC;
    at[i].find(p, r < p.n_rows ? r : p.n_rows - 1);
    slot[i] = r < p.n_rows ? __ldg(p.slots + at[i].token) : -1;
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    at[i].place(p, slot[i]);
    if (E4M3) {
      const uint2 c = *reinterpret_cast<const uint2 *>(at[i].values(p, D) + sub * 8);      // slot 0 if it is not live
      raw[i] = make_uint4(c.x, c.y, 0, 0);
      scale[i] = *reinterpret_cast<const uint8_t *>(at[i].scale(p));
    } else {
      raw[i] = *reinterpret_cast<const uint4 *>(at[i].values(p, 2 * D) + sub * 16);
    }
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    if (!at[i].live) continue;
    float f[8];
    if (E4M3) {
      const float s = __uint_as_float(scale[i] << 23);
      const uint32_t w[2] = {raw[i].x, raw[i].y};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 c = from_e4m3x2((uint16_t)(w[j >> 1] >> ((j & 1) * 16)));
        f[2 * j] = c.x * s;
        f[2 * j + 1] = c.y * s;
      }
    } else {
      Raw8<bf16> b;
      b.a = raw[i];
      b.unpack(f);
    }
    store8(at[i].row + sub * 8 * (int)sizeof(T), f, T());
  }
}

template <typename T, int D, bool E4M3, int U>
int launch_rows_u(const RowsParams &p, bool write, cudaStream_t st) {
  constexpr long long rows = (long long)kRowThreads / (D / 8) * U;
  const long long grid = (p.n_rows + rows - 1) / rows;
  if (grid > 0x7fffffffll) return KV_ERR_SHAPE;
  if (write)
    cache_write_kernel<T, D, E4M3, U><<<(unsigned)grid, kRowThreads, 0, st>>>(p);
  else
    cache_read_kernel<T, D, E4M3, U><<<(unsigned)grid, kRowThreads, 0, st>>>(p);
  KV_COUNT_LAUNCH();
  KV_CUDA(cudaGetLastError());
  return KV_OK;
}

// Four rows to a thread once that still gives every SM four CTAs, one below that (few rows: the chain slot -> row -> store
// is all there is, and more CTAs share it).
template <typename T, int D, bool E4M3>
int launch_rows(const RowsParams &p, bool write, cudaStream_t st) {
  const int device = current_device();
  if (device < 0) return KV_ERR_CUDA;
  const long long rows = kRowThreads / (D / 8);
  return p.n_rows >= 16 * rows * sm_count(device) ? launch_rows_u<T, D, E4M3, 4>(p, write, st)
                                                  : launch_rows_u<T, D, E4M3, 1>(p, write, st);
}

// strides are in elements of dtype
int rows_call(const kv_cache_desc *cache, int layer, const void *k, int64_t k_ts, int64_t k_hs, const void *v,
              int64_t v_ts, int64_t v_hs, int dtype, int n_tokens, const int64_t *slots, bool write, void *stream) {
  if (n_tokens < 0 || (dtype != KV_DTYPE_BF16 && dtype != KV_DTYPE_F32)) return KV_ERR_ARG;
  int rc = check_cache_desc(cache, true);
  if (rc != KV_OK) return rc;
  if (cache->head_dim != 64 && cache->head_dim != 128) return KV_ERR_SHAPE;
  if (layer < 0 || layer >= cache->n_layers) return KV_ERR_SHAPE;
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
  p.block_shift = p.token_shift = -1;
  for (int b = 0; b < 31; ++b) {
    if ((1 << b) == cache->block_size) p.block_shift = b;
    if ((1ll << b) == 2ll * cache->n_kv_heads) p.token_shift = b;
  }
  p.slots = reinterpret_cast<const long long *>(slots);
  p.k = (char *)const_cast<void *>(k);
  p.v = (char *)const_cast<void *>(v);
  p.k_ts = k_ts * size;
  p.k_hs = k_hs * size;
  p.v_ts = v_ts * size;
  p.v_hs = v_hs * size;
  p.n_rows = (long long)n_tokens * 2 * cache->n_kv_heads;
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
