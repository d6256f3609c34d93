// Rows of a paged cache in its three formats, as the kernels that write and read them share it (internal).  head_dim / 16 lanes
// own a row; a lane has two pieces of 8 values, half a row apart.
//
// e2m1 pages: a row's scale 2^e is the least power of two with max |x| <= 6 * 448 * 2^e, a group of 16 dims takes the least e4m3
// number s with max |x| <= 6 * s * 2^e, and a value the code nearest to |x| / (s * 2^e), halves up.  All three are comparisons
// with products that fp32 holds exactly (6 s: six bits, a border between two codes times s: seven), so they depend on no
// division's rounding; code * s * 2^e has six bits and is exact in bf16 and fp32, code * s in fp16.  s is e4m3 and no power of two:
// that would leave up to a binade of a group's 4 bits unused (3 dB on normal rows).
#pragma once
#include <float.h>

#include "common.cuh"

namespace kvr {
namespace {

constexpr int kMinExp = -110, kMaxExp = 119;
constexpr int kMaxExpE2m1 = 116;      // 6 * 448 * 2^e stays in fp32's range
// page formats as the kernels' template argument
constexpr int kBf16 = 2, kE4m3 = 1, kE2m1 = 0;
inline int format_of(int elem_bytes) { return elem_bytes == KV_ELEM_E2M1 ? kE2m1 : elem_bytes; }

// Where the rows of a layer lie: slot 0 of block 0 of head 0 of K, and the ways from there (bytes).
struct RowLayout {
  char *values;
  long long kv_stride, block_stride, head_stride, slot_stride;
  long long groups, scale, scale_stride;          // from a head's values to its scales of 16 dims; from K's to the scale bytes of head 0, a head
};
inline RowLayout row_layout(const CacheView &c, int layer) {
  RowLayout r;
  r.values = c.base + layer * c.layer_stride;
  r.kv_stride = c.kv_stride;
  r.block_stride = c.block_stride;
  const long long d = c.head_dim;
  if (c.elem_bytes == KV_ELEM_E2M1) {
    r.head_stride = r.scale_stride = c.record_bytes();
    r.slot_stride = d / 2;
    r.groups = c.block_size * (d / 2);
    r.scale = c.block_size * (d / 2 + d / 16);
  } else {
    r.head_stride = d * c.elem_bytes;
    r.slot_stride = c.n_kv_heads * d * c.elem_bytes;
    r.groups = 0;
    r.scale = c.value_bytes();
    r.scale_stride = c.block_size;
  }
  return r;
}
// A lane's pieces of the rows of head `head` of K or V: the first begins at dim `first`, a multiple of 8, the other `apart` dims further on, a
// multiple of 16.
template <int D, int FMT>
struct Pieces {
  char *values, *groups, *scale;
  __device__ __forceinline__ Pieces(const RowLayout &r, int kv, int head, int first) {
    char *page = r.values + kv * r.kv_stride, *row = page + head * r.head_stride;
    values = row + (FMT == kE2m1 ? first / 2 : first * FMT);
    groups = row + r.groups + first / 16;
    scale = page + r.scale + head * r.scale_stride;
  }
};
// bytes of so many dims of a row's values
template <int FMT>
__device__ __forceinline__ int value_bytes_of(int dims) { return FMT == kE2m1 ? dims / 2 : dims * FMT; }

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
  __device__ __forceinline__ void pack(int h, const float (&f)[8]);
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
  __device__ __forceinline__ void pack(int h, const float (&f)[8]) {
    a[h][0] = make_float4(f[0], f[1], f[2], f[3]);
    a[h][1] = make_float4(f[4], f[5], f[6], f[7]);
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
__device__ __forceinline__ void Raw<bf16>::pack(int h, const float (&f)[8]) { a[h] = pack_bf16(f); }
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

// eight e2m1 codes (the first in the low nibble) -> four pairs of fp16, exact.  One byte to a statement: each is then an operand of its
// own conversion, while four out of one unpacking cost two instructions more (3.0 against 2.0 clocks of an SM).  w comes of 32-bit
// loads: fed straight from an 8- or 16-bit load, the unpacking into bytes came out wrong (nvcc 12.9.86).
__device__ __forceinline__ void halves_of_e2m1(uint32_t w, uint32_t (&h)[4]) {
  asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\t}" : "=r"(h[0]) : "r"(w));
  asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, b;\n\t}" : "=r"(h[1]) : "r"(w));
  asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, c;\n\t}" : "=r"(h[2]) : "r"(w));
  asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, d;\n\t}" : "=r"(h[3]) : "r"(w));
}
__device__ __forceinline__ uint32_t mul_half2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ float2 floats_of_half2(uint32_t h) {
  float2 f;
  asm("{\n\t.reg .b16 l, u;\n\tmov.b32 {l, u}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, u;\n\t}"
      : "=f"(f.x), "=f"(f.y) : "r"(h));
  return f;
}
__device__ __forceinline__ uint32_t half2_of_e4m3x2(uint32_t two) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)two));
  return h;
}
// eight values -> codes, nearest; whoever calls it has moved halves off the borders, or looks at them again
__device__ __forceinline__ uint32_t e2m1x8(const float (&f)[8]) {
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\tcvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\tmov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r) : "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7]));
  return r;
}
// The code of y >= 0 in units of the group's scale: the borders that it reaches.  Three comparisons with exact products.
__device__ __forceinline__ uint32_t e2m1_exact(float y, float s) {
  const bool upper = y >= 1.75f * s;
  const float a = upper ? 3.5f * s : 0.75f * s;
  const bool mid = y >= a;
  const float b = upper ? (mid ? 5.f : 2.5f) * s : (mid ? 1.25f : 0.25f) * s;
  return (upper ? 4u : 0u) + (mid ? 2u : 0u) + (y >= b ? 1u : 0u);
}

// The scale of a group whose largest |x| is `top` in units of the row's 2^e: the least positive e4m3 number s with 6 s >= top.
__device__ __forceinline__ uint32_t group_scale(float top, float &s) {
  uint32_t code = e4m3x2(top * (1.f / 6.f), 0.f) & 255u;
  if (6.f * floats_of_half2(half2_of_e4m3x2(code)).x < top) ++code;
  code = min(max(code, 1u), 0x7eu);
  s = floats_of_half2(half2_of_e4m3x2(code)).x;
  return code;
}

// A lane's two pieces of a row into e2m1 codes and the scale codes of their groups, as defined; the lanes of a group are
// neighbours.  Infinities and NaN are left out of the maxima and make their group NaN.  All lanes of the row call it.  Returns the row's
// scale byte.
template <int LANES>
__device__ __forceinline__ uint32_t e2m1_row(const float (&f)[2][8], unsigned group, uint32_t (&codes)[2], uint32_t (&scales)[2]) {
  float most[2] = {0.f, 0.f};
  bool whole[2] = {true, true};
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float a = fabsf(f[h][j]);
      whole[h] &= a <= FLT_MAX;
      most[h] = fmaxf(most[h], a <= FLT_MAX ? a : 0.f);
    }
  float top = fmaxf(most[0], most[1]);
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(group, top, o));
  // |x| = m * 2^x with 1 <= m < 2; 6 * 448 = 1.3125 * 2^11
  const uint32_t bits = __float_as_uint(top);
  int e = (int)(bits >> 23) - 127 - 11 + ((bits & 0x7fffffu) > 0x280000u);
  e = min(max(e, kMinExp), kMaxExpE2m1);
  const float down = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    most[h] = fmaxf(most[h], __shfl_xor_sync(group, most[h], 1));
    const uint32_t other = __shfl_xor_sync(group, whole[h] ? 1u : 0u, 1);
    whole[h] &= other != 0;
    float s;
    scales[h] = group_scale(most[h] * down, s);
    // Quotients that are off by less than 2^-21, moved down and up by 2^-19: where all eight round alike, that is the answer.
    const float inv = __fdividef(1.f, s) * down, less = inv * (1.f - 0x1p-19f), greater = inv * (1.f + 0x1p-19f);
    float a[8], b[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      a[j] = f[h][j] * less;
      b[j] = f[h][j] * greater;
    }
    codes[h] = e2m1x8(a);
    if (codes[h] != e2m1x8(b)) {              // on a border, or next to it
      codes[h] = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        codes[h] |= (e2m1_exact(fabsf(f[h][j]) * down, s) | (__float_as_uint(f[h][j]) >> 31) << 3) << (4 * j);
    }
    if (!whole[h]) {
      codes[h] = 0;
      scales[h] = 0x7fu;      // NaN
    }
  }
  return (uint32_t)(e + 127);
}
// The same for finite bf16 rows.  x has 8 bits and a border 7, so one that is not on a border is 2^-8 away from it, and the quotient
// times 1 + 2^-12 rounds as the comparisons decide, halves up.  `tops`: the largest |x| of the two groups (bf16 patterns), top: of the row.
__device__ __forceinline__ uint32_t e2m1_row(const Raw<bf16> &raw, uint32_t tops, uint32_t top, uint32_t (&codes)[2], uint32_t (&scales)[2]) {
  int e = (int)(top >> 7) - 127 - 11 + ((top & 0x7fu) > 0x28u);
  e = min(max(e, kMinExp), kMaxExpE2m1);
  const float down = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float f[8], s;
    raw.unpack(h, f);
    scales[h] = group_scale(__uint_as_float(h ? tops & 0xffff0000u : tops << 16) * down, s);
    const float up = __fdividef(1.f + 0x1p-12f, s) * down;
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] *= up;
    codes[h] = e2m1x8(f);
  }
  return (uint32_t)(e + 127);
}
// The largest |x| of the two groups that a lane's pieces belong to (bf16 patterns), and of the row.
template <int LANES>
__device__ __forceinline__ void group_tops(const Raw<bf16> &raw, unsigned group, uint32_t &tops, uint32_t &top) {
  const uint32_t s = 0x7fff7fffu;
  const uint32_t x = Raw<bf16>::max2(Raw<bf16>::max2(raw.a[0].x & s, raw.a[0].y & s), Raw<bf16>::max2(raw.a[0].z & s, raw.a[0].w & s));
  const uint32_t y = Raw<bf16>::max2(Raw<bf16>::max2(raw.a[1].x & s, raw.a[1].y & s), Raw<bf16>::max2(raw.a[1].z & s, raw.a[1].w & s));
  tops = Raw<bf16>::max2(__byte_perm(x, y, 0x5410), __byte_perm(x, y, 0x7632));
  tops = Raw<bf16>::max2(tops, __shfl_xor_sync(group, tops, 1));
  uint32_t m = tops;
#pragma unroll
  for (int o = LANES / 2; o > 1; o >>= 1) m = Raw<bf16>::max2(m, __shfl_xor_sync(group, m, o));
  top = max(m & 0xffffu, m >> 16);
}
template <int LANES>
__device__ __forceinline__ void group_tops(const Raw<float> &, unsigned, uint32_t &tops, uint32_t &top) { tops = top = 0xffffu; }
__device__ __forceinline__ uint32_t e2m1_row(const Raw<float> &, uint32_t, uint32_t, uint32_t (&)[2], uint32_t (&)[2]) { return 0; }

// Takes infinities and NaN out of a lane's pieces (zeros in their place); whole[h]: there was none among the 16 dims of piece h.
__device__ __forceinline__ void take_out(Raw<bf16> &raw, unsigned group, bool (&whole)[2]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t w[4] = {raw.a[h].x, raw.a[h].y, raw.a[h].z, raw.a[h].w}, bad = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = (w[i] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u, hi = (w[i] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
      w[i] &= ~(lo | hi);
      bad |= lo | hi;
    }
    raw.a[h] = make_uint4(w[0], w[1], w[2], w[3]);
    whole[h] = (bad | __shfl_xor_sync(group, bad, 1)) == 0;
  }
}
__device__ __forceinline__ void take_out(Raw<float> &, unsigned, bool (&)[2]) {}

// One row, converted and stored by its lanes.  `to`: the lane's pieces in slot 0 of block 0; at = block * block_stride, offset in the block.
template <typename T, int D, int FMT>
__device__ __forceinline__ void put_row(const Raw<T> &raw, const Pieces<D, FMT> &to, long long slot_stride, int apart, long long at,
                                        int offset, int sub, unsigned group, bool live) {
  constexpr int LANES = D / 16;
  char *values = to.values + at + offset * slot_stride, *second = values + value_bytes_of<FMT>(apart);
  if (FMT == kE2m1) {
    uint32_t codes[2], scales[2], tops, top, byte;
    group_tops<LANES>(raw, group, tops, top);
    if (sizeof(T) == 2) {
      Raw<T> fine = raw;
      bool whole[2] = {true, true};
      if (top >= 0x7f80u) {      // the row's lanes all come here
        take_out(fine, group, whole);
        group_tops<LANES>(fine, group, tops, top);
      }
      byte = e2m1_row(fine, tops, top, codes, scales);
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (!whole[h]) {
          codes[h] = 0;
          scales[h] = 0x7fu;      // NaN
        }
    } else {
      float f[2][8];
      raw.unpack(0, f[0]);
      raw.unpack(1, f[1]);
      byte = e2m1_row<LANES>(f, group, codes, scales);
    }
    if (live) {
      *reinterpret_cast<uint32_t *>(values) = codes[0];
      *reinterpret_cast<uint32_t *>(second) = codes[1];
      if ((sub & 1) == 0) {
        char *groups = to.groups + at + (long long)offset * (D / 16);
        groups[0] = (char)scales[0];
        groups[apart / 16] = (char)scales[1];
      }
      if (sub == 0) to.scale[at + offset] = (char)byte;
    }
    return;
  }
  float f[2][8];
  raw.unpack(0, f[0]);
  raw.unpack(1, f[1]);
  if (FMT == kBf16) {
    if (live) {
      *reinterpret_cast<uint4 *>(values) = pack_bf16(f[0]);
      *reinterpret_cast<uint4 *>(second) = pack_bf16(f[1]);
    }
    return;
  }
  uint32_t bits = raw.template top<LANES>(group);
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
    for (int o = LANES / 2; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(group, most, o));
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
    *reinterpret_cast<uint2 *>(second) = c[1];
    if (sub == 0) to.scale[at + offset] = (char)(e + 127);
  }
}

// largest page pool for which slots fit 32 bits: the division by the block size is then a 32-bit one
constexpr long long kSlots32 = 0x7fffffffll;
// The slots of a pool: block and offset of one; false if it lies outside.
struct SlotMap {
  long long n_slots;
  int block_shift, block_size;                    // block_shift: log2(block_size), -1 if it is no power of two
  __device__ __forceinline__ bool split(long long slot, int &block, int &offset) const {
    block = offset = 0;
    if ((unsigned long long)slot >= (unsigned long long)n_slots) return false;
    if (block_shift >= 0)
      block = (int)(slot >> block_shift);
    else if (n_slots <= kSlots32)
      block = (int)((uint32_t)slot / (uint32_t)block_size);
    else
      block = (int)(slot / block_size);
    offset = (int)(slot - (long long)block * block_size);
    return true;
  }
};
inline SlotMap slot_map(const kv_cache_desc *c) {
  SlotMap m;
  m.n_slots = (long long)c->num_blocks * c->block_size;
  m.block_size = c->block_size;
  m.block_shift = -1;
  for (int b = 0; b < 31; ++b)
    if ((1 << b) == c->block_size) m.block_shift = b;
  return m;
}

}  // namespace
}  // namespace kvr
