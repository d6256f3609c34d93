// Attention of one new token per request over a paged cache: ragged requests, bf16, e4m3 or e2m1 pages, split over the
// contexts' length and joined; with one block table for all KV heads of a request, or one for each.
//
//   s_n = scale * q . k_n      o = sum_n 2^(t_n - m) v_n / sum_n 2^(t_n - m)      t = s * log2(e), m = max t
//
// Bound by HBM: each cached row is read once for all the query heads of its group (2 flops per byte and head), so what
// matters is to keep enough loads in flight (135 KB an SM) and every SM equally busy, whatever the lengths.  Measured in a graph /
// call after call in a stream, 64 query and 8 KV heads of 128: 32 requests of up to 18,433 tokens over e4m3 pages (512 MB)
// 89 / 92 us, 5.7 / 5.6 TB/s (97 to 102 us after seconds of it, when the power cap has taken the clock from 1.97 to 1.64 GHz);
// 16 of up to 8,192 over bf16 pages (305 MB) 55 / 57 us, 5.6 / 5.3 TB/s; one of 18,433 (38 MB) 16 / 18.5 us, of which 9 us are
// the fixed cost of a split call.
//
// Split.  The contexts of all requests are laid end to end in tiles (and one more for each request) and cut into equal
// ranges, one per CTA column, so one long request and a hundred short ones load the machine alike.  A range that holds a
// whole request writes its output; otherwise it leaves a record (m, l, o) and a second, small kernel joins the records
// of a request.  Lengths live on the device, so every CTA finds its own range with a scan over them.
//
// A warp works alone: it copies 16 or 32 keys of one KV head (K and V rows, 16 bytes per cp.async, whole rows per instruction)
// into a ring of its own and consumes them stage by stage with no barrier but the warp's, so loads never wait for other
// warps and run on across the end of a request.  Four warps of a CTA take four KV heads (batches: neighbouring heads'
// rows are neighbouring memory), or every fourth stage of one KV head (few requests: four times fewer records; their
// results meet in shared memory).
//
// The products run on mma.sync m16n8k16 with the keys (S^T = K Q^T) and the head's dims (O^T = V^T P^T) as the 16 rows and
// the query heads as the 8 columns: a KV group has 8 heads or fewer, so nothing is padding.  (A 128-row tcgen05 tile would
// hold 8 useful columns of at least 16 as well, but wants its operands through shared-memory descriptors, and e4m3 rows
// would have to be converted and written back there first.)  Groups of more than 8 heads are taken 8 at a time, each time with
// a copy of K and V from L2 (16 requests of up to 8,192, 64 / 128 / 256 query heads: 36 / 55 / 99 us, over bf16 pages 56 / 67 / 115).
// fp32 operands go in as sums of 16-bit parts that are multiplied one after the other.  Over e4m3 and e2m1 pages q and the weights p
// are two fp16: off by 2^-22 of themselves, and by up to 2^-36 of the query's largest value or of the request's largest contribution
// so far, where fp16 ends (a bf16 query is one part: exact down to 2^-28 of its largest value).
// Over bf16 pages they are three bf16 in fp32 calls (2^-24); in bf16 calls q is one part, exact, and p two (2^-16, a 256th of
// the rounding of the result; the sum of the weights, and lse, take them whole).  The second part of the weights costs bf16
// calls over e4m3 pages 0.5 % (128 requests of up to 577 tokens: 1.6 %): the loads are what bounds them.
//
// The running maximum is lazy: m is replaced only when a score passes it by more than 2^8 (e4m3 pages: 2^4, for the head room
// goes to small fp16 weights), so most stages need no reduction over the lanes and no rescaling.
//
// e4m3 pages: codes go to fp16 fragments (exact) and the power-of-two scales stay outside: K's multiplies the score,
// V's goes into the weight, w = 2^(t - m + e_v - M), with a running maximum M of t - m + e_v of its own, so that fp16 keeps the bits
// of every weight that matters next to the largest CONTRIBUTION, however the rows' scales differ.
//
// e2m1 pages: the same, and the scale of 16 dims is multiplied into the fp16 fragment (code times e4m3 number: six bits, exact).  The
// codes of two keys of V are paired as nibbles, before they are converted, so the fragments of V^T need no exchange after it.  In pages of a
// multiple of 16 slots a unit of 16 keys (codes, scales, scale bytes: three pieces of the record) is copied as it is, 1,168 bytes of K or V for
// 128 dims; in other pages row by row.  What bounds it is no longer HBM but instructions: 397 a warp for 16 keys and 8 heads, half of them
// conversions, scales and products, at 59 % of the issue slots (ALU pipe 46 %, tensor 29 %).  So bf16 calls have twelve warps an
// SM.  32 requests of up to 18,433 tokens (290 MB) 83 us in a graph, 87 call after call: 3.5 TB/s, against 91 us for the 512 MB of e4m3
// pages; the copies alone take 50.  (Weights of one fp16 part, 2^-11, would take 76 us, but last bits of bf16 results then move: 4e-4 of
// their norm off what fp32 weights give, against 5e-5.)  fp32 calls (two parts each, eight warps an SM) 102 us; a third CTA for them spills and is as
// often slower as faster (two / three: 128 requests of up to 577 tokens 28.8 / 28.2, 64 of 1,024 39.2 / 43.0).
#include "cache_format.cuh"

namespace kvr {
namespace {

constexpr int kBaWarps = 4;
constexpr int kBaWide = 8;           // warps that share a KV head where whole contexts are so few that each has an SM to itself
constexpr int kBaHeads = 8;          // query heads of a pass
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kLookAhead = 3;        // stages between looking a page up and copying its rows
constexpr int kNoRow = (int)0x80000000;
template <int ELEM>
constexpr float kLazy = ELEM == 2 ? 8.f : 4.f;      // a running maximum may be passed by 2^4 (2^8) before it is replaced
constexpr float kWeightBits = 11.f;  // fp16 weights: 2^11 at the running maximum, so at most 2^15
constexpr int kQueryBits = 12;       // ... and fp16 queries to less than 2^12

// A stage is what a warp loads and consumes at a time: 32 keys, so that the softmax's and the loads' bookkeeping is paid
// once for four 8-key fragments; 16 where 32 would leave the ring too few stages (bf16 rows of 128: 8 KB a stage either way).
// ELEM, the page format: 2 bf16, 1 e4m3, 0 e2m1, kUnits e2m1 in pages whose size is a multiple of 16: then 16 keys of a KV head and all
// that belongs to them lie in three pieces of the head's record (one, in pages of 16), which are copied as they are.
constexpr int kUnits = -1;
// CTAs of an SM: e2m1 pages and bf16 queries three, whose registers and rings fit (many instructions for few bytes: the more warps
// the better), two otherwise.
constexpr int ba_ctas(bool e2m1, bool bf16_queries) { return e2m1 && bf16_queries ? 3 : 2; }
__host__ __device__ constexpr int ba_warps(int kw) { return kw > kBaWarps ? kw : kBaWarps; }
template <int D, int ELEM, typename T>
struct BaCfg {
  static constexpr int row = ELEM <= 0 ? D / 2 : D * ELEM;               // bytes of a K or V row's values
  static constexpr int keys = row > 128 ? 16 : 32;
  static constexpr int codes = keys * row;
  static constexpr int unit = 16 * (D / 2 + D / 16 + 1);                 // 16 keys of an e2m1 record: codes, scales of 16 dims, scale bytes
  static constexpr int tile = ELEM == kUnits ? keys / 16 * unit : ELEM == 0 ? codes + keys * (D / 16) : codes;
  static constexpr int stage = 2 * tile + (ELEM == 2 || ELEM == kUnits ? 0 : 256);      // K, V, a word with the scale byte of each row
  static constexpr int stages = stage > 6144 || (ba_ctas(ELEM <= 0, sizeof(T) == 2) == 3 && D == 128) ? 3 : 5;
  static constexpr int ring = stages * stage;
  // outputs of warps 1-3 when they share a head; those of a wide CTA, which has one request, take the rings' place
  static constexpr int merge(int kw) { return kw == 1 ? 0 : (kw - 1) * kBaHeads * D * 4; }
  static constexpr int smem(int kw) { return kw <= kBaWarps ? kBaWarps * ring + merge(kw) : kw * ring > merge(kw) ? kw * ring : merge(kw); }
};

struct BaParams {
  CacheView cache;
  int layer, num_blocks, block_shift;
  int aligned16;          // block_size is a multiple of 16: 16 keys that start at a multiple of 16 share a page
  const void *q;
  void *out;
  float *lse;
  long long q_stride, out_stride, table_stride, head_stride;      // head_stride: from a KV head's table to the next, 0 if they share one
  const int *tables, *lens;
  int n_req, n_q_heads, group, passes, max_ctx;
  int parts;              // ranges; 0: one CTA per request (blockIdx.x), nothing is split
  float scale;            // softmax_scale * log2(e)
  long long *tile_start;  // scratch: [n_req + 1]
  float2 *ml;             // scratch: (m, l) per (query head, part, first | last)
  float *o;               // scratch: [D] each
};

__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// 16 bytes, or zeros.  e4m3 rows are 128 or 64 bytes and the next head's follow: L2 fetches 256 bytes at once (32 requests
// of up to 18,433 tokens: 94.6 us against 99.1 us; no gain for bf16 rows).
template <int ELEM>
__device__ __forceinline__ void cp16(uint32_t dst, const char *src, bool valid) {
  if (ELEM != 2)
    asm volatile("cp.async.cg.shared.global.L2::256B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
  else
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
}
template <int ELEM>
__device__ __forceinline__ void cp16(uint32_t dst, const char *src) {
  asm volatile("cp.async.cg.shared.global.L2::256B [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp4(uint32_t dst, const char *src, bool valid) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(valid ? 4 : 0) : "memory");
}
__device__ __forceinline__ void cp8(uint32_t dst, const char *src, bool valid) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(valid ? 8 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait_group() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_trans(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint4 lds16(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds8(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t lds4(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t lds2(uint32_t a) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t lds1(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
// x and y as the sum of N bf16 each (8 significant bits a part) or of N fp16 (11): what a part leaves goes to the next.
template <int N>
__device__ __forceinline__ void split_bf16(float x, float y, uint32_t (&parts)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
    const float2 f = __bfloat1622float2(h);
    parts[i] = *reinterpret_cast<const uint32_t *>(&h);
    x -= f.x;
    y -= f.y;
  }
}
template <int N>
__device__ __forceinline__ void split_f16(float x, float y, uint32_t (&parts)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(parts[i]) : "f"(y), "f"(x));
    float fx, fy;
    asm("{\n\t.reg .b16 l, u;\n\tmov.b32 {l, u}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, u;\n\t}"
        : "=f"(fx), "=f"(fy) : "r"(parts[i]));
    x -= fx;
    y -= fy;
  }
}
// Two fp32 operations in one instruction: the scores of a lane's two heads.
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 r;
  asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmul.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {      // NaN only if all are
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
template <int N>
__device__ __forceinline__ float2 max_of(const float2 (&t)[N]) {
  if (N == 2) return make_float2(fmaxf(t[0].x, t[1].x), fmaxf(t[0].y, t[1].y));
  return make_float2(fmaxf(max3(t[0].x, t[1].x, t[2 % N].x), t[3 % N].x), fmaxf(max3(t[0].y, t[1].y, t[2 % N].y), t[3 % N].y));
}
// c += A B for the parts of B.  The matrix instruction truncates as it accumulates, some 2^-24 of the accumulator each time and always
// towards zero: over the tiles of a long context that adds up to more than fp32 results should lose.  So fp32 calls over bf16 and e2m1
// pages start from zero and add what comes out, rounded (APART; of the results' norm, 1,024 keys of 128 requests 1.2e-7, 16,384 3.5e-7, which accumulated
// inside would be 3e-5 to 5e-5).  Over e4m3 pages they accumulate inside, as bf16 calls do, whose own rounding is far larger: 1,024
// keys of 128 requests 9e-7, 16,384 of one request 1e-7, of 16 3e-6, of 128 4e-5; apart, these calls would take 2 to 9 % longer.
template <bool APART, bool BF16, int N, int M>
__device__ __forceinline__ void add_product(float (&c)[4], const uint32_t (&a)[4], const uint32_t (&b)[N][M], int at) {
  float own[4] = {};
  float (&to)[4] = APART ? own : c;
#pragma unroll
  for (int h = 0; h < N; ++h) {
    if (BF16)
      mma_bf16(to, a, b[h][at], b[h][at + 1]);
    else
      mma_f16(to, a, b[h][at], b[h][at + 1]);
  }
  if (APART) {
    const float2 x = add2(make_float2(c[0], c[1]), make_float2(own[0], own[1])), y = add2(make_float2(c[2], c[3]), make_float2(own[2], own[3]));
    c[0] = x.x; c[1] = x.y; c[2] = y.x; c[3] = y.y;
  }
}
// 8x8 16-bit values, two of a row to a lane -> the same of the transposed block
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
// The D / 4 values of a query head that a lane (c = lane % 4) turns into fragments, as they were loaded.  Pair i of
// ELEM 2 is dims 8 i + 2 c, + 1; of the others dims c D / 4 + 2 i, + 1.
template <int D, int ELEM, typename T>
struct RawQuery {
  static constexpr int W = sizeof(T) / 2;            // 32-bit words of a pair
  uint32_t w[D / 8 * W];
  __device__ __forceinline__ void load(const T *q, int c) {
    if (ELEM != 2) {
      const uint4 *src = reinterpret_cast<const uint4 *>(q + c * (D / 4));
#pragma unroll
      for (int i = 0; i < D / 8 * W / 4; ++i) {
        const uint4 x = src[i];
        w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        if (W == 1) {
          w[i] = *reinterpret_cast<const uint32_t *>(q + 8 * i + 2 * c);
        } else {
          const uint2 x = *reinterpret_cast<const uint2 *>(q + 8 * i + 2 * c);
          w[W * i] = x.x; w[W * i + W - 1] = x.y;
        }
      }
    }
  }
  __device__ __forceinline__ float2 pair(int i) const {
    if (W == 1) return make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    return make_float2(__uint_as_float(w[W * i]), __uint_as_float(w[W * i + W - 1]));
  }
};
// x, or NaN for an infinity: results say that something infinite entered them in one way, however it met the parts of a
// weight or of a query (infinity times a positive part, a negative one or zero).
__device__ __forceinline__ float nan_of_inf(float x) { return fmaf(x, 0.f, x); }
__device__ __forceinline__ void store4(float *p, float a, float b, float c, float d) {
  *reinterpret_cast<float4 *>(p) = make_float4(a, b, c, d);
}
__device__ __forceinline__ void store4(bf16 *p, float a, float b, float c, float d) {
  const __nv_bfloat162 x = __floats2bfloat162_rn(a, b), y = __floats2bfloat162_rn(c, d);
  *reinterpret_cast<uint2 *>(p) = make_uint2(*reinterpret_cast<const uint32_t *>(&x), *reinterpret_cast<const uint32_t *>(&y));
}
__device__ __forceinline__ void store2(float *p, float a, float b) { *reinterpret_cast<float2 *>(p) = make_float2(a, b); }
__device__ __forceinline__ void store2(bf16 *p, float a, float b) {
  *reinterpret_cast<__nv_bfloat162 *>(p) = __floats2bfloat162_rn(a, b);
}
// The lane's share of the D values (times f) of head cq + i.  ELEM 2: dims 16 mt + lane / 4 + {0, 8}; the others: D / 8
// consecutive ones.
template <int D, int ELEM, typename P>
__device__ __forceinline__ void store_head(P *row, const float (&oc)[D / 16][4], int i, int g, float f) {
  if (ELEM == 2) {
#pragma unroll
    for (int mt = 0; mt < D / 16; ++mt) {
      row[mt * 16 + g] = (P)nan_of_inf(oc[mt][i] * f);
      row[mt * 16 + g + 8] = (P)nan_of_inf(oc[mt][2 + i] * f);
    }
  } else {
#pragma unroll
    for (int mt = 0; mt < D / 16; mt += 2)
      store4(row + g * (D / 8) + 2 * mt, nan_of_inf(oc[mt][i] * f), nan_of_inf(oc[mt][2 + i] * f), nan_of_inf(oc[mt + 1][i] * f),
             nan_of_inf(oc[mt + 1][2 + i] * f));
  }
}
__device__ __forceinline__ float column_max(float v) {      // over the eight lanes that share lane % 4
  v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 4));
  v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 8));
  return fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 16));
}
__device__ __forceinline__ float quad_max(float v) {
  v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 1));
  return fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 2));
}

// Byte offset of 16-byte chunk c of row r in a tile: chunks are permuted inside 128-byte lines so that the fragment
// loads of eight neighbouring lanes fall into different banks.
template <int D, int ELEM>
__device__ __forceinline__ uint32_t chunk_at(int r, int c) {
  if (ELEM <= 0) return (uint32_t)(r * (D / 2) + (ELEM == 0 && D == 128 ? c ^ (r & 2) : c) * 16);
  if (ELEM == 1 && D == 64) return (uint32_t)((r >> 1) * 128 + ((((r & 1) * 4 + c) ^ (r & 6)) * 16));
  if (ELEM == 1) return (uint32_t)(r * 128 + ((c ^ (r & 7)) * 16));
  return (uint32_t)(r * (D * 2) + ((c & ~7) | ((c ^ r) & 7)) * 16);
}

// The key (of eight) that row x of a fragment holds.  e2m1 rows are 64 or 32 bytes, so that four of them, in natural order, would
// share banks; any order will do, as long as K's rows and the weights agree.
template <int ELEM>
__device__ __forceinline__ int key_of(int x) { return ELEM <= 0 ? x ^ (x >> 2) : x; }

__device__ __forceinline__ int clamped_len(const BaParams &p, int r) {
  return min(max(__ldg(p.lens + r), 0), p.max_ctx);
}

// Tiles of a request of n keys.  One more than its keys need: starting and finishing a request (query fragments, sums over
// the lanes, the result) takes as long as a tile, and a request of no keys has to be somebody's (128 requests of up to 577
// tokens: 25.7 us against 27.8 us without it).
__device__ __forceinline__ int tiles_of(int n, int tile_keys) { return (n + tile_keys - 1) / tile_keys + 1; }

// Sum over the lanes up to this one.
__device__ __forceinline__ int warp_scan(int v, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += up;
  }
  return v;
}

// Whether a bf16 key among `steps` stages of KEYS keys, the first at position `first`, each `tile` further on, holds an infinity or
// NaN.  Hardly ever called, so it stands apart: in the kernel it cost a call for one request of 161 tokens 0.15 of 4.5 us.
template <int KEYS>
__device__ __noinline__ bool infinite_key(const BaParams &p, int req, int kvh, int first, int tile, int steps, int n) {
  const int lane = threadIdx.x & 31, row_bytes = p.cache.head_dim * 2;
  bool found = false;
  for (int s = 0; s < steps; ++s) {
    const int pos = first + s * tile + lane % KEYS;
    if (pos >= n) continue;
    const int b = pos / p.cache.block_size, blk = __ldg(p.tables + req * p.table_stride + kvh * p.head_stride + b);
    if ((unsigned)blk >= (unsigned)p.num_blocks) continue;
    const char *row = p.cache.page(p.layer, 0, blk) +
                      ((long long)(pos - b * p.cache.block_size) * p.cache.n_kv_heads + kvh) * row_bytes;
    for (int i = lane / KEYS * 16; i < row_bytes; i += 32 / KEYS * 16) {
      const uint4 x = *reinterpret_cast<const uint4 *>(row + i);
      const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) found |= (w[j] & 0x7f80u) == 0x7f80u || (w[j] & 0x7f800000u) == 0x7f800000u;
    }
  }
  return __any_sync(0xffffffffu, found);
}

// Where a warp stands in the sequence of tiles of its range.
struct Cursor {
  int r, tile, n_tiles, n, n_next;
  __device__ __forceinline__ void open(const BaParams &p, int req, int tile_keys) {
    r = req;
    n = r < p.n_req ? clamped_len(p, r) : 0;
    n_next = r + 1 < p.n_req ? clamped_len(p, r + 1) : 0;
    n_tiles = tiles_of(n, tile_keys);
    tile = 0;
  }
  __device__ __forceinline__ void step(const BaParams &p, int tile_keys) {
    if (++tile < n_tiles) return;
    ++r;
    n = n_next;
    n_next = r + 1 < p.n_req ? clamped_len(p, r + 1) : 0;      // loaded a request ahead
    n_tiles = tiles_of(n, tile_keys);
    tile = 0;
  }
};

template <int D, int ELEM, typename T, int KW>      // KW: warps that share a KV head
__global__ void __launch_bounds__(ba_warps(KW) * 32, KW == kBaWide ? 1 : ba_ctas(ELEM <= 0, sizeof(T) == 2))
    paged_attention_batched_kernel(const __grid_constant__ BaParams p) {
  typedef BaCfg<D, ELEM, T> C;
  constexpr bool WIDE = KW > kBaWarps;       // whole contexts only
  constexpr int WARPS = ba_warps(KW);
  constexpr int KS = D / 16;                 // k-steps of S^T = K Q^T
  constexpr int NT = D / 8;                  // dims of a lane's V fragments (ELEM 1, 0)
  constexpr int MO = D / 16;                 // 16-dim tiles of O^T
  constexpr int QP = sizeof(T) == 2 ? 1 : (ELEM == 2 ? 3 : 2);          // parts of a query
  constexpr int PP = sizeof(T) == 4 && ELEM == 2 ? 3 : 2;      // parts of a weight
  constexpr int CH = C::row / 16;            // 16-byte chunks of a row
  constexpr int RPI = 32 / CH;               // rows per copy instruction
  constexpr int KEYS = C::keys;
  constexpr int MK = KEYS / 16;              // 16-key tiles of S^T
  constexpr int TILE = KW * KEYS;            // keys of a tile of the split
  extern __shared__ __align__(128) unsigned char ba_smem[];
  __shared__ float2 ml_s[2][WARPS][kBaHeads];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int kg = warp % KW;                                        // which of the tile's stages
  const int vh = blockIdx.y * (WARPS / KW) + warp / KW;         // (KV head, pass over its query heads)
  if (KW == 1 && vh >= p.cache.n_kv_heads * p.passes) return;
  const int kvh = vh / p.passes, pass = vh % p.passes;
  const int head0 = kvh * p.group + pass * kBaHeads, nh = min(kBaHeads, p.group - pass * kBaHeads);
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(ba_smem) + warp * C::ring;

  // ---- this CTA's range of tiles
  Cursor cons;
  long long todo, total = 0, first_tile = 0;
  const int part = blockIdx.x;
  if (WIDE || p.parts == 0) {
    cons.open(p, blockIdx.x, TILE);
    todo = cons.n_tiles;
  } else {
    // 128 requests at a time, four to a lane, whose lengths are loaded together; a batch of up to 128 keeps them
    int tiles[4];
    auto load_tiles = [&](int r0) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = r0 + j * 32 + lane;
        tiles[j] = r < p.n_req ? clamped_len(p, r) : -1;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) tiles[j] = tiles[j] < 0 ? 0 : tiles_of(tiles[j], TILE);
    };
    for (int r0 = 0; r0 < p.n_req; r0 += 128) {
      load_tiles(r0);
      total += __reduce_add_sync(0xffffffffu, tiles[0] + tiles[1] + tiles[2] + tiles[3]);
    }
    // no more ranges than tiles: every range that is left holds one (the joining kernel counts on it)
    const long long ranges = min((long long)p.parts, total);
    if (part >= ranges) return;
    if ((part + 1) * total <= 0xffffffffll) {
      first_tile = (uint32_t)(part * total) / (uint32_t)ranges;
      todo = (uint32_t)((part + 1) * total) / (uint32_t)ranges - first_tile;
    } else {
      first_tile = part * total / ranges;
      todo = (part + 1) * total / ranges - first_tile;
    }
    long long before = 0;
    int at = -1;
    for (int r0 = 0; at < 0; r0 += 128) {
      if (p.n_req > 128) load_tiles(r0);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (at >= 0) break;
        const int inc = warp_scan(tiles[j], lane), sum = __shfl_sync(0xffffffffu, inc, 31);
        if (first_tile < before + sum) {
          const int l = __ffs(__ballot_sync(0xffffffffu, first_tile < before + inc)) - 1;
          at = r0 + j * 32 + l;
          before += __shfl_sync(0xffffffffu, inc - tiles[j], l);
        } else {
          before += sum;
        }
      }
    }
    cons.open(p, at, TILE);
    cons.tile = (int)(first_tile - before);
  }

  asm volatile("griddepcontrol.launch_dependents;");      // the joining kernel may be put in place

  // ---- loads.  Lane l looks up the page of row l % KEYS of a stage, kLookAhead stages before its copies are issued: a
  // table entry can be a microsecond away.
  const int *tables = p.tables + kvh * p.head_stride;
  Cursor prod = cons;
  long long to_look = todo;
  int blks[kLookAhead] = {}, offs[kLookAhead] = {};   // of the next stages to be copied: block and slot of the lane's row (kNoRow: none)
  const int my_row = lane % KEYS;
  // e2m1 units: the lanes' unit begins at `at` (lanes 0 to 15 the first of the stage, the others the second)
  int at = (prod.tile * KW + kg) * KEYS + (lane & 16);
  const int *table = tables + prod.r * p.table_stride;
  auto look_up_unit = [&](int &blk, int &off) {
    off = kNoRow;
    if (to_look > 0) {
      if (at < prod.n) {
        int b;
        if (p.block_shift >= 0) {
          b = at >> p.block_shift;
          off = at & (p.cache.block_size - 1);
        } else {
          b = at / p.cache.block_size;
          off = at - b * p.cache.block_size;
        }
        blk = __ldg(table + b);
      }
      --to_look;
      at += TILE;
      const int r = prod.r;
      prod.step(p, TILE);
      if (prod.r != r) {
        at = kg * KEYS + (lane & 16);
        table = tables + prod.r * p.table_stride;
      }
    }
  };
  auto look_up = [&](int &blk, int &off) {
    if (ELEM == kUnits) {
      look_up_unit(blk, off);
      return;
    }
    const int pos = (prod.tile * KW + kg) * KEYS + my_row;
    blk = -1;
    off = 0;
    if (to_look > 0) {
      if (pos < prod.n) {
        const int b = p.block_shift >= 0 ? pos >> p.block_shift : pos / p.cache.block_size;
        off = pos - b * p.cache.block_size;
        blk = __ldg(tables + prod.r * p.table_stride + b);
      }
      off |= pos < prod.n ? 0 : kNoRow;
      --to_look;
      prod.step(p, TILE);
    } else {
      off = kNoRow;
    }
  };
  const long long row_stride = ELEM <= 0 ? C::row : (long long)p.cache.n_kv_heads * C::row;
  // the lane's chunk of row lane / CH, and the scale bytes, in block 0 of K (e2m1: both in the KV head's record)
  const char *rec0 = p.cache.page(p.layer, 0, 0) + kvh * (ELEM <= 0 ? p.cache.record_bytes() : (long long)C::row);
  const char *base0 = rec0 + (lane / CH) * row_stride + (lane % CH) * 16;
  const char *scale0 = ELEM <= 0 ? rec0 + (long long)p.cache.block_size * (D / 2 + D / 16)
                                 : p.cache.page(p.layer, 0, 0) + p.cache.value_bytes();
  unsigned poison = 0;                       // bit s: the stage in ring slot s has a row outside the pool
  int put = 0;                               // ring slot to fill next
  auto advance = [&]() {
    put = put + 1 == C::stages ? 0 : put + 1;
#pragma unroll
    for (int i = 0; i + 1 < kLookAhead; ++i) {
      blks[i] = blks[i + 1];
      offs[i] = offs[i + 1];
    }
    look_up(blks[kLookAhead - 1], offs[kLookAhead - 1]);
  };
  // The unit of lanes 0 to 15 and that of the others, by all lanes: 16 rows of codes, then the piece of scales of 16 dims or of scale bytes that
  // is the lane's.  What a context leaves of its last unit comes along (and is kept from the results below); a unit behind it does not.
  constexpr int CODES = 16 * (D / 2) / 512, EXTRA = D / 16 + 1;      // copies of a lane; lanes that have a piece behind the codes
  const long long extra0 = lane < D / 16 ? (long long)p.cache.block_size * (D / 2) + lane * 16 : (long long)p.cache.block_size * (D / 2 + D / 16);
  const int extra_step = lane < D / 16 ? D / 16 : 1;
  auto issue_units = [&]() {
    const bool is = offs[0] >= 0, inside = is && (unsigned)blks[0] < (unsigned)p.num_blocks;
    if (__any_sync(0xffffffffu, is != inside)) poison |= 1u << put;
    const uint32_t dst0 = ring + put * C::stage + lane * 16;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int blk = __shfl_sync(0xffffffffu, inside ? blks[0] : -1, u * 16), off = __shfl_sync(0xffffffffu, offs[0], u * 16);
      if (blk >= 0) {
        const char *rec = rec0 + blk * p.cache.block_stride;
        const char *codes = rec + (long long)off * (D / 2) + lane * 16, *extra = rec + extra0 + off * extra_step;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          const uint32_t dst = dst0 + u * C::unit + kv * C::tile;
#pragma unroll
          for (int i = 0; i < CODES; ++i) cp16<ELEM>(dst + i * 512, codes + i * 512);
          if (lane < EXTRA) cp16<ELEM>(dst + CODES * 512, extra);
          codes += p.cache.kv_stride;
          extra += p.cache.kv_stride;
        }
      }
    }
    cp_commit();
    advance();
  };
  auto issue = [&]() {
    if (ELEM == kUnits) {
      issue_units();
      return;
    }
    const bool row_is = offs[0] >= 0;                                            // the lane's row is one of the context
    const int blk = row_is && (unsigned)blks[0] < (unsigned)p.num_blocks ? blks[0] : -1;      // -1: never followed
    const int off = row_is ? offs[0] : 0;
    const bool any = __any_sync(0xffffffffu, row_is);
    const bool bad = __any_sync(0xffffffffu, row_is && blk < 0);
    poison = (poison & ~(1u << put)) | ((unsigned)bad << put);
    if (any) {
      const uint32_t k_s = ring + put * C::stage, v_s = k_s + C::tile;
      const int sub = lane / CH, c = lane % CH;
      const unsigned live = __ballot_sync(0xffffffffu, blk >= 0);
      if (p.aligned16) {      // one address per 16 rows
#pragma unroll
        for (int half = 0; half < KEYS / 16; ++half) {
          const int b = __shfl_sync(0xffffffffu, blk, half * 16), o = __shfl_sync(0xffffffffu, off, half * 16);
          const char *src = base0 + (b >= 0 ? b * p.cache.block_stride + o * row_stride : 0);
#pragma unroll
          for (int i = 0; i < 16 / RPI; ++i) {
            const int row = half * 16 + i * RPI + sub;
            const bool ok = (live >> row) & 1u;
            const uint32_t dst = chunk_at<D, ELEM>(row, c);
            cp16<ELEM>(k_s + dst, src, ok);                             // rows that are not there are zeros
            cp16<ELEM>(v_s + dst, src + p.cache.kv_stride, ok);
            src += RPI * row_stride;
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < KEYS / RPI; ++i) {
          const int row = i * RPI + sub;
          const int b = __shfl_sync(0xffffffffu, blk, row), o = __shfl_sync(0xffffffffu, off, row);
          const bool ok = b >= 0;
          const char *src = base0 + (ok ? b * p.cache.block_stride + (o - sub) * row_stride : 0);
          const uint32_t dst = chunk_at<D, ELEM>(row, c);
          cp16<ELEM>(k_s + dst, src, ok);
          cp16<ELEM>(v_s + dst, src + p.cache.kv_stride, ok);
        }
      }
      if (ELEM != 2) {   // the words that hold the scale bytes of row l of K and of V
        const bool ok = blk >= 0;
        if (ELEM <= 0) {      // ... and its scales of 16 dims
          const char *src = rec0 + (ok ? blk * p.cache.block_stride : 0) + (long long)p.cache.block_size * (D / 2) + (ok ? off : 0) * (D / 16);
          const uint32_t dst = k_s + C::codes + lane * (D / 16);
          if (D == 128) {
            cp8(dst, src, ok);
            cp8(dst + C::tile, src + p.cache.kv_stride, ok);
          } else {
            cp4(dst, src, ok);
            cp4(dst + C::tile, src + p.cache.kv_stride, ok);
          }
        }
        const int at = (ELEM <= 0 ? 0 : kvh * p.cache.block_size) + (ok ? off : 0);
        const char *src = scale0 + (ok ? blk * p.cache.block_stride : 0) + (at & ~3);
        cp4(k_s + 2 * C::tile + lane * 4, src, ok);
        cp4(k_s + 2 * C::tile + 128 + lane * 4, src + p.cache.kv_stride, ok);
      }
    }
    cp_commit();
    advance();
  };
#pragma unroll
  for (int i = 0; i < kLookAhead; ++i) look_up(blks[i], offs[i]);
  const int g = lane >> 2, c = lane & 3, cq = c * 2;   // the lane's query fragments are of head g, its results of cq, cq + 1
  const int kg8 = key_of<ELEM>(g);                     // of eight keys, the one that row g of a fragment holds
  RawQuery<D, ELEM, T> raw;
  auto load_query = [&](int req) {
    raw.load(static_cast<const T *>(p.q) + req * p.q_stride + (long long)(head0 + min(g, nh - 1)) * D, c);
  };
  load_query(cons.r);
#pragma unroll
  for (int i = 0; i < C::stages - 1; ++i) issue();

  // ---- per request of the range
  int get = 0, seg = 0;
  long long done = 0;
  while (todo > 0) {
    const int req = cons.r, n = cons.n, s_tile = cons.tile;
    const int steps = (int)min((long long)(cons.n_tiles - s_tile), todo);
    // for the joining kernel: where the request's tiles start
    if (!WIDE && p.parts > 0 && s_tile == 0 && blockIdx.y == 0 && threadIdx.x == 0) {
      p.tile_start[req] = first_tile + done;
      if (req == 0) p.tile_start[p.n_req] = total;
    }
    done += steps;
    uint32_t qf[QP][KS][2];
    // What makes scores (log2 units) of the products: q_pre, a power of two, ahead of the key's 2^e, and q_scale behind it.
    float2 q_pre = {1.f, 1.f}, q_scale = {p.scale, p.scale};
    {
      const float on = g < nh ? 1.f : 0.f;
      if (ELEM == 2) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float2 a = raw.pair(2 * ks + j);
            uint32_t parts[QP];
            split_bf16(nan_of_inf(a.x) * on, nan_of_inf(a.y) * on, parts);      // a bf16 query is its own one part
#pragma unroll
            for (int h = 0; h < QP; ++h) qf[h][ks][j] = parts[h];
          }
        }
      } else {
        // the lane's dims: 4 KS consecutive ones, so that a key's codes are read as 16-byte vectors
        float x[4 * KS], most = 0.f;
#pragma unroll
        for (int i = 0; i < 2 * KS; ++i) {
          const float2 a = raw.pair(i);
          x[2 * i] = a.x * on;
          x[2 * i + 1] = a.y * on;
          most = fmaxf(most, fmaxf(fabsf(x[2 * i]), fabsf(x[2 * i + 1])));
        }
        most = quad_max(most);
        const int e = min(max((int)(__float_as_uint(most) >> 23) - 126, -100), 127);       // most < 2^e
        // NaN times everything where the largest is infinite
        const float up = __uint_as_float(most <= FLT_MAX ? (uint32_t)(127 + kQueryBits - e) << 23 : 0x7fc00000u);
        // Products, below 2^31, are in units of 2^(e - kQueryBits); with the power of two of p.scale, 2^whole.  All of it goes to q_pre
        // within 2^-100 .. 2^96, so that nothing on the way leaves fp32 where the score does not: product * q_pre stays below 2^127, and what is
        // left for q_scale is 1 to 2 there, more above (the score is then the largest of all), less below (where scores are 0).
        const uint32_t bits = __float_as_uint(p.scale);
        const int whole = e - kQueryBits + (int)(bits >> 23) - 127;
        const int rest = min(max(whole - min(max(whole, -100), 96), -126), 126);      // no zero: times the -inf of a key that is not there it would be NaN
        const float pre = __uint_as_float((uint32_t)(127 + whole - rest) << 23), post = __uint_as_float((bits & 0x7fffffu) | (uint32_t)(127 + rest) << 23);
        q_pre.x = __shfl_sync(0xffffffffu, pre, cq * 4);
        q_pre.y = __shfl_sync(0xffffffffu, pre, cq * 4 + 4);
        q_scale.x = __shfl_sync(0xffffffffu, post, cq * 4);
        q_scale.y = __shfl_sync(0xffffffffu, post, cq * 4 + 4);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            uint32_t parts[QP];
            split_f16(x[4 * ks + 2 * j] * up, x[4 * ks + 2 * j + 1] * up, parts);      // bf16: exact in one
#pragma unroll
            for (int h = 0; h < QP; ++h) qf[h][ks][j] = parts[h];
          }
        }
      }
    }
    // per head cq + i: running maxima, m of the scores in units of q_scale and mw of score + e_v (not ELEM 2) in log2 units from m on (-inf:
    // none yet, then 0 is subtracted), the lane's sum
    float2 m = {-INFINITY, -INFINITY}, mw = m, l = {};
    float2 m_neg = {}, w_neg = {};      // what is added to scores, and in the exponents of the weights
    float low = INFINITY;      // ELEM 2: the lowest product
    float oc[MO][4];
#pragma unroll
    for (int mt = 0; mt < MO; ++mt)
#pragma unroll
      for (int i = 0; i < 4; ++i) oc[mt][i] = 0.f;

    for (int s = 0; s < steps; ++s) {
      cp_wait_group<C::stages - 2>();
      __syncwarp();
      issue();                                        // into the slot that the previous step has left
      const uint32_t k_s = ring + get * C::stage, v_s = k_s + C::tile;
      const int key0 = (cons.tile * KW + kg) * KEYS;
      if (key0 < n) {
        // ---- S^T = K Q^T: the lane ends with keys kg8 + 8 j of heads cq, cq + 1.  t * q_scale is the score (log2 units); the maximum is
        // taken off t, and the difference multiplied, so a score is not rounded at its own size, and the largest comes out as 0 whatever its size
        uint32_t kx[MK][D / 32], ky[MK][D / 32], gx[MK], gy[MK];      // e2m1: codes and group scales of the lane's keys
        if (ELEM <= 0) {
#pragma unroll
          for (int mt = 0; mt < MK; ++mt) {
            const uint32_t rows = ELEM == kUnits ? k_s + mt * C::unit : k_s + mt * 16 * C::row;
            const uint32_t rx = (ELEM == kUnits ? rows + 16 * C::row : k_s + C::codes + mt * 16 * (D / 16)) + kg8 * (D / 16), ry = rx + 8 * (D / 16);
            if (D == 128) {
              const uint4 x = lds16(rows + chunk_at<D, ELEM>(kg8, c)), y = lds16(rows + chunk_at<D, ELEM>(kg8 + 8, c));
              kx[mt][0] = x.x; kx[mt][1] = x.y; kx[mt][D / 32 - 2] = x.z; kx[mt][D / 32 - 1] = x.w;
              ky[mt][0] = y.x; ky[mt][1] = y.y; ky[mt][D / 32 - 2] = y.z; ky[mt][D / 32 - 1] = y.w;
              gx[mt] = lds2(rx + 2 * c);
              gy[mt] = lds2(ry + 2 * c);
            } else {
              const uint2 x = lds8(rows + kg8 * C::row + c * 8), y = lds8(rows + (kg8 + 8) * C::row + c * 8);
              kx[mt][0] = x.x; kx[mt][1] = x.y;
              ky[mt][0] = y.x; ky[mt][1] = y.y;
              gx[mt] = lds1(rx + c) * 0x101u;
              gy[mt] = lds1(ry + c) * 0x101u;
            }
          }
        }
        float2 t[2 * MK];
#pragma unroll
        for (int mt = 0; mt < MK; ++mt) {
          float sc[2][4] = {};                        // two chains: even and odd k-steps
          if (ELEM == 2) {
            const int row = mt * 16 + (lane & 15);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
              uint32_t a[4];
              ldsm4(k_s + chunk_at<D, ELEM>(row, ks * 2 + (lane >> 4)), a);
#pragma unroll
              for (int h = 0; h < QP; ++h) mma_bf16(sc[ks & 1], a, qf[h][ks][0], qf[h][ks][1]);
            }
          } else if (ELEM <= 0) {
            // D / 4 consecutive codes of two keys, a word for two k-steps, and the scales of their groups
            const uint32_t ex = half2_of_e4m3x2(gx[mt]), ey = half2_of_e4m3x2(gy[mt]);
            uint32_t sx[D / 64], sy[D / 64];
            sx[0] = D == 128 ? __byte_perm(ex, 0, 0x1010) : ex;
            sy[0] = D == 128 ? __byte_perm(ey, 0, 0x1010) : ey;
            if (D == 128) {
              sx[D / 64 - 1] = __byte_perm(ex, 0, 0x3232);
              sy[D / 64 - 1] = __byte_perm(ey, 0, 0x3232);
            }
#pragma unroll
            for (int w = 0; w < D / 32; ++w) {
              uint32_t vx[4], vy[4];
              halves_of_e2m1(kx[mt][w], vx);
              halves_of_e2m1(ky[mt][w], vy);
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                vx[i] = mul_half2(vx[i], sx[w / 2]);
                vy[i] = mul_half2(vy[i], sy[w / 2]);
              }
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const uint32_t a[4] = {vx[2 * i], vy[2 * i], vx[2 * i + 1], vy[2 * i + 1]};
#pragma unroll
                for (int h = 0; h < QP; ++h) mma_f16(sc[i & 1], a, qf[h][2 * w + i][0], qf[h][2 * w + i][1]);
              }
            }
          } else {
#pragma unroll
            for (int j = 0; j < KS / 4; ++j) {
              const uint4 x = lds16(k_s + chunk_at<D, ELEM>(mt * 16 + g, c * (KS / 4) + j));
              const uint4 y = lds16(k_s + chunk_at<D, ELEM>(mt * 16 + g + 8, c * (KS / 4) + j));
              const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const uint32_t a[4] = {half2_of_e4m3x2(xs[i]), half2_of_e4m3x2(ys[i]), half2_of_e4m3x2(xs[i] >> 16),
                                       half2_of_e4m3x2(ys[i] >> 16)};
#pragma unroll
                for (int h = 0; h < QP; ++h) mma_f16(sc[i & 1], a, qf[h][4 * j + i][0], qf[h][4 * j + i][1]);
              }
            }
          }
          t[2 * mt] = add2(make_float2(sc[0][0], sc[0][1]), make_float2(sc[1][0], sc[1][1]));
          t[2 * mt + 1] = add2(make_float2(sc[0][2], sc[0][3]), make_float2(sc[1][2], sc[1][3]));
          if (ELEM != 2) {
            t[2 * mt] = mul2(t[2 * mt], q_pre);
            t[2 * mt + 1] = mul2(t[2 * mt + 1], q_pre);
          }
        }
        if (ELEM == 2) {
#pragma unroll
          for (int j = 0; j < 2 * MK; ++j) low = fminf(low, fminf(t[j].x, t[j].y));
        }
        float ev[2 * MK];
        if (ELEM == kUnits) {
#pragma unroll
          for (int j = 0; j < 2 * MK; ++j) {
            const uint32_t at = k_s + (j >> 1) * C::unit + 16 * (D / 2 + D / 16) + (j & 1) * 8 + kg8;
            const float ek = __uint_as_float(lds1(at) << 23);
            t[j] = mul2(t[j], make_float2(ek, ek));
            ev[j] = __uint_as_float(0x4b000000u + lds1(at + C::tile)) - 8388735.f;      // 2^23 + byte, less 2^23 + 127
          }
        } else if (ELEM != 2) {
          // lane l has the scale bytes of row l: K's goes to the exponent field of a float, V's to the low bits
          const int pos = min(key0 + my_row, n - 1);
          const int o = p.block_shift >= 0 ? pos & (p.cache.block_size - 1) : pos % p.cache.block_size;
          const int shift = 8 * (((ELEM <= 0 ? 0 : kvh * p.cache.block_size) + o) & 3);
          const uint32_t ek = (lds4(k_s + 2 * C::tile + lane * 4) >> shift) & 255u;
          const uint32_t both = ek << 23 | ((lds4(k_s + 2 * C::tile + 128 + lane * 4) >> shift) & 255u);
#pragma unroll
          for (int j = 0; j < 2 * MK; ++j) {
            const uint32_t b = __shfl_sync(0xffffffffu, both, 8 * j + kg8);
            const float ek = __uint_as_float(b & 0x7f800000u);
            t[j] = mul2(t[j], make_float2(ek, ek));
            ev[j] = __uint_as_float(0x4b000000u | (b & 255u)) - 8388735.f;      // 2^23 + byte, less 2^23 + 127
          }
        }
        if (key0 + KEYS > n) {
#pragma unroll
          for (int j = 0; j < 2 * MK; ++j)
            if (key0 + 8 * j + kg8 >= n) t[j] = make_float2(-INFINITY, -INFINITY);
        }
        // ---- running maxima, and the exponents of the weights: t off m, and e_v more
        const float2 top = max_of(t);
        float2 x[2 * MK], w[2 * MK];
        auto off_maximum = [&]() {
#pragma unroll
          for (int j = 0; j < 2 * MK; ++j) {
            x[j] = mul2(add2(t[j], m_neg), q_scale);
            if (ELEM != 2) w[j] = add2(x[j], make_float2(ev[j], ev[j]));
          }
        };
        off_maximum();
        float over = fmaxf((top.x - m.x) * q_scale.x, (top.y - m.y) * q_scale.y);      // NaN where both are -inf: no
        if (ELEM != 2) {
          const float2 wtop = max_of(w);
          over = max3(over, wtop.x - mw.x, wtop.y - mw.y);
        }
        if (__any_sync(0xffffffffu, over > kLazy<ELEM>)) {
          float corr[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float &m_i = i ? m.y : m.x, &w_i = i ? mw.y : mw.x;
            const float m_new = fmaxf(m_i, column_max(i ? top.y : top.x));
            const float sub = m_new == -INFINITY ? 0.f : m_new;
            const float down = (m_i - sub) * (i ? q_scale.y : q_scale.x);
            corr[i] = ex2(down);
            (i ? l.y : l.x) *= corr[i];
            m_i = m_new;
            w_i += down;
            (i ? m_neg.y : m_neg.x) = -sub;
          }
          off_maximum();
          if (ELEM != 2) {
            const float2 wtop = max_of(w);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              float &w_i = i ? mw.y : mw.x;
              const float w_new = fmaxf(w_i, column_max(i ? wtop.y : wtop.x));
              const float wsub = w_new == -INFINITY ? 0.f : w_new;
              corr[i] = ex2(w_i - wsub);
              w_i = w_new;
              (i ? w_neg.y : w_neg.x) = kWeightBits - wsub;
            }
          }
#pragma unroll
          for (int mt = 0; mt < MO; ++mt) {
            oc[mt][0] *= corr[0];
            oc[mt][1] *= corr[1];
            oc[mt][2] *= corr[0];
            oc[mt][3] *= corr[1];
          }
        }
        // ---- weights, as B fragments of P^T (head g, two keys to a register)
        uint32_t pf[PP][2 * MK];
#pragma unroll
        for (int j = 0; j < 2 * MK; ++j) {
          const float p0 = ex2(x[j].x), p1 = ex2(x[j].y);
          l = add2(l, make_float2(p0, p1));
          uint32_t parts[PP];
          if (ELEM == 2) {
            split_bf16(p0, p1, parts);
          } else {
            const float2 u = add2(w[j], w_neg);
            split_f16(ex2(u.x), ex2(u.y), parts);
          }
#pragma unroll
          for (int h = 0; h < PP; ++h) pf[h][j] = transpose8(parts[h]);
        }
        if (ELEM == kUnits ? poison != 0 && ((poison >> get) & 1u) : (poison >> get) & 1u) l.x = l.y = __uint_as_float(0x7fc00000u);   // a row outside the pool: the request is NaN
        // the values' codes and scales, on their way through the softmax
        uint32_t vc[MK][4][NT / 8], vg[MK][4];
        if (ELEM <= 0) {
#pragma unroll
          for (int kk = 0; kk < MK; ++kk) {
            const uint32_t rows = ELEM == kUnits ? v_s + kk * C::unit : v_s + kk * 16 * C::row;
            const uint32_t groups = ELEM == kUnits ? rows + 16 * C::row : v_s + C::codes + kk * 16 * (D / 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int row = key_of<ELEM>(cq + (i & 1)) + (i >> 1) * 8;
              if (D == 128) {
                const uint2 x = lds8(rows + chunk_at<D, ELEM>(row, g >> 1) + (g & 1) * 8);
                vc[kk][i][0] = x.x; vc[kk][i][NT / 8 - 1] = x.y;
                vg[kk][i] = lds1(groups + row * (D / 16) + g);
              } else {
                vc[kk][i][0] = lds4(rows + row * C::row + g * 4);
                vg[kk][i] = lds1(groups + row * (D / 16) + (g >> 1));
              }
            }
            if (ELEM == kUnits && key0 + KEYS > n) {      // what stands behind a context may be anything, NaN too: its weights are zero
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (key0 + kk * 16 + key_of<ELEM>(cq + (i & 1)) + (i >> 1) * 8 >= n) vg[kk][i] = 0;
            }
          }
        }
        // ---- O^T += V^T P^T
#pragma unroll
        for (int kk = 0; kk < MK; ++kk) {
          if (ELEM == 2) {
            const int row = kk * 16 + (lane & 7) + (lane >> 4) * 8;
#pragma unroll
            for (int mt = 0; mt < MO; ++mt) {
              uint32_t a[4];
              ldsm4_trans(v_s + chunk_at<D, ELEM>(row, mt * 2 + ((lane >> 3) & 1)), a);
              add_product<sizeof(T) == 4, true>(oc[mt], a, pf, 2 * kk);
            }
          } else if (ELEM <= 0) {
            // As below, NT consecutive codes of four keys and the scale of their group: even and odd dims of two keys to a byte each
            const uint32_t s0 = half2_of_e4m3x2(vg[kk][0] | vg[kk][1] << 8), s1 = half2_of_e4m3x2(vg[kk][2] | vg[kk][3] << 8);
#pragma unroll
            for (int j = 0; j < NT / 8; ++j) {
              constexpr uint32_t kLow = 0x0f0f0f0fu;
              uint32_t even0[4], odd0[4], even1[4], odd1[4];
              halves_of_e2m1((vc[kk][0][j] & kLow) | (vc[kk][1][j] << 4 & ~kLow), even0);
              halves_of_e2m1((vc[kk][0][j] >> 4 & kLow) | (vc[kk][1][j] & ~kLow), odd0);
              halves_of_e2m1((vc[kk][2][j] & kLow) | (vc[kk][3][j] << 4 & ~kLow), even1);
              halves_of_e2m1((vc[kk][2][j] >> 4 & kLow) | (vc[kk][3][j] & ~kLow), odd1);
#pragma unroll
              for (int b = 0; b < 4; ++b) {
                const uint32_t x[4] = {mul_half2(even0[b], s0), mul_half2(odd0[b], s0), mul_half2(even1[b], s1), mul_half2(odd1[b], s1)};
                add_product<sizeof(T) == 4, false>(oc[4 * j + b], x, pf, 2 * kk);
              }
            }
          } else {
            // rows g and g + 8 of tile mt are dims g NT + 2 mt and + 1: the lane reads NT consecutive codes of four keys
            uint32_t v[4][NT / 4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int row = kk * 16 + cq + (i & 1) + (i >> 1) * 8;
              if (NT == 16) {
                const uint4 x = lds16(v_s + chunk_at<D, ELEM>(row, g));
                v[i][0] = x.x; v[i][1] = x.y; v[i][NT / 4 - 2] = x.z; v[i][NT / 4 - 1] = x.w;
              } else {
                const uint2 x = lds8(v_s + chunk_at<D, ELEM>(row, g >> 1) + (g & 1) * 8);
                v[i][0] = x.x; v[i][1] = x.y;
              }
            }
#pragma unroll
            for (int j = 0; j < NT / 4; ++j) {
              // bytes (key, key + 1) of dims 4 j, 4 j + 1 and of 4 j + 2, 4 j + 3
              const uint32_t a0 = __byte_perm(v[0][j], v[1][j], 0x5140), a1 = __byte_perm(v[0][j], v[1][j], 0x7362);
              const uint32_t b0 = __byte_perm(v[2][j], v[3][j], 0x5140), b1 = __byte_perm(v[2][j], v[3][j], 0x7362);
              const uint32_t x[4] = {half2_of_e4m3x2(a0), half2_of_e4m3x2(a0 >> 16), half2_of_e4m3x2(b0), half2_of_e4m3x2(b0 >> 16)};
              const uint32_t y[4] = {half2_of_e4m3x2(a1), half2_of_e4m3x2(a1 >> 16), half2_of_e4m3x2(b1), half2_of_e4m3x2(b1 >> 16)};
              add_product<false, false>(oc[2 * j], x, pf, 2 * kk);
              add_product<false, false>(oc[2 * j + 1], y, pf, 2 * kk);
            }
          }
        }
      }
      if (ELEM == kUnits) poison &= ~(1u << get);      // the slot's next stage says so itself
      get = get + 1 == C::stages ? 0 : get + 1;
      cons.step(p, TILE);
    }
    todo -= steps;
    if (todo > 0) load_query(cons.r);        // on its way while this one is finished

    // A score of -inf is a finite one below fp32's range, which weighs nothing, or comes of an infinity in the key and has to
    // show.  (bf16 pages: e4m3 has no infinities.  Scores of +inf and NaN show by themselves.)
    if (ELEM == 2 && __any_sync(0xffffffffu, low == -INFINITY) &&
        infinite_key<KEYS>(p, req, kvh, (s_tile * KW + kg) * KEYS, TILE, steps, n))
      l.x = l.y = __uint_as_float(0x7fc00000u);

    // ---- the request's share: sums over the lanes of a column, fp16 weights back to 2^(t - m)
    float f[2];
    float ms[2] = {m.x * q_scale.x, m.y * q_scale.y}, ls[2] = {l.x, l.y};
    const float mws[2] = {mw.x, mw.y};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      ls[i] += __shfl_xor_sync(0xffffffffu, ls[i], 4);
      ls[i] += __shfl_xor_sync(0xffffffffu, ls[i], 8);
      ls[i] += __shfl_xor_sync(0xffffffffu, ls[i], 16);
      // a largest score below fp32's range leaves no weight, one beyond it NaN
      ls[i] = ms[i] == -INFINITY ? ls[i] * 0.f : fmaf(ms[i], 0.f, ls[i]);
      f[i] = ELEM != 2 && mws[i] != -INFINITY ? ex2(mws[i] - kWeightBits) : 1.f;
    }
    const bool whole = WIDE || s_tile == 0 && steps == tiles_of(n, TILE);
    const long long rec_slot = s_tile == 0 ? 1 : 0;      // a range can begin and end inside a request: two records
    auto finish = [&]() {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (cq + i >= nh) break;
        const int h = head0 + cq + i;
        if (whole) {
          store_head<D, ELEM>(static_cast<T *>(p.out) + req * p.out_stride + (long long)h * D, oc, i, g, n == 0 ? 0.f : f[i] / ls[i]);
          if (p.lse != nullptr && g == 0)
            p.lse[(long long)req * p.n_q_heads + h] = n == 0 ? -INFINITY : nan_of_inf((ms[i] + log2f(ls[i])) * (1.f / kLog2e));
        } else {
          const long long rec = ((long long)h * p.parts + part) * 2 + rec_slot;
          store_head<D, ELEM>(p.o + rec * D, oc, i, g, f[i]);
          if (g == 0) p.ml[rec] = make_float2(ms[i], ls[i]);
        }
      }
    };
    if (KW == 1) {
      finish();
    } else {
      // the CTA's warps share the head: brought to the common maximum, the others hand theirs to warp 0, lane by lane.
      // (ml_s takes turns: warp 0 may still read it while the others write the next request's.)
      float4 *buf = reinterpret_cast<float4 *>(ba_smem + (WIDE ? 0 : kBaWarps * C::ring));
      if (WIDE) cp_wait_group<0>();
      float2(*ml)[kBaHeads] = ml_s[seg & 1];
      if (g == 0) {
        ml[warp][cq] = make_float2(ms[0], ls[0]);
        ml[warp][cq + 1] = make_float2(ms[1], ls[1]);
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float all = -INFINITY;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) all = fmaxf(all, ml[w][cq + i].x);
        f[i] = ms[i] == -INFINITY ? 0.f : f[i] * ex2(ms[i] - all);
        ls[i] = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
          const float2 x = ml[w][cq + i];
          ls[i] += x.x == -INFINITY ? x.y : x.y * ex2(x.x - all);
        }
        ms[i] = all;
#pragma unroll
        for (int mt = 0; mt < MO; ++mt) {
          oc[mt][i] *= f[i];
          oc[mt][2 + i] *= f[i];
        }
        f[i] = 1.f;
      }
      if (warp > 0) {
#pragma unroll
        for (int mt = 0; mt < MO; ++mt)
          buf[((warp - 1) * MO + mt) * 32 + lane] = make_float4(oc[mt][0], oc[mt][1], oc[mt][2], oc[mt][3]);
      }
      __syncthreads();
      if (warp == 0) {
#pragma unroll
        for (int w = 0; w < WARPS - 1; ++w)
#pragma unroll
          for (int mt = 0; mt < MO; ++mt) {
            const float4 x = buf[(w * MO + mt) * 32 + lane];
            oc[mt][0] += x.x; oc[mt][1] += x.y; oc[mt][2] += x.z; oc[mt][3] += x.w;
          }
        finish();
      }
      ++seg;
    }
  }
  cp_wait_group<0>();
}

// Joins the records of a (request, query head): the parts that hold its tiles follow from the starts.  Its blocks are placed as
// CTAs of the first kernel leave (programmatic launch; two of those for 128 dims fill an SM's registers); everything that kernel wrote is
// read behind the wait, past L1.
// A chain of loads from L2 is all this costs, so a warp has the (m, l) and the outputs of kJoinBatch records in flight at
// once, and where there are few requests (with many records each) four warps share a head.
constexpr int kJoinThreads = 128;
constexpr int kJoinBatch = 10;
__device__ __forceinline__ void load_past_l1(const float *p, float (&v)[4]) {
  const float4 x = __ldcg(reinterpret_cast<const float4 *>(p));
  v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
}
__device__ __forceinline__ void load_past_l1(const float *p, float (&v)[2]) {
  const float2 x = __ldcg(reinterpret_cast<const float2 *>(p));
  v[0] = x.x; v[1] = x.y;
}
template <int D, typename T, int WPH>      // WPH: warps per head
__global__ void __launch_bounds__(kJoinThreads) paged_attention_join_kernel(const __grid_constant__ BaParams p, int tile_keys) {
  constexpr int V = D / 32;                // values of a lane
  constexpr int HEADS = kJoinThreads / 32 / WPH;
  __shared__ float m_s[WPH], l_s[WPH], o_s[WPH][WPH > 1 ? D : 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part_of = warp % WPH;
  const int req = blockIdx.x, h = blockIdx.y * HEADS + warp / WPH;
  long long total = 0, t0 = 0, t1;
  if (WPH > 1) {
    // Few requests: their lengths give the starts as well, before the wait (past L1: these blocks may share an SM with
    // what ran before the lengths were written).
    for (int r0 = 0; r0 < p.n_req; r0 += 32) {
      const int r = r0 + lane;
      const int t = r < p.n_req ? tiles_of(min(max(__ldcg(p.lens + r), 0), p.max_ctx), tile_keys) : 0;
      t0 += __reduce_add_sync(0xffffffffu, r < req ? t : 0);
      total += __reduce_add_sync(0xffffffffu, t);
    }
    t1 = t0 + tiles_of(min(max(__ldcg(p.lens + req), 0), p.max_ctx), tile_keys);
    asm volatile("griddepcontrol.wait;" ::: "memory");
  } else {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    total = __ldcg(p.tile_start + p.n_req);
    t0 = __ldcg(p.tile_start + req);
    t1 = __ldcg(p.tile_start + req + 1);
  }
  if (h >= p.n_q_heads) return;            // WPH > 1: one head per block, so the block leaves together
  const long long ranges = min((long long)p.parts, total);
  int first, last;
  if (total * ranges <= 0xffffffffll) {
    first = (int)((uint32_t)((t0 + 1) * ranges - 1) / (uint32_t)total);
    last = (int)((uint32_t)(t1 * ranges - 1) / (uint32_t)total);
  } else {
    first = (int)(((t0 + 1) * ranges - 1) / total);
    last = (int)((t1 * ranges - 1) / total);
  }
  if (first == last) return;               // one part held it all and wrote the output
  const long long rec0 = (long long)h * p.parts * 2;
  float m = -INFINITY, l = 0.f, acc[V] = {};
  for (int q0 = first + part_of; q0 <= last; q0 += kJoinBatch * WPH) {
    float2 ml[kJoinBatch];
    float v[kJoinBatch][V];
#pragma unroll
    for (int b = 0; b < kJoinBatch; ++b) {
      const int q = q0 + b * WPH;
      if (q <= last) {
        ml[b] = __ldcg(p.ml + rec0 + 2 * q + (q == first));
        load_past_l1(p.o + (rec0 + 2 * q + (q == first)) * D + lane * V, v[b]);
      } else {
        ml[b] = make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int i = 0; i < V; ++i) v[b][i] = 0.f;
      }
    }
    float top = m;
#pragma unroll
    for (int b = 0; b < kJoinBatch; ++b) top = fmaxf(top, ml[b].x);
    const float old = m == -INFINITY ? 0.f : ex2(m - top);
    l *= m == -INFINITY ? 1.f : old;       // without a maximum l is 0, or NaN to keep
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] *= old;
#pragma unroll
    for (int b = 0; b < kJoinBatch; ++b) {
      const float f = ml[b].x == -INFINITY ? 0.f : ex2(ml[b].x - top);
      l += ml[b].x == -INFINITY ? ml[b].y : ml[b].y * f;
#pragma unroll
      for (int i = 0; i < V; ++i) acc[i] += f * v[b][i];
    }
    m = top;
  }
  if (WPH > 1) {
    if (lane == 0) {
      m_s[part_of] = m;
      l_s[part_of] = l;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) o_s[part_of][lane * V + i] = acc[i];
    __syncthreads();
    if (part_of > 0) return;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < WPH; ++w) top = fmaxf(top, m_s[w]);
    l = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.f;
#pragma unroll
    for (int w = 0; w < WPH; ++w) {
      const float f = m_s[w] == -INFINITY ? 0.f : ex2(m_s[w] - top);
      l += m_s[w] == -INFINITY ? l_s[w] : l_s[w] * f;
#pragma unroll
      for (int i = 0; i < V; ++i) acc[i] += f * o_s[w][lane * V + i];
    }
    m = top;
  }
  T *out = static_cast<T *>(p.out) + req * p.out_stride + (long long)h * D + lane * V;
  const float inv = 1.f / l;
#pragma unroll
  for (int i = 0; i < V; ++i) acc[i] = nan_of_inf(acc[i] * inv);
  if (V == 4)
    store4(out, acc[0], acc[1], acc[V - 2], acc[V - 1]);
  else
    store2(out, acc[0], acc[1]);
  if (p.lse != nullptr && lane == 0)
    p.lse[(long long)req * p.n_q_heads + h] = nan_of_inf((m + log2f(l)) * (1.f / kLog2e));
}

// Short contexts are not split: one launch, a CTA per request and KV head or four.  Splitting costs a second kernel and the
// search for the range (3 to 5 us), not splitting leaves the longest request to one CTA.  Measured (8 KV heads of 128, 64
// query heads, uniform lengths; split against whole): 32 of up to 577 13.1 / 9.7 us, of 1,000 15.7 / 13.8; with a warp per KV head 128 of up to
// 400 23.7 / 20.7 and of up to 577 27.0 / 25.9 (fp32 queries: 25.7 / 30.0).
constexpr int kBaNeverSplit = 384;   // the least that this can be
constexpr int kBaWholeWarp = 512;    // with a warp per KV head
// Where every (request, head) has an SM to itself, its CTA has eight warps: contexts last longer whole.  Measured, split / four warps /
// eight, 32 query and 8 KV heads of 128, bf16 queries over bf16 pages, fp32 over bf16, bf16 over e4m3, bf16 over e2m1: one request of 384 tokens
// 7.2 / 8.1 / 7.4, 7.9 / 9.9 / 8.3, 7.5 / 7.7 / 6.7, 7.6 / 7.3 / 6.9 us; of 512 7.2 / 9.2 / 8.1, 7.7 / 11.7 / 9.5, 7.8 / 8.5 / 7.2, 8.2 / 8.5 /
// 7.6; four of 512 9.3 / 9.2 / 8.2, 10.0 / 11.8 / 9.6, 8.3 / 8.5 / 7.3, 8.9 / 8.7 / 7.7, ragged of up to 768 8.0 / 11.5 / 9.6, 8.7 / 15.0 / 11.4,
// 8.1 / 10.2 / 8.6, 8.7 / 10.6 / 9.2; eight of 1,024 12.6 / 14.2 / 11.4, 14.1 / 18.7 / 13.9, 11.5 / 12.6 / 10.2, 13.3 / 13.2 / 11.0; 16 ragged of up to
// 1,024 12.3 / 14.0 / 11.3, 13.9 / 18.7 / 13.9, 12.3 / 12.2 / 9.7, 13.5 / 13.1 / 11.1, of up to 1,536 13.7 / 18.9 / 14.5, 15.4 / 25.4 / 18.0, 12.8 /
// 16.2 / 12.6, 15.2 / 17.2 / 14.0.  Up to 128 tokens four warps are as good (eight of 128 over e4m3 pages, fp32, 5.1 / 5.7).
constexpr int kBaWideCtx = 128;
// Beyond that, e2m1 pages: a CTA works longer on a context of the same bytes, and there is as much to gain from the heads that run beside it.
// Split / whole, 32 requests over 8 heads, all of 1,024, 22.6 / 18.4 us; fp32 queries, 64 over 8 heads of 1,024 29.1 / 31.8.  (Six warps to
// a CTA for up to two heads an SM: 3 to 7 % faster from 768 tokens on, 5 % slower at 256.)
int ba_whole_ctx(int n_req, long long heads, int kw, int elem_bytes, int slots, int sms) {
  if (kw == 1) return kBaWholeWarp;
  if (heads <= sms) return heads >= 64 ? 1024 : heads >= 32 || elem_bytes != 2 ? 512 : kBaNeverSplit;
  if (elem_bytes == KV_ELEM_E2M1) return 4 * heads > 5ll * slots ? 768 : 1024;
  return n_req >= 8 ? 768 : (elem_bytes == 1 ? 512 : kBaNeverSplit);
}
constexpr int kBaShort = 1024;       // ... although up to half of the warps have no head
// Positions and the tiles of 32 requests are counted in 32 bits.
constexpr int kBaMaxCtx = 1 << 26;

struct BaPlan {
  int kw, parts, columns;   // warps per KV head, ranges if contexts are split, CTAs over the KV heads
  bool whole;               // they are not: a CTA per request
  bool wide;                // ... of eight warps
};

BaPlan ba_plan(int n_req, int vheads, int max_ctx, int elem_bytes, int dtype, int sms) {
  BaPlan b;
  // A warp per KV head once the batch has a (request, head) for every other warp of the machine; four warps per head below
  // that.  Measured, a warp / four warps: 128 requests of up to 577 tokens 28.8 / 34.2 us, 256 of up to 500 39.4 / 48.3,
  // 64 of up to 4,608 71.3 / 72.4; 4 of up to 4,608 15.1 / 11.2, one of 18,433 20.8 / 16.2.
  // A warp without a head leaves, and its share of the loads in flight with it.  Where that is less than one warp in eight, it does
  // not matter; where it is half of them or more, heads keep four warps each (700 requests of up to 500 tokens over 1, 2 KV heads, 8
  // bits, a warp / four: 35 / 22, 43 / 37 us; of up to 4,096 157 / 78, 223 / 136).  Between the two it is the contexts: short ones are
  // better off without bringing four warps together (700 of up to 700 over 3, 5, 6 heads 55 / 76, 97 / 122, 96 / 138 us), long ones
  // with every warp at work (of up to 4,096 251 / 210, 493 / 348, 523 / 390), and so are whole ones up to six heads an SM (120 of
  // up to 500 over 5, 6 heads 25.5 / 20.0, 25.3 / 22.8; 300 over 3, 5, 6 heads 26 / 28, 40 / 40, 44 / 45).
  const long long heads = (long long)n_req * vheads;
  const int slots = (vheads + kBaWarps - 1) / kBaWarps * kBaWarps;
  bool single = heads >= 4ll * sms;
  if (8 * vheads < 7 * slots)
    single = 2 * vheads > slots && max_ctx <= kBaShort && heads >= (max_ctx <= kBaWholeWarp ? 6ll : 4ll) * sms;
  b.kw = single ? 1 : kBaWarps;
  const int per_cta = kBaWarps / b.kw;
  b.columns = (vheads + per_cta - 1) / per_cta;
  const int ctas = ba_ctas(elem_bytes == KV_ELEM_E2M1, dtype == KV_DTYPE_BF16);
  b.whole = max_ctx <= ba_whole_ctx(n_req, heads, b.kw, elem_bytes, ctas * sms, sms);
  b.wide = b.whole && b.kw == kBaWarps && heads <= sms && max_ctx > kBaWideCtx;
  // As many ranges as CTAs run at once.  Three to an SM leave a head of few requests more records than the joining kernel's four warps have in flight
  // (e2m1 pages, bf16 queries, 8 heads, three / two: one request of 18,433 tokens 17.7 / 14.1 us, of 60,000 31.8 / 29.2; four of 9,000
  // ragged 15.9 / 15.7, all alike 23.4 / 21.4; eight of 6,000 17.5 / 18.2 and 26.1 / 27.9).
  const int at_once = (heads < 64 && ctas > 2 ? 2 : ctas) * sms;
  // no more parts than 16-key tiles (the shortest there are) could give work to
  const long long tiles = (long long)n_req * ((max_ctx + b.kw * 16 - 1) / (b.kw * 16) + 1);
  long long parts = at_once / b.columns;
  parts = parts < 1 ? 1 : parts;
  b.parts = (int)(parts < tiles ? parts : tiles);
  return b;
}

int ba_passes(int group) { return (group + kBaHeads - 1) / kBaHeads; }

struct BaScratch {
  long long ml, o, bytes;   // byte offsets
};
BaScratch ba_scratch(int n_req, int n_q_heads, int head_dim, int parts) {
  BaScratch s;
  auto up = [](long long v) { return (v + 255) / 256 * 256; };
  const long long recs = (long long)n_q_heads * parts * 2;
  s.ml = up((long long)(n_req + 1) * 8);
  s.o = s.ml + up(recs * 8);
  s.bytes = s.o + up(recs * head_dim * 4);
  return s;
}
// Ranges that the size function counts: those of e2m1 pages and bf16 queries, of which there are the most.  One size for every format; calls
// over the others do with less where their own ranges are fewer.
int ba_scratch_parts(int n_req, int vheads, int max_ctx, int sms) {
  return ba_plan(n_req, vheads, max_ctx, KV_ELEM_E2M1, KV_DTYPE_BF16, sms).parts;
}

template <int D, int ELEM, typename T, int KW>
int ba_launch(const BaParams &p, const BaPlan &b, int device, cudaStream_t st) {
  static bool attr_set[kMaxDevices] = {};
  auto kernel = paged_attention_batched_kernel<D, ELEM, T, KW>;
  if (!attr_set[device]) {
    KV_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, BaCfg<D, ELEM, T>::smem(KW)));
    attr_set[device] = true;
  }
  const dim3 grid(b.whole ? p.n_req : b.parts, b.columns);
  kernel<<<grid, ba_warps(KW) * 32, BaCfg<D, ELEM, T>::smem(KW), st>>>(p);
  KV_COUNT_LAUNCH();
  KV_CUDA(cudaGetLastError());
  if (KW > kBaWarps || b.whole) return KV_OK;
  // Four warps per head up to eight heads an SM, one beyond that.  Measured, the whole call, four / one, 64 heads: one request of
  // 18,433 tokens 16.0 / 21.2 us, 4 of up to 4,608 10.7 / 12.8, 16 23.8 / 24.0, 32 39.8 / 38.1, 128 of up to 577 48.6 / 28.4 (nearly
  // every block has nothing, or two records, to join).
  const int wph = (long long)p.n_req * p.n_q_heads <= 8ll * sm_count(device) ? 4 : 1, heads = kJoinThreads / 32 / wph;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.n_req, (p.n_q_heads + heads - 1) / heads);
  cfg.blockDim = dim3(kJoinThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  KV_CUDA(wph == 4 ? cudaLaunchKernelEx(&cfg, paged_attention_join_kernel<D, T, 4>, p, KW * BaCfg<D, ELEM, T>::keys)
                   : cudaLaunchKernelEx(&cfg, paged_attention_join_kernel<D, T, 1>, p, KW * BaCfg<D, ELEM, T>::keys));
  KV_COUNT_LAUNCH();
  return KV_OK;
}

template <int D, int ELEM, typename T>
int ba_pick(const BaParams &p, const BaPlan &b, int device, cudaStream_t st) {
  if (b.wide) return ba_launch<D, ELEM, T, kBaWide>(p, b, device, st);
  return b.kw == 1 ? ba_launch<D, ELEM, T, 1>(p, b, device, st) : ba_launch<D, ELEM, T, kBaWarps>(p, b, device, st);
}

template <int D, int ELEM>
int ba_type(const BaParams &p, const BaPlan &b, int dtype, int device, cudaStream_t st) {
  return dtype == KV_DTYPE_F32 ? ba_pick<D, ELEM, float>(p, b, device, st) : ba_pick<D, ELEM, bf16>(p, b, device, st);
}

template <int ELEM>
int ba_dim(const BaParams &p, const BaPlan &b, int dtype, int device, cudaStream_t st) {
  return p.cache.head_dim == 128 ? ba_type<128, ELEM>(p, b, dtype, device, st) : ba_type<64, ELEM>(p, b, dtype, device, st);
}

// head_stride: elements between the tables of a request's KV heads, 0 if they share one
int ba_call(const void *q_dev, int64_t q_stride, int dtype, int n_req, int n_q_heads, const kv_cache_desc *cache, int layer,
            const int32_t *block_tables_dev, int64_t table_stride, int64_t head_stride, const int32_t *context_lens_dev, int max_ctx,
            float softmax_scale, void *scratch_dev, int64_t scratch_bytes, void *out_dev, int64_t out_stride, float *lse_out_dev,
            void *stream) {
  if (n_req < 0 || n_q_heads <= 0 || max_ctx <= 0 || (dtype != KV_DTYPE_BF16 && dtype != KV_DTYPE_F32)) return KV_ERR_ARG;
  if (!(softmax_scale > 0.f) || softmax_scale > FLT_MAX / 2.f) return KV_ERR_ARG;      // times log2(e) it stays finite
  if (max_ctx > kBaMaxCtx) return KV_ERR_SHAPE;
  int rc = check_cache_desc(cache, true);
  if (rc != KV_OK) return rc;
  if (layer < 0 || layer >= cache->n_layers || n_q_heads % cache->n_kv_heads != 0 ||
      (cache->head_dim != 64 && cache->head_dim != 128))
    return KV_ERR_SHAPE;
  if (n_req == 0) return KV_OK;
  if (q_dev == nullptr || out_dev == nullptr || block_tables_dev == nullptr || context_lens_dev == nullptr) return KV_ERR_ARG;
  const int size = dtype == KV_DTYPE_BF16 ? 2 : 4;
  const long long width = (long long)n_q_heads * cache->head_dim;
  if (((uintptr_t)q_dev & 15) || ((uintptr_t)out_dev & 15) || q_stride * size % 16 != 0 || out_stride * size % 16 != 0)
    return KV_ERR_ARG;
  if (((uintptr_t)block_tables_dev & 3) || ((uintptr_t)context_lens_dev & 3) || ((uintptr_t)lse_out_dev & 3)) return KV_ERR_ARG;
  if (q_stride < 0 || table_stride < 0 || head_stride < 0 || (n_req > 1 && out_stride < width)) return KV_ERR_ARG;
  if (q_dev == out_dev && n_req > 1 && q_stride != out_stride) return KV_ERR_ARG;      // one request's out would be another's query
  const long long blocks = ((long long)max_ctx + cache->block_size - 1) / cache->block_size;
  if (table_stride < blocks || (head_stride != 0 && head_stride < blocks)) return KV_ERR_TABLE_SHORT;
  const int device = current_device();
  BaParams p;
  p.group = n_q_heads / cache->n_kv_heads;
  p.passes = ba_passes(p.group);
  const long long vheads = (long long)cache->n_kv_heads * p.passes;
  if (vheads > 65535 || n_q_heads > 65535) return KV_ERR_SHAPE;      // second dimension of the grids
  const BaPlan b = ba_plan(n_req, (int)vheads, max_ctx, cache->elem_bytes, dtype, sm_count(device));
  const BaScratch s = ba_scratch(n_req, n_q_heads, cache->head_dim, b.parts);      // this call's own ranges: no more than the size function counts
  if (!b.whole) {
    if (scratch_dev == nullptr || ((uintptr_t)scratch_dev & 15) || scratch_bytes < s.bytes) return KV_ERR_WORKSPACE;
  }
  if (device < 0) return KV_ERR_CUDA;
  p.cache = make_view(cache);
  p.layer = layer;
  p.num_blocks = cache->num_blocks;
  p.block_shift = -1;
  for (int i = 0; i < 31; ++i)
    if ((1 << i) == cache->block_size) p.block_shift = i;
  p.aligned16 = cache->block_size % 16 == 0;
  p.q = q_dev;
  p.out = out_dev;
  p.lse = lse_out_dev;
  p.q_stride = q_stride;
  p.out_stride = out_stride;
  p.table_stride = table_stride;
  p.head_stride = head_stride;
  p.tables = block_tables_dev;
  p.lens = context_lens_dev;
  p.n_req = n_req;
  p.n_q_heads = n_q_heads;
  p.max_ctx = max_ctx;
  p.parts = b.whole ? 0 : b.parts;
  p.scale = fmaxf(softmax_scale * kLog2e, FLT_MIN);
  char *base = static_cast<char *>(scratch_dev);
  p.tile_start = reinterpret_cast<long long *>(base);
  p.ml = reinterpret_cast<float2 *>(base + s.ml);
  p.o = reinterpret_cast<float *>(base + s.o);
  cudaStream_t st = (cudaStream_t)stream;
  switch (format_of(cache->elem_bytes)) {
    case kBf16: return ba_dim<kBf16>(p, b, dtype, device, st);
    case kE4m3: return ba_dim<kE4m3>(p, b, dtype, device, st);
    default: return p.aligned16 ? ba_dim<kUnits>(p, b, dtype, device, st) : ba_dim<kE2m1>(p, b, dtype, device, st);
  }
}

}  // namespace
}  // namespace kvr

extern "C" {

int64_t kv_paged_attention_batched_scratch_bytes(int32_t n_req, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                                 int32_t max_ctx) {
  using namespace kvr;
  if (n_req < 0 || n_q_heads <= 0 || n_kv_heads <= 0 || max_ctx <= 0) return KV_ERR_ARG;
  if (max_ctx > kBaMaxCtx) return KV_ERR_SHAPE;
  if (n_q_heads % n_kv_heads != 0 || (head_dim != 64 && head_dim != 128)) return KV_ERR_SHAPE;
  const int vheads = n_kv_heads * ba_passes(n_q_heads / n_kv_heads);
  // As if contexts were split wherever any batch's are: more requests and longer contexts never need less, so that scratch for
  // the largest batch serves every smaller one.  A warp per KV head makes more ranges than four do: more requests can only
  // change to it, longer contexts also from it.
  if (max_ctx <= kBaNeverSplit || n_req == 0) return 256;
  const int sms = sm_count(current_device());
  int parts = ba_scratch_parts(n_req, vheads, max_ctx, sms);
  if (max_ctx > kBaShort) {
    const int short_parts = ba_scratch_parts(n_req, vheads, kBaShort, sms);
    parts = parts > short_parts ? parts : short_parts;
  }
  return ba_scratch(n_req, n_q_heads, head_dim, parts).bytes;
}

int32_t kv_op_paged_attention_batched(const void *q_dev, int64_t q_stride, int32_t dtype, int32_t n_req,
                                      int32_t n_q_heads, const kv_cache_desc *cache, int32_t layer,
                                      const int32_t *block_tables_dev, int64_t table_stride,
                                      const int32_t *context_lens_dev, int32_t max_ctx, float softmax_scale,
                                      void *scratch_dev, int64_t scratch_bytes, void *out_dev, int64_t out_stride,
                                      float *lse_out_dev, void *stream) {
  return kvr::ba_call(q_dev, q_stride, dtype, n_req, n_q_heads, cache, layer, block_tables_dev, table_stride, 0, context_lens_dev, max_ctx,
                      softmax_scale, scratch_dev, scratch_bytes, out_dev, out_stride, lse_out_dev, stream);
}

int32_t kv_op_paged_attention_selected(const void *q_dev, int64_t q_stride, int32_t dtype, int32_t n_req, int32_t n_q_heads,
                                       const kv_cache_desc *cache, int32_t layer, const int32_t *kept_dev, int64_t kept_stride,
                                       int64_t kept_head_stride, const int32_t *kept_lens_dev, int32_t max_len, float softmax_scale,
                                       void *scratch_dev, int64_t scratch_bytes, void *out_dev, int64_t out_stride,
                                       float *lse_out_dev, void *stream) {
  if (kept_head_stride <= 0) return KV_ERR_ARG;
  return kvr::ba_call(q_dev, q_stride, dtype, n_req, n_q_heads, cache, layer, kept_dev, kept_stride, kept_head_stride, kept_lens_dev, max_len,
                      softmax_scale, scratch_dev, scratch_bytes, out_dev, out_stride, lse_out_dev, stream);
}

}  // extern "C"
