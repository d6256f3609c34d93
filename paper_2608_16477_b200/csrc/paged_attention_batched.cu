// Attention of one new token per request over a paged cache: ragged requests, bf16 or e4m3 pages, split over the
// contexts' length and joined.
//
//   s_n = scale * q . k_n      o = sum_n 2^(t_n - m) v_n / sum_n 2^(t_n - m)      t = s * log2(e), m = max t
//
// Bound by HBM: each cached row is read once for all the query heads of its group (2 flops per byte and head), so what
// matters is to keep enough loads in flight and every SM equally busy, whatever the lengths.
//
// Split.  The contexts of all requests are laid end to end in tiles (every request at least one) and cut into equal
// ranges, one per CTA column, so one long request and a hundred short ones load the machine alike.  A range that holds a
// whole request writes its output; otherwise it leaves a record (m, l, o) and a second, small kernel joins the records
// of a request.  Lengths live on the device, so every CTA finds its own range with a scan over them.
//
// A warp works alone: it copies 16 keys of one KV head (K and V rows, 16 bytes per cp.async, whole rows per instruction)
// into a ring of its own and consumes them stage by stage with no barrier but the warp's, so loads never wait for other
// warps and run on across the end of a request.  Four warps of a CTA take four KV heads (batches: neighbouring heads'
// rows are neighbouring memory), or every fourth stage of one KV head (few requests: four times fewer records; their
// results meet in shared memory).
//
// The products run on mma.sync m16n8k16 with the query heads as rows: a KV group has 8 heads or fewer, and the tile's 16
// rows hold each head twice, the high and the low half of an operand that is split in two: q (rows 0-7: high, 8-15: low)
// against K, p against V.  The two rows are added afterwards, which gives fp32-level accuracy at the price of one pass.
// (A 128-row tcgen05 tile would be fifteen sixteenths padding.)  Groups of more than 8 heads are taken 8 at a time.
//
// e4m3 pages: codes go to fp16 fragments (exact) and the power-of-two scales stay outside: K's multiplies the score,
// V's goes into the weight, w = 2^(t + e_v - M), with its own running maximum M of t + e_v, so that fp16 keeps 22 bits
// of every weight that matters next to the largest CONTRIBUTION, however the rows' scales differ.
#include <float.h>

#include "common.cuh"

namespace kvr {
namespace {

constexpr int kBaWarps = 4;
constexpr int kBaThreads = kBaWarps * 32;
constexpr int kBaKeys = 16;          // keys of a stage
constexpr int kBaHeads = 8;          // query heads of a pass
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kWeightBits = 12.f;  // fp16 weights are scaled to at most 2^12
constexpr int kQueryBits = 12;       // ... and fp16 queries to less than 2^12

template <int D, int ELEM>
struct BaCfg {
  static constexpr int row = D * ELEM;                                   // bytes of a K or V row
  static constexpr int tile = kBaKeys * row;
  static constexpr int stage = 2 * tile + (ELEM == 1 ? 128 : 0);         // K, V, 32 words with the scale bytes
  static constexpr int stages = stage > 6144 ? 3 : (stage > 3072 ? 5 : 8);
  static constexpr int ring = stages * stage;
  static constexpr int merge = kBaWarps * kBaHeads * D * 4;              // the warps' outputs when they share a head
  static constexpr int smem = kBaWarps * ring + merge;
};

struct BaParams {
  CacheView cache;
  int layer, num_blocks, block_shift;
  const void *q;
  void *out;
  float *lse;
  long long q_stride, out_stride, table_stride;
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
__device__ __forceinline__ void cp16(uint32_t dst, const char *src, bool valid) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp4(uint32_t dst, const char *src, bool valid) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(valid ? 4 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait_group() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
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
// two e4m3 codes -> two fp16 (exact)
__device__ __forceinline__ uint32_t half2_of_e4m3(uint32_t two) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)two));
  return h;
}
// x = hi + lo: two bf16 with 16 significant bits together, two fp16 with 22
__device__ __forceinline__ void split_bf16(float x, float y, uint32_t &hi, uint32_t &lo) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
  const float2 f = __bfloat1622float2(h);
  const __nv_bfloat162 l = __floats2bfloat162_rn(x - f.x, y - f.y);
  hi = *reinterpret_cast<const uint32_t *>(&h);
  lo = *reinterpret_cast<const uint32_t *>(&l);
}
__device__ __forceinline__ void split_f16(float x, float y, uint32_t &hi, uint32_t &lo) {
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(hi) : "f"(y), "f"(x));
  float fx, fy;
  asm("{\n\t.reg .b16 l, u;\n\tmov.b32 {l, u}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, u;\n\t}"
      : "=f"(fx), "=f"(fy) : "r"(hi));
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(lo) : "f"(y - fy), "f"(x - fx));
}
__device__ __forceinline__ float quad_max(float v) {
  v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 1));
  return fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 2));
}

// Byte offset of 16-byte chunk c of row r in a tile: chunks are permuted inside 128-byte lines so that the fragment
// loads of eight neighbouring lanes fall into different banks.
template <int D, int ELEM>
__device__ __forceinline__ uint32_t chunk_at(int r, int c) {
  if (ELEM == 1 && D == 64) return (uint32_t)((r >> 1) * 128 + ((((r & 1) * 4 + c) ^ (r & 6)) * 16));
  if (ELEM == 1) return (uint32_t)(r * 128 + ((c ^ (r & 7)) * 16));
  return (uint32_t)(r * (D * 2) + ((c & ~7) | ((c ^ r) & 7)) * 16);
}

__device__ __forceinline__ int clamped_len(const BaParams &p, int r) {
  return min(max(__ldg(p.lens + r), 0), p.max_ctx);
}

// Where a warp stands in the sequence of tiles of its range.
struct Cursor {
  int r, tile, n_tiles, n, n_next;
  __device__ __forceinline__ void open(const BaParams &p, int req, int tile_keys) {
    r = req;
    n = r < p.n_req ? clamped_len(p, r) : 0;
    n_next = r + 1 < p.n_req ? clamped_len(p, r + 1) : 0;
    n_tiles = max(1, (n + tile_keys - 1) / tile_keys);
    tile = 0;
  }
  __device__ __forceinline__ void step(const BaParams &p, int tile_keys) {
    if (++tile < n_tiles) return;
    ++r;
    n = n_next;
    n_next = r + 1 < p.n_req ? clamped_len(p, r + 1) : 0;      // loaded a request ahead
    n_tiles = max(1, (n + tile_keys - 1) / tile_keys);
    tile = 0;
  }
};

template <int D, int ELEM, typename T, int KW>      // KW: warps that share a KV head
__global__ void __launch_bounds__(kBaThreads, 2) paged_attention_batched_kernel(const __grid_constant__ BaParams p) {
  typedef BaCfg<D, ELEM> C;
  constexpr int KS = D / 16;                 // k-steps of S = Q K^T
  constexpr int NT = D / 8;                  // n-tiles of O = P V
  constexpr int CH = C::row / 16;            // 16-byte chunks of a row
  constexpr int RPI = 32 / CH;               // rows per copy instruction
  constexpr int TILE = KW * kBaKeys;         // keys of a tile of the split
  extern __shared__ __align__(128) unsigned char ba_smem[];
  __shared__ float2 ml_s[2][kBaWarps][kBaHeads];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int kg = warp % KW;                                        // which of the tile's stages
  const int vh = blockIdx.y * (kBaWarps / KW) + warp / KW;         // (KV head, pass over its query heads)
  if (KW == 1 && vh >= p.cache.n_kv_heads * p.passes) return;
  const int kvh = vh / p.passes, pass = vh % p.passes;
  const int head0 = kvh * p.group + pass * kBaHeads, nh = min(kBaHeads, p.group - pass * kBaHeads);
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(ba_smem) + warp * C::ring;

  // ---- this CTA's range of tiles
  Cursor cons;
  long long todo;
  const int part = blockIdx.x;
  if (p.parts == 0) {
    cons.open(p, blockIdx.x, TILE);
    todo = cons.n_tiles;
  } else {
    long long total = 0;
    for (int r0 = 0; r0 < p.n_req; r0 += 32) {
      const int r = r0 + lane;
      int t = r < p.n_req ? max(1, (clamped_len(p, r) + TILE - 1) / TILE) : 0;
      if (blockIdx.x == 0 && blockIdx.y == 0 && warp == 0) {      // the joining kernel wants the starts
        int inc = t;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int up = __shfl_up_sync(0xffffffffu, inc, o);
          if (lane >= o) inc += up;
        }
        if (r < p.n_req) p.tile_start[r + 1] = total + inc;
        if (r == 0) p.tile_start[0] = 0;
      }
      total += __reduce_add_sync(0xffffffffu, t);
    }
    // no more ranges than tiles: every range that is left holds one (the joining kernel counts on it)
    const long long ranges = min((long long)p.parts, total);
    if (part >= ranges) return;
    const long long first_tile = part * total / ranges;
    todo = (part + 1) * total / ranges - first_tile;
    long long before = 0;
    int at = 0;
    for (int r0 = 0; r0 < p.n_req; r0 += 32) {
      const int r = r0 + lane;
      const int t = r < p.n_req ? max(1, (clamped_len(p, r) + TILE - 1) / TILE) : 0;
      int inc = t;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += up;
      }
      const int sum = __shfl_sync(0xffffffffu, inc, 31);
      if (first_tile < before + sum) {
        const unsigned hit = __ballot_sync(0xffffffffu, first_tile < before + inc);
        const int l = __ffs(hit) - 1;
        at = r0 + l;
        before += __shfl_sync(0xffffffffu, inc - t, l);
        break;
      }
      before += sum;
    }
    cons.open(p, at, TILE);
    cons.tile = (int)(first_tile - before);
  }

  // ---- loads.  Lane l looks up the page of row l % 16 of the stage to come, one stage ahead of its copies.
  Cursor prod = cons;
  long long to_load = todo;
  int blk = -1, off = 0;                     // row of the stage that `prod` stands at: block (-1: none), slot
  const int my_row = lane & 15;
  auto look_up = [&]() {
    const int pos = (prod.tile * KW + kg) * kBaKeys + my_row;
    blk = -1;
    if (to_load > 0 && pos < prod.n) {
      const int b = p.block_shift >= 0 ? pos >> p.block_shift : pos / p.cache.block_size;
      off = pos - b * p.cache.block_size;
      blk = __ldg(p.tables + prod.r * p.table_stride + b);
      if ((unsigned)blk >= (unsigned)p.num_blocks) blk = -2;      // not in the pool: never followed
    }
  };
  unsigned poison = 0;                       // bit s: the stage in ring slot s has a row outside the pool
  int put = 0;                               // ring slot to fill next
  auto issue = [&]() {
    const bool any = __any_sync(0xffffffffu, blk != -1);
    const bool bad = __any_sync(0xffffffffu, blk == -2);
    poison = (poison & ~(1u << put)) | ((unsigned)bad << put);
    if (any) {
      const uint32_t k_s = ring + put * C::stage, v_s = k_s + C::tile;
      const int sub = lane / CH, c = lane % CH;
#pragma unroll
      for (int i = 0; i < kBaKeys / RPI; ++i) {
        const int row = i * RPI + sub;
        const int b = __shfl_sync(0xffffffffu, blk, row), o = __shfl_sync(0xffffffffu, off, row);
        const bool ok = b >= 0;
        const char *src = p.cache.page(p.layer, 0, ok ? b : 0) +
                          ((long long)(ok ? o : 0) * p.cache.n_kv_heads + kvh) * C::row + c * 16;
        const uint32_t dst = chunk_at<D, ELEM>(row, c);
        cp16(k_s + dst, src, ok);                                 // rows that are not there are zeros
        cp16(v_s + dst, src + p.cache.kv_stride, ok);
      }
      if (ELEM == 1) {   // the word that holds the scale byte of row l % 16 of K (lanes 0-15) or V
        const bool ok = blk >= 0;
        const int at = kvh * p.cache.block_size + (ok ? off : 0);
        const char *src = p.cache.page(p.layer, lane >> 4, ok ? blk : 0) + p.cache.value_bytes() + (at & ~3);
        cp4(k_s + 2 * C::tile + lane * 4, src, ok);
      }
    }
    cp_commit();
    put = put + 1 == C::stages ? 0 : put + 1;
    if (to_load > 0) {
      --to_load;
      prod.step(p, TILE);
    }
    look_up();
  };
  look_up();
#pragma unroll
  for (int i = 0; i < C::stages - 1; ++i) issue();

  // ---- per request of the range
  const int r0 = lane >> 2, cq = (lane & 3) * 2;      // query head (row) and first column of the lane's fragments
  int get = 0, seg = 0;
  while (todo > 0) {
    const int req = cons.r, n = cons.n, s_tile = cons.tile;
    const int steps = (int)min((long long)(cons.n_tiles - s_tile), todo);
    // Q fragments: row r0 high parts, row r0 + 8 low parts of head head0 + r0
    uint32_t qf[KS][4];
    float q_scale = 1.f;
    {
      const T *q = static_cast<const T *>(p.q) + req * p.q_stride + (long long)(head0 + min(r0, nh - 1)) * D;
      const float on = r0 < nh ? 1.f : 0.f;
      if (ELEM == 2) {
        const float f = on * p.scale;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const int d0 = ks * 16 + cq;
          split_bf16((float)q[d0] * f, (float)q[d0 + 1] * f, qf[ks][0], qf[ks][1]);
          split_bf16((float)q[d0 + 8] * f, (float)q[d0 + 9] * f, qf[ks][2], qf[ks][3]);
        }
      } else {
        // the lane's dims: 4 KS consecutive ones, so that a key's codes are read as 16-byte vectors
        const T *ql = q + (lane & 3) * (4 * KS);
        float x[4 * KS], most = 0.f;
#pragma unroll
        for (int i = 0; i < 4 * KS; ++i) {
          x[i] = (float)ql[i] * on;
          most = fmaxf(most, fabsf(x[i]));
        }
        most = quad_max(most);
        const int e = min(max((int)(__float_as_uint(most) >> 23) - 126, -100), 127);       // most < 2^e
        const float up = __uint_as_float((uint32_t)(127 + kQueryBits - e) << 23);
        q_scale = p.scale * __uint_as_float((uint32_t)(127 - kQueryBits + e) << 23);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          split_f16(x[4 * ks] * up, x[4 * ks + 1] * up, qf[ks][0], qf[ks][1]);
          split_f16(x[4 * ks + 2] * up, x[4 * ks + 3] * up, qf[ks][2], qf[ks][3]);
        }
      }
    }
    float m = -INFINITY, mw = -INFINITY, l = 0.f;     // running maxima of t and of t + e_v (ELEM 1), the lane's sum
    float oc[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 4; ++i) oc[nt][i] = 0.f;

    for (int s = 0; s < steps; ++s) {
      cp_wait_group<C::stages - 2>();
      __syncwarp();
      issue();                                        // into the slot that the previous step has left
      const uint32_t k_s = ring + get * C::stage, v_s = k_s + C::tile;
      const int key0 = (cons.tile * KW + kg) * kBaKeys;
      if (key0 < n) {
        // ---- S = Q K^T: two n-tiles of 8 keys; the lane ends with keys cq, cq + 1, cq + 8, cq + 9 of head r0
        float sc[2][4];
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
#pragma unroll
          for (int i = 0; i < 4; ++i) sc[nt][i] = 0.f;
          if (ELEM == 2) {
            const int row = nt * 8 + (lane & 7);
#pragma unroll
            for (int ks = 0; ks < KS; ks += 2) {
              uint32_t b[4];
              ldsm4(k_s + chunk_at<D, ELEM>(row, ks * 2 + (lane >> 3)), b);
              mma_bf16(sc[nt], qf[ks], b[0], b[1]);
              mma_bf16(sc[nt], qf[ks + 1], b[2], b[3]);
            }
          } else {
            const int row = nt * 8 + r0;
#pragma unroll
            for (int c = 0; c < KS / 4; ++c) {
              const uint4 v = lds16(k_s + chunk_at<D, ELEM>(row, (lane & 3) * (KS / 4) + c));
              const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
              for (int i = 0; i < 4; ++i) mma_f16(sc[nt], qf[4 * c + i], half2_of_e4m3(w[i]), half2_of_e4m3(w[i] >> 16));
            }
          }
        }
        float t[4] = {sc[0][0] + sc[0][2], sc[0][1] + sc[0][3], sc[1][0] + sc[1][2], sc[1][1] + sc[1][3]};
        float ev[4];
        if (ELEM == 1) {
          // lane l has the scale byte of K row l (l < 16) or V row l - 16
          const int pos = min(key0 + my_row, n - 1);
          const int o = p.block_shift >= 0 ? pos & (p.cache.block_size - 1) : pos % p.cache.block_size;
          const int byte = (kvh * p.cache.block_size + o) & 3;
          const int e = (int)((lds4(k_s + 2 * C::tile + lane * 4) >> (8 * byte)) & 255u);
          const int both = e | (__shfl_down_sync(0xffffffffu, e, 16) << 8);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int b = __shfl_sync(0xffffffffu, both, cq + (i & 1) + (i >> 1) * 8);
            t[i] = (t[i] * q_scale) * __uint_as_float((uint32_t)(b & 255) << 23);
            ev[i] = (float)((b >> 8) - 127);
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (key0 + cq + (i & 1) + (i >> 1) * 8 >= n) t[i] = -INFINITY;
        const float m_new = fmaxf(m, quad_max(fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]))));
        const float m_use = m_new == -INFINITY ? 0.f : m_new;      // no score yet: nothing to subtract
        float w[4], corr;
        if (ELEM == 2) {
          corr = ex2(m - m_use);
          l *= corr;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            w[i] = ex2(t[i] - m_use);
            l += w[i];
          }
        } else {
          l *= ex2(m - m_use);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            l += ex2(t[i] - m_use);
            t[i] += ev[i];
          }
          const float w_new = fmaxf(mw, quad_max(fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]))));
          const float w_use = w_new == -INFINITY ? 0.f : w_new;
          corr = ex2(mw - w_use);
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = ex2(t[i] - w_use + kWeightBits);
          mw = w_new;
        }
        m = m_new;
        if (__any_sync(0xffffffffu, corr != 1.f)) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) oc[nt][i] *= corr;
        }
        if ((poison >> get) & 1u) l = __uint_as_float(0x7fc00000u);      // a row outside the pool: the request is NaN
        // ---- O += P V: the high parts are row r0, the low parts row r0 + 8
        uint32_t pf[4];
        if (ELEM == 2) {
          split_bf16(w[0], w[1], pf[0], pf[1]);
          split_bf16(w[2], w[3], pf[2], pf[3]);
          const int row = ((lane >> 3) & 1) * 8 + (lane & 7);
#pragma unroll
          for (int nt = 0; nt < NT; nt += 2) {
            uint32_t b[4];
            ldsm4_trans(v_s + chunk_at<D, ELEM>(row, nt + (lane >> 4)), b);
            mma_bf16(oc[nt], pf, b[0], b[1]);
            mma_bf16(oc[nt + 1], pf, b[2], b[3]);
          }
        } else {
          split_f16(w[0], w[1], pf[0], pf[1]);
          split_f16(w[2], w[3], pf[2], pf[3]);
          // column r0 of n-tile nt is dim r0 * NT + nt: the lane reads NT consecutive codes of its four keys
          uint32_t v[4][NT / 4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int row = cq + (i & 1) + (i >> 1) * 8;
            if (NT == 16) {
              const uint4 x = lds16(v_s + chunk_at<D, ELEM>(row, r0));
              v[i][0] = x.x; v[i][1] = x.y; v[i][NT / 4 - 2] = x.z; v[i][NT / 4 - 1] = x.w;
            } else {
              const uint2 x = lds8(v_s + chunk_at<D, ELEM>(row, r0 >> 1) + (r0 & 1) * 8);
              v[i][0] = x.x; v[i][1] = x.y;
            }
          }
#pragma unroll
          for (int j = 0; j < NT / 4; ++j) {
            const uint32_t a0 = __byte_perm(v[0][j], v[1][j], 0x5140), a1 = __byte_perm(v[0][j], v[1][j], 0x7362);
            const uint32_t b0 = __byte_perm(v[2][j], v[3][j], 0x5140), b1 = __byte_perm(v[2][j], v[3][j], 0x7362);
            mma_f16(oc[4 * j], pf, half2_of_e4m3(a0), half2_of_e4m3(b0));
            mma_f16(oc[4 * j + 1], pf, half2_of_e4m3(a0 >> 16), half2_of_e4m3(b0 >> 16));
            mma_f16(oc[4 * j + 2], pf, half2_of_e4m3(a1), half2_of_e4m3(b1));
            mma_f16(oc[4 * j + 3], pf, half2_of_e4m3(a1 >> 16), half2_of_e4m3(b1 >> 16));
          }
        }
      }
      get = get + 1 == C::stages ? 0 : get + 1;
      cons.step(p, TILE);
    }
    todo -= steps;

    // ---- the request's share: row sums over the quad, high and low rows together, fp16 weights back to 2^(t - m)
    l += __shfl_xor_sync(0xffffffffu, l, 1);
    l += __shfl_xor_sync(0xffffffffu, l, 2);
    const float back = ELEM == 1 && mw != -INFINITY ? ex2(mw - m - kWeightBits) : 1.f;
    float ov[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      ov[nt][0] = (oc[nt][0] + oc[nt][2]) * back;
      ov[nt][1] = (oc[nt][1] + oc[nt][3]) * back;
    }
    const bool whole = s_tile == 0 && steps == max(1, (n + TILE - 1) / TILE);
    const long long rec_slot = s_tile == 0 ? 1 : 0;      // a range can begin and end inside a request: two records

    if (KW == 1) {
      if (r0 < nh) {
        const int h = head0 + r0;
        float *rec_o = nullptr;
        T *out = nullptr;
        float inv = 1.f;
        if (whole) {
          out = static_cast<T *>(p.out) + req * p.out_stride + (long long)h * D;
          inv = n == 0 ? 0.f : 1.f / l;
          if (p.lse != nullptr && (lane & 3) == 0)
            p.lse[(long long)req * p.n_q_heads + h] = n == 0 ? -INFINITY : (m + log2f(l)) * (1.f / kLog2e);
        } else {
          const long long rec = ((long long)h * p.parts + part) * 2 + rec_slot;
          rec_o = p.o + rec * D;
          if ((lane & 3) == 0) p.ml[rec] = make_float2(m, l);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int d = ELEM == 2 ? nt * 8 + cq + i : (cq + i) * NT + nt;
            if (whole)
              out[d] = (T)(ov[nt][i] * inv);
            else
              rec_o[d] = ov[nt][i];
          }
        }
      }
    } else {
      // the CTA's four warps share the head: common maximum, outputs added in shared memory
      float *buf = reinterpret_cast<float *>(ba_smem + kBaWarps * C::ring);
      const int par = seg & 1;
      if ((lane & 3) == 0) ml_s[par][warp][r0] = make_float2(m, l);
      __syncthreads();
      float all = -INFINITY;
#pragma unroll
      for (int w = 0; w < kBaWarps; ++w) all = fmaxf(all, ml_s[par][w][r0].x);
      const float f = m == -INFINITY ? 0.f : ex2(m - all);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int d = ELEM == 2 ? nt * 8 + cq + i : (cq + i) * NT + nt;
          buf[(warp * kBaHeads + r0) * D + d] = m == -INFINITY && ov[nt][i] == 0.f ? 0.f : ov[nt][i] * f;
        }
      __syncthreads();
      for (int e = threadIdx.x; e < nh * D; e += kBaThreads) {
        const int row = e / D, d = e % D, h = head0 + row;
        float o = 0.f, mm = -INFINITY, ll = 0.f;
#pragma unroll
        for (int w = 0; w < kBaWarps; ++w) mm = fmaxf(mm, ml_s[par][w][row].x);
#pragma unroll
        for (int w = 0; w < kBaWarps; ++w) {
          const float2 x = ml_s[par][w][row];
          o += buf[(w * kBaHeads + row) * D + d];
          ll += x.x == -INFINITY ? x.y : x.y * ex2(x.x - mm);
        }
        if (whole) {
          T *out = static_cast<T *>(p.out) + req * p.out_stride + (long long)h * D;
          out[d] = (T)(n == 0 ? 0.f : o / ll);
          if (p.lse != nullptr && d == 0)
            p.lse[(long long)req * p.n_q_heads + h] = n == 0 ? -INFINITY : (mm + log2f(ll)) * (1.f / kLog2e);
        } else {
          const long long rec = ((long long)h * p.parts + part) * 2 + rec_slot;
          p.o[rec * D + d] = o;
          if (d == 0) p.ml[rec] = make_float2(mm, ll);
        }
      }
      ++seg;
    }
  }
  cp_wait_group<0>();
}

// Joins the records of one (request, query head): the parts that hold its tiles follow from the starts.
template <int D, typename T>
__global__ void __launch_bounds__(D) paged_attention_join_kernel(const __grid_constant__ BaParams p) {
  const int req = blockIdx.x, h = blockIdx.y, d = threadIdx.x;
  const long long total = __ldcg(p.tile_start + p.n_req);
  const long long t0 = __ldcg(p.tile_start + req), t1 = __ldcg(p.tile_start + req + 1);
  const long long ranges = min((long long)p.parts, total);
  const int first = (int)(((t0 + 1) * ranges - 1) / total), last = (int)((t1 * ranges - 1) / total);
  if (first == last) return;                       // one part held it all and wrote the output
  float m = -INFINITY;
  for (int q = first; q <= last; ++q) m = fmaxf(m, __ldcg(p.ml + ((long long)h * p.parts + q) * 2 + (q == first)).x);
  float l = 0.f, o = 0.f;
  for (int q = first; q <= last; ++q) {
    const long long rec = ((long long)h * p.parts + q) * 2 + (q == first);
    const float2 x = __ldcg(p.ml + rec);
    const float f = x.x == -INFINITY ? 0.f : ex2(x.x - m);
    l += x.x == -INFINITY ? x.y : x.y * f;
    o += f * __ldcg(p.o + rec * D + d);
  }
  static_cast<T *>(p.out)[req * p.out_stride + (long long)h * D + d] = (T)(o / l);
  if (p.lse != nullptr && d == 0) p.lse[(long long)req * p.n_q_heads + h] = (m + log2f(l)) * (1.f / kLog2e);
}

// Contexts of at most this many tokens are not split: one launch, a CTA per (request, KV head).
constexpr int kBaWholeCtx = 512;
// Positions and the tiles of 32 requests are counted in 32 bits.
constexpr int kBaMaxCtx = 1 << 26;

struct BaPlan {
  int kw, parts, columns;   // warps per KV head, ranges (0: a CTA per request), CTAs over the KV heads
};

BaPlan ba_plan(int n_req, int vheads, int max_ctx, int sms) {
  BaPlan b;
  // A warp per KV head once the batch has a tile for every warp of the machine; four warps per head below that.
  b.kw = (long long)n_req * vheads >= 4ll * sms ? 1 : kBaWarps;
  const int per_cta = kBaWarps / b.kw;
  b.columns = (vheads + per_cta - 1) / per_cta;
  if (max_ctx <= kBaWholeCtx) {
    b.parts = 0;
    return b;
  }
  const long long tiles = (long long)n_req * ((max_ctx + b.kw * kBaKeys - 1) / (b.kw * kBaKeys));
  long long parts = 2ll * sms / b.columns;         // two CTAs per SM
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

template <int D, int ELEM, typename T, int KW>
int ba_launch(const BaParams &p, const BaPlan &b, int device, cudaStream_t st) {
  static bool attr_set[kMaxDevices] = {};
  auto kernel = paged_attention_batched_kernel<D, ELEM, T, KW>;
  if (!attr_set[device]) {
    KV_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, BaCfg<D, ELEM>::smem));
    attr_set[device] = true;
  }
  const dim3 grid(b.parts == 0 ? p.n_req : b.parts, b.columns);
  kernel<<<grid, kBaThreads, BaCfg<D, ELEM>::smem, st>>>(p);
  KV_COUNT_LAUNCH();
  KV_CUDA(cudaGetLastError());
  if (b.parts == 0) return KV_OK;
  paged_attention_join_kernel<D, T><<<dim3(p.n_req, p.n_q_heads), D, 0, st>>>(p);
  KV_COUNT_LAUNCH();
  KV_CUDA(cudaGetLastError());
  return KV_OK;
}

template <int D, int ELEM, typename T>
int ba_pick(const BaParams &p, const BaPlan &b, int device, cudaStream_t st) {
  return b.kw == 1 ? ba_launch<D, ELEM, T, 1>(p, b, device, st) : ba_launch<D, ELEM, T, kBaWarps>(p, b, device, st);
}

template <int D, int ELEM>
int ba_type(const BaParams &p, const BaPlan &b, int dtype, int device, cudaStream_t st) {
  return dtype == KV_DTYPE_F32 ? ba_pick<D, ELEM, float>(p, b, device, st) : ba_pick<D, ELEM, bf16>(p, b, device, st);
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
  const BaPlan b = ba_plan(n_req > 0 ? n_req : 1, vheads, max_ctx, sm_count(current_device()));
  return b.parts == 0 ? 256 : ba_scratch(n_req, n_q_heads, head_dim, b.parts).bytes;
}

int32_t kv_op_paged_attention_batched(const void *q_dev, int64_t q_stride, int32_t dtype, int32_t n_req,
                                      int32_t n_q_heads, const kv_cache_desc *cache, int32_t layer,
                                      const int32_t *block_tables_dev, int64_t table_stride,
                                      const int32_t *context_lens_dev, int32_t max_ctx, float softmax_scale,
                                      void *scratch_dev, int64_t scratch_bytes, void *out_dev, int64_t out_stride,
                                      float *lse_out_dev, void *stream) {
  using namespace kvr;
  if (n_req < 0 || n_q_heads <= 0 || max_ctx <= 0 || (dtype != KV_DTYPE_BF16 && dtype != KV_DTYPE_F32)) return KV_ERR_ARG;
  if (!(softmax_scale > 0.f) || softmax_scale > FLT_MAX) return KV_ERR_ARG;
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
  if (q_stride < 0 || table_stride < 0 || (n_req > 1 && out_stride < width)) return KV_ERR_ARG;
  const long long blocks = ((long long)max_ctx + cache->block_size - 1) / cache->block_size;
  if (table_stride < blocks) return KV_ERR_TABLE_SHORT;
  const int device = current_device();
  BaParams p;
  p.group = n_q_heads / cache->n_kv_heads;
  p.passes = ba_passes(p.group);
  const long long vheads = (long long)cache->n_kv_heads * p.passes;
  if (vheads > 65535 || n_q_heads > 65535) return KV_ERR_SHAPE;      // second dimension of the grids
  const BaPlan b = ba_plan(n_req, (int)vheads, max_ctx, sm_count(device));
  const BaScratch s = ba_scratch(n_req, n_q_heads, cache->head_dim, b.parts);
  if (b.parts > 0) {
    if (scratch_dev == nullptr || ((uintptr_t)scratch_dev & 15) || scratch_bytes < s.bytes) return KV_ERR_WORKSPACE;
  }
  if (device < 0) return KV_ERR_CUDA;
  p.cache = make_view(cache);
  p.layer = layer;
  p.num_blocks = cache->num_blocks;
  p.block_shift = -1;
  for (int i = 0; i < 31; ++i)
    if ((1 << i) == cache->block_size) p.block_shift = i;
  p.q = q_dev;
  p.out = out_dev;
  p.lse = lse_out_dev;
  p.q_stride = q_stride;
  p.out_stride = out_stride;
  p.table_stride = table_stride;
  p.tables = block_tables_dev;
  p.lens = context_lens_dev;
  p.n_req = n_req;
  p.n_q_heads = n_q_heads;
  p.max_ctx = max_ctx;
  p.parts = b.parts;
  p.scale = softmax_scale * kLog2e;
  char *base = static_cast<char *>(scratch_dev);
  p.tile_start = reinterpret_cast<long long *>(base);
  p.ml = reinterpret_cast<float2 *>(base + s.ml);
  p.o = reinterpret_cast<float *>(base + s.o);
  cudaStream_t st = (cudaStream_t)stream;
  if (cache->head_dim == 128)
    return cache->elem_bytes == 2 ? ba_type<128, 2>(p, b, dtype, device, st) : ba_type<128, 1>(p, b, dtype, device, st);
  return cache->elem_bytes == 2 ? ba_type<64, 2>(p, b, dtype, device, st) : ba_type<64, 1>(p, b, dtype, device, st);
}

}  // extern "C"
