// Blocks of a paged cache that are worth attending to: what each block's keys span, and the choice of the blocks whose span
// promises the largest scores.
//
// Bounds, per (block, KV head): for every dim the largest key value rounded up and the smallest rounded down, 8-bit whole numbers in
// units of one power of two.  No key of the block has q . k above  sum_d max(q_d top_d, q_d low_d).
//
// Score of a block for a KV head: that bound summed over the group's query heads, which is u+ . top + u- . low with u+ (u-) the
// sums of the positive (negative) parts of the heads' queries.  u is taken in 15 bits and a sign, so the score is a whole
// number (at most 256 * 127 * 32767 < 2^31) times a power of two: it does not depend on the order of any sum, so neither does the
// choice, and equal scores go to the lowest block.
//
// Measured in a graph, 8 KV heads of 128 (floor: the bytes at a copy's rate).  Bounds of 4,096 blocks of 16: bf16 pages 25 us (21.7), e4m3
// 26.1 (11.6), e2m1 27.2 (7.1: issue slots 78 %, ALU pipe 71 %); of 64 blocks 2.7.  Selection, 64 query heads: one request of 1,153 blocks 7.8 us (0.4), 16 of up to 512 9.5 (1.4), 32
// of up to 1,153 15.4 (4.8), of which finding the score of the last rank and writing the list take 3 us.
#include <cooperative_groups.h>

#include "cache_format.cuh"

namespace kvr {
namespace {

constexpr int kInfinite = 255;          // scale byte of a block that no bound covers: always chosen
constexpr int kMinBound = -60, kMaxBound = 60;      // exponents of a bound's unit
constexpr int kSelMaxCtx = 1 << 26;

// ---------------------------------------------------------------- bounds
struct BoundsParams {
  RowLayout layout;
  int block_size, n_kv_heads, num_blocks, n;
  const int *blocks, *counts;
  int8_t *codes;        // [num_blocks][n_kv_heads][2][D]
  uint8_t *scales;      // [num_blocks][n_kv_heads]
};

constexpr int kBoundThreads = 256;

__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {      // NaN if one is
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t min_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// A warp takes a (block, KV head), a lane eight dims of every second key (D = 64: fourth), with the loads of 16 (32) keys in flight.
// Bound by HBM over bf16 pages, whose keys are compared two at a time as they are, and by instructions over the others, whose values bf16
// holds exactly.
template <int D, int FMT>
__global__ void __launch_bounds__(kBoundThreads) block_bounds_kernel(const __grid_constant__ BoundsParams p) {
  constexpr int LANES = D / 8, ROWS = 32 / LANES, AHEAD = 8;      // lanes of a key; keys of a load, loads in flight
  const int lane = threadIdx.x & 31, sub = lane % LANES, mine = lane / LANES;
  const long long item = blockIdx.x * (long long)(kBoundThreads / 32) + (threadIdx.x >> 5);
  const int heads = p.n_kv_heads;
  const long long i = item / heads;
  const int head = (int)(item - i * heads);
  if (i >= p.n) return;
  const int block = __ldg(p.blocks + i), count = min(__ldg(p.counts + i), p.block_size);
  if ((unsigned)block >= (unsigned)p.num_blocks || count <= 0) return;
  const Pieces<D, FMT> at(p.layout, 0, head, sub * 8);
  const long long from = block * p.layout.block_stride;
  const char *keys = at.values + from;
  const uint8_t *groups = reinterpret_cast<const uint8_t *>(at.groups + from), *scale = reinterpret_cast<const uint8_t *>(at.scale + from);
  uint32_t top2[4], low2[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    top2[j] = 0xff80ff80u;      // -inf, -inf
    low2[j] = 0x7f807f80u;
  }
  const long long step = ROWS * p.layout.slot_stride;
  const char *row = keys + mine * p.layout.slot_stride;
  for (int s0 = 0; s0 < count; s0 += AHEAD * ROWS) {
    uint4 raw[AHEAD];
    uint32_t units = 0, group[AHEAD];
    // the scale bytes of up to 32 keys, one to a lane
    if (FMT != kBf16) units = scale[min(s0 + lane, count - 1)];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const int s = min(s0 + a * ROWS + mine, count - 1);
      const char *from = s0 + a * ROWS + mine < count ? row : keys + (count - 1) * p.layout.slot_stride;      // behind the last key: the last again
      row += step;
      if (FMT == kBf16) {
        raw[a] = *reinterpret_cast<const uint4 *>(from);
      } else if (FMT == kE4m3) {
        const uint2 x = *reinterpret_cast<const uint2 *>(from);
        raw[a].x = x.x;
        raw[a].y = x.y;
      } else {
        raw[a].x = *reinterpret_cast<const uint32_t *>(from);
        group[a] = groups[(long long)s * (D / 16)];
      }
    }
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      uint32_t w[4] = {raw[a].x, raw[a].y, raw[a].z, raw[a].w};
      if (FMT != kBf16) {                               // exact in bf16: at most six bits
        uint32_t h[4];
        if (FMT == kE4m3) {
#pragma unroll
          for (int j = 0; j < 4; ++j) h[j] = half2_of_e4m3x2((j < 2 ? raw[a].x : raw[a].y) >> (16 * (j & 1)));
        } else {
          halves_of_e2m1(raw[a].x, h);
          const uint32_t s16 = half2_of_e4m3x2(group[a] * 0x101u);
#pragma unroll
          for (int j = 0; j < 4; ++j) h[j] = mul_half2(h[j], s16);
        }
        const float u = __uint_as_float(__shfl_sync(0xffffffffu, units, a * ROWS + mine) << 23);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 x = floats_of_half2(h[j]);
          const __nv_bfloat162 y = __floats2bfloat162_rn(x.x * u, x.y * u);
          w[j] = *reinterpret_cast<const uint32_t *>(&y);
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        top2[j] = max_bf16x2(top2[j], w[j]);
        low2[j] = min_bf16x2(low2[j], w[j]);
      }
    }
  }
  // over the keys of the other lanes, and the largest size over the dims: NaN if there is one, infinite if there is an infinity
  uint32_t size2 = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
#pragma unroll
    for (int o = LANES; o < 32; o <<= 1) {
      top2[j] = max_bf16x2(top2[j], __shfl_xor_sync(0xffffffffu, top2[j], o));
      low2[j] = min_bf16x2(low2[j], __shfl_xor_sync(0xffffffffu, low2[j], o));
    }
    size2 = max_bf16x2(size2, max_bf16x2(top2[j] & 0x7fff7fffu, low2[j] & 0x7fff7fffu));
  }
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) size2 = max_bf16x2(size2, __shfl_xor_sync(0xffffffffu, size2, o));
  size2 = max_bf16x2(size2, size2 >> 16 | size2 << 16);
  const uint32_t bits = size2 << 16;
  const bool fine = __uint_as_float(bits) <= 127.f * 0x1p60f;
  // size = m * 2^x with 1 <= m < 2; 127 = 1.984375 * 2^6
  const int e = max((int)(bits >> 23) - 127 - 6 + ((bits & 0x7fffffu) > 0x7e0000u), kMinBound);
  const float down = __uint_as_float((uint32_t)(127 - min(e, kMaxBound)) << 23);
  uint32_t up[2] = {}, lo[2] = {};
  if (fine) {
    // 1.5 * 2^23 added, rounded up or down: the whole number is in the lowest byte.  (The ieee forms: the others take subnormal keys for 0.)
    constexpr float kWhole = 12582912.f;
    uint32_t u8[8], l8[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t t = j & 1 ? top2[j / 2] & 0xffff0000u : top2[j / 2] << 16, l = j & 1 ? low2[j / 2] & 0xffff0000u : low2[j / 2] << 16;
      u8[j] = __float_as_uint(__fmaf_ieee_ru(__uint_as_float(t), down, kWhole));
      l8[j] = __float_as_uint(__fmaf_ieee_rd(__uint_as_float(l), down, kWhole));
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      up[h] = __byte_perm(__byte_perm(u8[4 * h], u8[4 * h + 1], 0x40), __byte_perm(u8[4 * h + 2], u8[4 * h + 3], 0x40), 0x5410);
      lo[h] = __byte_perm(__byte_perm(l8[4 * h], l8[4 * h + 1], 0x40), __byte_perm(l8[4 * h + 2], l8[4 * h + 3], 0x40), 0x5410);
    }
  }
  if (mine == 0) {
    int8_t *to = p.codes + ((long long)block * heads + head) * (2 * D) + sub * 8;
    *reinterpret_cast<uint2 *>(to) = make_uint2(up[0], up[1]);
    *reinterpret_cast<uint2 *>(to + D) = make_uint2(lo[0], lo[1]);
  }
  if (lane == 0) p.scales[(long long)block * heads + head] = (uint8_t)(fine ? e + 127 : kInfinite);
}

template <int D, int FMT>
int launch_bounds(const BoundsParams &p, cudaStream_t st) {
  const long long warps = (long long)p.n * p.n_kv_heads, ctas = (warps + kBoundThreads / 32 - 1) / (kBoundThreads / 32);
  if (ctas > 0x7fffffffll) return KV_ERR_SHAPE;
  block_bounds_kernel<D, FMT><<<(unsigned)ctas, kBoundThreads, 0, st>>>(p);
  KV_COUNT_LAUNCH();
  KV_CUDA(cudaGetLastError());
  return KV_OK;
}

template <int FMT>
int bounds_format(const BoundsParams &p, int d, cudaStream_t st) {
  return d == 128 ? launch_bounds<128, FMT>(p, st) : launch_bounds<64, FMT>(p, st);
}

// ---------------------------------------------------------------- scores
struct SelectParams {
  const void *q;
  long long q_stride, table_stride;
  int n_req, heads, group, num_blocks, block_size, max_ctx, max_blocks;
  int first, last, keep;
  const int8_t *codes;
  const uint8_t *scales;
  const int *tables, *lens;
  uint32_t *keys;             // scratch: [n_req][heads][max_blocks], the scores in an order-preserving code
  int *kept, *kept_lens;
};

__device__ __forceinline__ int blocks_of(const SelectParams &p, int r, int &len) {
  len = min(max(__ldg(p.lens + r), 0), p.max_ctx);
  return (len + p.block_size - 1) / p.block_size;
}
// fp32 -> a number whose order is the score's
__device__ __forceinline__ uint32_t key_of_score(float s) {
  const uint32_t b = __float_as_uint(s);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
constexpr uint32_t kAlways = 0xffffffffu;

__device__ __forceinline__ int dp4_ss(uint32_t a, uint32_t b, int c) {
  int r;
  asm("dp4a.s32.s32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}
__device__ __forceinline__ int dp4_su(uint32_t a, uint32_t b, int c) {
  int r;
  asm("dp4a.s32.u32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}

template <typename T>
__device__ __forceinline__ double value_of(T x);
template <>
__device__ __forceinline__ double value_of<float>(float x) { return fabsf(x) <= FLT_MAX ? (double)x : 0.0; }
template <>
__device__ __forceinline__ double value_of<bf16>(bf16 x) { return value_of<float>(__bfloat162float(x)); }

constexpr int kScoreThreads = 256;
constexpr int kScoreBlocks = 32;      // of a warp: a CTA's share is a multiple

// The code of a KV head's queries into shared memory: hi[i] * 256 + lo[i] for value i of [u+ | u-].  The sums are fp64: with up to 2^29
// between the heads' values they are exact.
template <int D, typename T>
__device__ __forceinline__ void query_code(const SelectParams &p, int req, int head, int8_t *hi, uint8_t *lo, double *warp_most) {
  const int i = threadIdx.x, lane = i & 31, warp = i >> 5;
  double u = 0.0;
  if (i < 2 * D) {
    const T *q = static_cast<const T *>(p.q) + req * p.q_stride + (long long)head * p.group * D + i % D;
#pragma unroll 8
    for (int h = 0; h < p.group; ++h) {
      const double x = value_of<T>(q[(long long)h * D]);
      u += i < D ? fmax(x, 0.0) : fmin(x, 0.0);
    }
  }
  double most = fabs(u);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) most = fmax(most, __shfl_xor_sync(0xffffffffu, most, o));
  if (lane == 0) warp_most[warp] = most;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kScoreThreads / 32; ++w) most = fmax(most, warp_most[w]);
  // most = m * 2^x with 1 <= m < 2; 32767 = (2 - 2^-14) * 2^14
  const unsigned long long bits = (unsigned long long)__double_as_longlong(most);
  int e = (int)(bits >> 52) - 1023 - 14 + ((bits & 0xfffffffffffffull) > 0xfffc000000000ull);
  e = max(e, -100);
  const int c = __double2int_rn(u * __longlong_as_double((long long)(1023 - e) << 52));
  if (i < 2 * D) {
    hi[i] = (int8_t)(c >> 8);
    lo[i] = (uint8_t)c;
  }
  __syncthreads();
}

// The scores of blocks [from, to) of a request for a KV head, in an order-preserving code; emit(block, key, id).  A warp takes a stage of
// 16 blocks (D = 64: 32) at a time: half a warp (a quarter) copies a block's codes, 16 bytes to a lane, and the sums over its lanes are
// exchanged so that lanes end with one block's each.  The copies of two stages, 8 KB a warp, are in flight in a ring of shared memory from
// which each lane reads what it copied itself (32 requests of up to 1,153 blocks, the whole selection 15.4 us; three stages 16.2; 8 KB in
// registers, with nothing in flight under the products, 17.8).  Table entries are looked up a stage before they are needed, and the first
// copies are on their way while the query's code is formed.
constexpr int kScoreStages = 2, kStageBytes = 4096;
constexpr int kRingBytes = kScoreThreads / 32 * kScoreStages * kStageBytes;
template <int D, typename T, typename Emit>
__device__ __forceinline__ void score_blocks(const SelectParams &p, int req, int head, int from, int to, unsigned char *ring, Emit emit) {
  constexpr int LPB = D / 8;                  // lanes of a block
  constexpr int N = 8;                        // blocks of those lanes in a stage
  constexpr int BLOCKS = N * (32 / LPB);      // of a stage
  constexpr int SHARE = LPB / N;              // lanes that end with the same block
  __shared__ __align__(16) int8_t hi_s[2 * D];
  __shared__ __align__(16) uint8_t lo_s[2 * D];
  __shared__ double most_s[kScoreThreads / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int l = lane % LPB;                   // the lane has values 16 l ... of a block's codes
  const int mine = lane / LPB * N + l / SHARE;      // the block of a stage that the lane looks up and ends with
  const int *table = p.tables + req * p.table_stride;
  const uint32_t mem = (uint32_t)__cvta_generic_to_shared(ring) + warp * (kScoreStages * kStageBytes) + lane * 16;
  int look = from + warp * BLOCKS + mine, put = 0;
  int next = -1, ids[kScoreStages], units[kScoreStages];      // ids and scale bytes of the stages in flight, the oldest first
  auto look_up = [&]() {
    next = look < to ? __ldg(table + look) : -1;
    look += kScoreThreads / 32 * BLOCKS;
  };
  auto issue = [&](int &id, int &unit) {
    id = next;
    const bool there = (unsigned)id < (unsigned)p.num_blocks;
    const bool any = look - kScoreThreads / 32 * BLOCKS - mine < to;      // the stage has blocks
    look_up();
    if (any) {
      const long long entry = there ? (long long)id * p.heads + head : 0;
      unit = there ? (int)__ldg(p.scales + entry) : kInfinite;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const long long at = __shfl_sync(0xffffffffu, entry, lane / LPB * LPB + i * SHARE);
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(mem + put * kStageBytes + i * 512), "l"(p.codes + at * (2 * D) + l * 16)
                     : "memory");
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    put = put + 1 == kScoreStages ? 0 : put + 1;
  };
  look_up();
#pragma unroll
  for (int i = 0; i < kScoreStages; ++i) issue(ids[i], units[i]);
  query_code<D, T>(p, req, head, hi_s, lo_s, most_s);
  const uint4 hv = *reinterpret_cast<const uint4 *>(hi_s + 16 * l), lv = *reinterpret_cast<const uint4 *>(lo_s + 16 * l);
  const uint32_t hi[4] = {hv.x, hv.y, hv.z, hv.w}, lo[4] = {lv.x, lv.y, lv.z, lv.w};
  for (int b0 = from + warp * BLOCKS; b0 < to; b0 += kScoreThreads / 32 * BLOCKS) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kScoreStages - 1) : "memory");
    int sum[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      uint32_t w[4];
      asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(mem + put * kStageBytes + i * 512) : "memory");
      int a = 0, c = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        a = dp4_ss(w[j], hi[j], a);
        c = dp4_su(w[j], lo[j], c);
      }
      sum[i] = a * 256 + c;
    }
    const int b = b0 + mine, id = ids[0], unit = units[0];
#pragma unroll
    for (int i = 0; i + 1 < kScoreStages; ++i) {
      ids[i] = ids[i + 1];
      units[i] = units[i + 1];
    }
    issue(ids[kScoreStages - 1], units[kScoreStages - 1]);      // into the stage just read
    // sums over the LPB lanes: half of the blocks handed over in each round, until one is left
#pragma unroll
    for (int o = LPB / 2; o > 0; o >>= 1) {
      constexpr int first = LPB / 2;
      const int left = N * o / first / 2;     // blocks after this round
      const bool upper = l & o;
      if (left == 0) {
        sum[0] += __shfl_xor_sync(0xffffffffu, sum[0], o);
        continue;
      }
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        if (i >= left) break;
        const int keep = upper ? sum[i + left] : sum[i], give = upper ? sum[i] : sum[i + left];
        sum[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
      }
    }
    const float score = (float)sum[0] * __uint_as_float((uint32_t)min(unit, 254) << 23);
    if (l % SHARE == 0 && b < to) emit(b, unit == kInfinite ? kAlways : key_of_score(score), id);
  }
}

// ---------------------------------------------------------------- choice
// What a context leaves for the choice: the middle blocks [from, to), of which `want` are taken; false if there is nothing to choose.  The
// blocks at the ends, or all of a short context, are written here, by the whole CTA.
__device__ __forceinline__ bool write_ends(const SelectParams &p, int req, int head, int n, int len, int *out, int &from, int &to, int &want) {
  const int tid = threadIdx.x, kept = min(n, p.keep);
  const int *table = p.tables + req * p.table_stride;
  if (head == 0 && tid == 0) p.kept_lens[req] = len - (n - kept) * p.block_size;
  for (int i = kept + tid; i < p.keep; i += kScoreThreads) out[i] = -1;
  if (n <= p.keep) {
    for (int i = tid; i < n; i += kScoreThreads) out[i] = __ldg(table + i);
    return false;
  }
  from = p.first;
  to = n - p.last;
  want = p.keep - p.first - p.last;
  for (int i = tid; i < p.first; i += kScoreThreads) out[i] = __ldg(table + i);
  for (int i = tid; i < p.last; i += kScoreThreads) out[p.keep - p.last + i] = __ldg(table + to + i);
  return want > 0;
}

// Up to kOwn keys of each thread stay in registers.
constexpr int kOwn = 8;
// The bar, which is the key of rank `want`, by a histogram of the scores: 512 bins, equal steps between the least and the largest finite
// one.  The bar's bin has a few keys, which one warp orders.  Returns the bar and how many keys reach it; 0 of them: the bin has more
// keys than a warp has lanes (equal scores, or one far from the others).
constexpr int kBins = 512;
__device__ __forceinline__ float score_of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ uint2 bar_of_few(const uint32_t (&own)[kOwn], int want, uint32_t least) {
  constexpr int W = kScoreThreads / 32, PER = kBins / 32;
  __shared__ int hist[kBins + 32];             // bin b at b + b / PER: the warp that adds them up reads without bank conflicts
  __shared__ uint32_t most_s[W], cand_s[32];
  __shared__ int bin_s, above_s, count_s, taken_s;
  __shared__ uint2 found_s;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  uint32_t most = 0;                          // of the finite ones
#pragma unroll
  for (int r = 0; r < kOwn; ++r) most = max(most, own[r] == kAlways ? 0u : own[r]);
  most = __reduce_max_sync(0xffffffffu, most);
  if (lane == 0) most_s[warp] = most;
#pragma unroll
  for (int i = tid; i < kBins + 32; i += kScoreThreads) hist[i] = 0;
  if (tid == 0) taken_s = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < W; ++w) most = max(most, most_s[w]);
  if (most <= least) return make_uint2(0, 0);
  const float low = score_of_key(least), scale = (kBins - 2) / (score_of_key(most) - low);
  if (!(scale > 0.f) || !(scale <= FLT_MAX)) return make_uint2(0, 0);
  // kBins - 1: without a bound.  Rounding keeps the order, so a bin's keys are neighbours.
  auto bin_of = [&](uint32_t k) { return k == kAlways ? kBins - 1 : min((int)((score_of_key(k) - low) * scale), kBins - 2); };
#pragma unroll
  for (int r = 0; r < kOwn; ++r)
    if (own[r] != 0) {
      const int b = bin_of(own[r]);
      atomicAdd(&hist[b + b / PER], 1);
    }
  __syncthreads();
  if (warp == 0) {
    // lane l has the PER bins from kBins - 1 - PER l down
    const int first = (31 - lane) * PER, *bins = hist + first + (31 - lane);
    int total = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) total += bins[i];
    int above = total;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, above, o);
      if (lane >= o) above += up;
    }
    above -= total;
    if (above < want && want <= above + total) {
      for (int i = PER - 1; i >= 0; --i) {
        const int c = bins[i];
        if (want <= above + c) {
          bin_s = first + i;
          above_s = above;
          count_s = c;
          break;
        }
        above += c;
      }
    }
  }
  __syncthreads();
  const int bin = bin_s, above = above_s, count = count_s;
  if (count > 32) return make_uint2(0, 0);
#pragma unroll
  for (int r = 0; r < kOwn; ++r)
    if (own[r] != 0 && bin_of(own[r]) == bin) cand_s[atomicAdd(&taken_s, 1)] = own[r];
  __syncthreads();
  if (warp == 0) {
    const uint32_t k = lane < count ? cand_s[lane] : 0;
    int more = 0, same = 0;
    for (int i = 0; i < count; ++i) {
      const uint32_t other = __shfl_sync(0xffffffffu, k, i);
      more += other > k;
      same += other == k;
    }
    if (k != 0 && above + more < want && want <= above + more + same) found_s = make_uint2(k, above + more + same);
  }
  __syncthreads();
  return found_s;
}

// The `want` largest of keys(0 .. m) by one CTA, the first of equal ones, written in their order: out[i] = ids(index).  0 < want <= m, and
// no key is 0.
// The bar comes from the histogram where all keys are in registers.  Otherwise, or where that gives none, it is found two bits at a
// time, from the first in which keys differ, with three counts of larger keys in each round; that ends as soon as a count is `want`.
// The histogram takes 1 to 1.5 us off the search of 500 to 1,150 keys.
template <typename Keys, typename Ids>
__device__ __forceinline__ void pick(const Keys &keys, int m, int want, const Ids &ids, int *out) {
  constexpr int W = kScoreThreads / 32;
  __shared__ uint32_t most_s[W], least_s[W];
  __shared__ int count_s[2][3][W];
  __shared__ __align__(8) uint32_t sums[kOwn * W];      // also read two at a time
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const bool few = m <= kOwn * kScoreThreads;
  uint32_t own[kOwn];
#pragma unroll
  for (int r = 0; r < kOwn; ++r) own[r] = tid + r * kScoreThreads < m ? keys(tid + r * kScoreThreads) : 0;
  auto each = [&](auto f) {
#pragma unroll
    for (int r = 0; r < kOwn; ++r) f(own[r]);
    if (!few)
      for (int i = tid + kOwn * kScoreThreads; i < m; i += kScoreThreads) f(keys(i));
  };
  uint32_t most = 0, least = 0xffffffffu;
  each([&](uint32_t k) {
    most = max(most, k);
    least = min(least, k - 1u);               // 0 is none
  });
  most = __reduce_max_sync(0xffffffffu, most);
  least = __reduce_min_sync(0xffffffffu, least);
  if (lane == 0) {
    most_s[warp] = most;
    least_s[warp] = least;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < W; ++w) {
    most = max(most, most_s[w]);
    least = min(least, least_s[w]);
  }
  ++least;
  const uint2 found = few ? bar_of_few(own, want, least) : make_uint2(0, 0);
  // the largest bar with at least `want` keys that reach it, its bits from the top one in which keys differ
  int bits = most == least || found.y ? 0 : 32 - __clz(most ^ least), reach = found.y ? (int)found.y : m;
  bits += bits & 1;
  uint32_t bar = found.y ? found.x : bits >= 32 ? 0u : most & ~((1u << bits) - 1u);
  for (int turn = 0; bits > 0 && reach != want; turn ^= 1) {
    bits -= 2;
    const uint32_t b1 = bar + (1u << bits), b2 = bar + (2u << bits), b3 = bar + (3u << bits);
    int c1 = 0, c2 = 0, c3 = 0;               // keys that reach them
    each([&](uint32_t k) {
      c1 += k >= b1;
      c2 += k >= b2;
      c3 += k >= b3;
    });
    c1 = __reduce_add_sync(0xffffffffu, c1);
    c2 = __reduce_add_sync(0xffffffffu, c2);
    c3 = __reduce_add_sync(0xffffffffu, c3);
    if (lane < 3) count_s[turn][lane][warp] = lane == 0 ? c1 : lane == 1 ? c2 : c3;
    __syncthreads();
    c1 = c2 = c3 = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      c1 += count_s[turn][0][w];
      c2 += count_s[turn][1][w];
      c3 += count_s[turn][2][w];
    }
    if (c3 >= want) {
      bar = b3;
      reach = c3;
    } else if (c2 >= want) {
      bar = b2;
      reach = c2;
    } else if (c1 >= want) {
      bar = b1;
      reach = c1;
    }
  }
  // ---- keys above the bar, and of those on it what is wanting (all, if the search ended early)
  const bool all = reach == want;
  int ties = 0;
  if (!all) {                                 // the bar is a key, and has equals
    uint32_t above = 0;
    each([&](uint32_t k) { above += k > bar; });
    above = __reduce_add_sync(0xffffffffu, above);
    __syncthreads();
    if (lane == 0) count_s[0][0][warp] = (int)above;
    __syncthreads();
    ties = want;
#pragma unroll
    for (int w = 0; w < W; ++w) ties -= count_s[0][0][w];
  }
  // ---- their places: rounds of kOwn keys a thread, the counts of all warps and all keys of a round scanned by one warp
  int taken = 0, equals = 0;                  // so far
  const unsigned below = (1u << lane) - 1u;
  for (int i0 = 0; i0 < m; i0 += kOwn * kScoreThreads) {
    unsigned more_w[kOwn], same_w[kOwn];
#pragma unroll
    for (int r = 0; r < kOwn; ++r) {
      const int i = i0 + r * kScoreThreads + tid;
      const uint32_t k = i0 == 0 ? own[r] : i < m ? keys(i) : 0;
      more_w[r] = __ballot_sync(0xffffffffu, all ? k >= bar && k > 0 : k > bar);
      same_w[r] = __ballot_sync(0xffffffffu, !all && k == bar);
      if (lane == r) sums[r * W + warp] = __popc(more_w[r]) | __popc(same_w[r]) << 16;
    }
    __syncthreads();
    if (warp == 0) {
      const uint2 two = reinterpret_cast<const uint2 *>(sums)[lane];
      uint32_t scan = two.x + two.y;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t up = __shfl_up_sync(0xffffffffu, scan, o);
        if (lane >= o) scan += up;
      }
      reinterpret_cast<uint2 *>(sums)[lane] = make_uint2(scan - two.y, scan);      // inclusive
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kOwn; ++r) {
      const int i = i0 + r * kScoreThreads + tid;
      const uint32_t before = r * W + warp > 0 ? sums[r * W + warp - 1] : 0;
      const int same_before = equals + (int)(before >> 16) + __popc(same_w[r] & below);
      const int more_before = (int)(before & 0xffffu) + __popc(more_w[r] & below);
      const bool take = (more_w[r] >> lane & 1u) || ((same_w[r] >> lane & 1u) && same_before < ties);
      if (take) out[taken + more_before + min(same_before, ties) - min(equals, ties)] = ids(i);
    }
    const uint32_t total = sums[kOwn * W - 1];
    const int equals_new = equals + (int)(total >> 16);
    taken += (int)(total & 0xffffu) + min(equals_new, ties) - min(equals, ties);
    equals = equals_new;
    if (taken >= want) break;
    __syncthreads();
  }
}

// Up to kClusterBlocks blocks: a cluster of CTAs shares the blocks of a (request, KV head), hands the keys and the blocks' ids to its first CTA's
// shared memory, and that one chooses.  One launch, and no keys in global memory (32 requests of up to 1,153 blocks, before the ring, against a kernel
// for the scores and one for the choice: 19.9 / 29.8 us).
constexpr int kClusterBlocks = 16384;      // 128 KB of keys and ids, and the ring
constexpr int kSmBytes = 228 * 1024, kSelectStatic = 4608;      // shared memory of an SM; of a CTA beside that: its static arrays, and 1 KB that is reserved
template <int D, typename T>
__global__ void __launch_bounds__(kScoreThreads) select_cluster_kernel(const __grid_constant__ SelectParams p) {
  extern __shared__ __align__(16) unsigned char select_smem[];
  uint32_t *keys_s = reinterpret_cast<uint32_t *>(select_smem + kRingBytes);
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  const int req = blockIdx.z, head = blockIdx.y, rank = (int)cluster.block_rank(), ctas = (int)cluster.num_blocks();
  int len, from = 0, to = 0, want = 0;
  const int n = blocks_of(p, req, len);
  if (n <= p.keep || p.keep == p.first + p.last) {      // nothing to choose: the same for the whole cluster
    if (rank == 0) write_ends(p, req, head, n, len, p.kept + ((long long)req * p.heads + head) * p.keep, from, to, want);
    return;
  }
  if (ctas > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  from = p.first;
  to = n - p.last;
  // whole rounds of the warps to a CTA
  const int each = ((to - from + ctas - 1) / ctas + kScoreBlocks - 1) / kScoreBlocks * kScoreBlocks;
  const int mine = from + rank * each;
  int *ids_s = reinterpret_cast<int *>(keys_s + p.max_blocks);
  uint32_t *keys = ctas > 1 ? cluster.map_shared_rank(keys_s, 0) : keys_s;
  int *ids = reinterpret_cast<int *>(keys + p.max_blocks);
  if (ctas > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");      // the first CTA is there
  if (mine < to)
    score_blocks<D, T>(p, req, head, mine, min(mine + each, to), select_smem, [&](int b, uint32_t key, int id) {
      keys[b - from] = key;
      ids[b - from] = id;
    });
  if (ctas > 1)
    cluster.sync();
  else
    __syncthreads();
  if (rank > 0) return;
  int *out = p.kept + ((long long)req * p.heads + head) * p.keep;
  write_ends(p, req, head, n, len, out, from, to, want);
  pick([&](int i) { return keys_s[i]; }, to - from, want, [&](int i) { return ids_s[i]; }, out + p.first);
}

// More blocks than that: the keys go through global memory, and a CTA for each (request, KV head) chooses.
template <int D, typename T>
__global__ void __launch_bounds__(kScoreThreads) block_score_kernel(const __grid_constant__ SelectParams p, int chunk) {
  const int req = blockIdx.z, head = blockIdx.y;
  int len;
  const int n = blocks_of(p, req, len);
  if (n <= p.keep) return;                    // all of them are chosen
  const int from = p.first + blockIdx.x * chunk, to = min(from + chunk, n - p.last);
  if (from >= to) return;
  uint32_t *keys = p.keys + ((long long)req * p.heads + head) * p.max_blocks;
  extern __shared__ __align__(16) unsigned char select_smem[];
  score_blocks<D, T>(p, req, head, from, to, select_smem, [&](int b, uint32_t key, int) { keys[b] = key; });
}
__global__ void __launch_bounds__(kScoreThreads) block_pick_kernel(const __grid_constant__ SelectParams p) {
  const int req = blockIdx.x, head = blockIdx.y;
  int len, from, to, want;
  const int n = blocks_of(p, req, len);
  int *out = p.kept + ((long long)req * p.heads + head) * p.keep;
  if (!write_ends(p, req, head, n, len, out, from, to, want)) return;
  const uint32_t *keys = p.keys + ((long long)req * p.heads + head) * p.max_blocks + from;
  const int *table = p.tables + req * p.table_stride + from;
  pick([&](int i) { return keys[i]; }, to - from, want, [&](int i) { return __ldg(table + i); }, out + p.first);
}

int select_max_blocks(int max_ctx, int block_size) { return (int)(((long long)max_ctx + block_size - 1) / block_size); }

template <int D, typename T>
int launch_select(const SelectParams &p, int device, cudaStream_t st) {
  const int middle = p.max_blocks - p.first - p.last, sms = sm_count(device);
  const long long lines = (long long)p.n_req * p.heads;
  if (p.max_blocks <= kClusterBlocks) {
    auto kernel = select_cluster_kernel<D, T>;
    static bool attr_set[kMaxDevices] = {};
    if (!attr_set[device]) {
      KV_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingBytes + kClusterBlocks * 8));
      attr_set[device] = true;
    }
    // As many CTAs as run at once, of at least four warps' blocks each.  Two to an SM: twice as many CTAs, 16 requests of up to 512
    // blocks 9.4 -> 11.3 us, 32 of up to 1,153 15.4 -> 19.7.  One, where keys and ids of more than some 5,800 blocks leave no room for a second:
    // with CTAs for two, 4 / 8 / 16 requests of 8,192 blocks 33.8 / 43.8 / 62.6 -> 43.5 / 59.1 / 79.7 us, all of 16,384 51 / 74 / 111 -> 66 / 97 /
    // 136; ragged ones 10 % slower to 10 % faster.
    const int per_sm = 2 * (kRingBytes + p.max_blocks * 8 + kSelectStatic) <= kSmBytes ? 2 : 1;
    int ctas = 1;
    while (ctas < 8 && lines * ctas * 2 <= (long long)per_sm * sms && middle > ctas * 4 * kScoreBlocks) ctas *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas, p.heads, p.n_req);
    cfg.blockDim = dim3(kScoreThreads);
    cfg.dynamicSmemBytes = p.max_blocks > p.keep ? (size_t)(kRingBytes + p.max_blocks * 8) : 0;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    KV_CUDA(cudaLaunchKernelEx(&cfg, kernel, p));
    KV_COUNT_LAUNCH();
    return KV_OK;
  }
  if (p.max_blocks > p.keep) {
    // a batch of blocks for every warp, or as many more as leave two CTAs for each SM
    const long long batches = (middle + kScoreThreads - 1) / kScoreThreads;
    const long long each = batches * lines / (2ll * sms);
    const int chunk = (int)(each > 1 ? each < batches ? each : batches : 1) * kScoreThreads;
    const dim3 grid((middle + chunk - 1) / chunk, p.heads, p.n_req);
    static bool score_set[kMaxDevices] = {};
    if (!score_set[device]) {
      KV_CUDA(cudaFuncSetAttribute(block_score_kernel<D, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingBytes));
      score_set[device] = true;
    }
    block_score_kernel<D, T><<<grid, kScoreThreads, kRingBytes, st>>>(p, chunk);
    KV_COUNT_LAUNCH();
    KV_CUDA(cudaGetLastError());
  }
  block_pick_kernel<<<dim3(p.n_req, p.heads), kScoreThreads, 0, st>>>(p);
  KV_COUNT_LAUNCH();
  KV_CUDA(cudaGetLastError());
  return KV_OK;
}

}  // namespace
}  // namespace kvr

extern "C" {

int32_t kv_op_block_bounds(const kv_cache_desc *cache, int32_t layer, const int32_t *blocks_dev, const int32_t *counts_dev, int32_t n,
                           int8_t *bounds_dev, uint8_t *bound_scales_dev, void *stream) {
  using namespace kvr;
  if (n < 0) return KV_ERR_ARG;
  int rc = check_cache_desc(cache, true);
  if (rc != KV_OK) return rc;
  if (cache->head_dim != 64 && cache->head_dim != 128) return KV_ERR_SHAPE;
  if (layer < 0 || layer >= cache->n_layers) return KV_ERR_SHAPE;
  if (cache->block_size > 1 << 30) return KV_ERR_SHAPE;      // keys are counted in 32 bits, those of a load ahead
  if (n == 0) return KV_OK;
  if (blocks_dev == nullptr || counts_dev == nullptr || bounds_dev == nullptr || bound_scales_dev == nullptr) return KV_ERR_ARG;
  if (((uintptr_t)blocks_dev & 3) || ((uintptr_t)counts_dev & 3) || ((uintptr_t)bounds_dev & 15)) return KV_ERR_ARG;
  BoundsParams p;
  p.layout = row_layout(make_view(cache), layer);
  p.block_size = cache->block_size;
  p.n_kv_heads = cache->n_kv_heads;
  p.num_blocks = cache->num_blocks;
  p.n = n;
  p.blocks = blocks_dev;
  p.counts = counts_dev;
  p.codes = bounds_dev;
  p.scales = bound_scales_dev;
  cudaStream_t st = (cudaStream_t)stream;
  switch (format_of(cache->elem_bytes)) {
    case kBf16: return bounds_format<kBf16>(p, cache->head_dim, st);
    case kE4m3: return bounds_format<kE4m3>(p, cache->head_dim, st);
    default: return bounds_format<kE2m1>(p, cache->head_dim, st);
  }
}

int64_t kv_select_blocks_scratch_bytes(int32_t n_req, int32_t n_kv_heads, int32_t block_size, int32_t max_ctx) {
  using namespace kvr;
  if (n_req < 0 || n_kv_heads <= 0 || block_size <= 0 || max_ctx <= 0) return KV_ERR_ARG;
  if (max_ctx > kSelMaxCtx) return KV_ERR_SHAPE;
  return ((long long)n_req * n_kv_heads * select_max_blocks(max_ctx, block_size) * 4 + 255) / 256 * 256;
}

int32_t kv_op_select_blocks(const void *q_dev, int64_t q_stride, int32_t dtype, int32_t n_req, int32_t n_q_heads, int32_t n_kv_heads,
                            int32_t head_dim, const int8_t *bounds_dev, const uint8_t *bound_scales_dev, int32_t num_blocks,
                            int32_t block_size, const int32_t *block_tables_dev, int64_t table_stride, const int32_t *context_lens_dev,
                            int32_t max_ctx, int32_t first, int32_t last, int32_t keep, void *scratch_dev, int64_t scratch_bytes,
                            int32_t *kept_dev, int32_t *kept_lens_dev, void *stream) {
  using namespace kvr;
  if (n_req < 0 || n_q_heads <= 0 || n_kv_heads <= 0 || num_blocks <= 0 || block_size <= 0 || max_ctx <= 0) return KV_ERR_ARG;
  if (dtype != KV_DTYPE_BF16 && dtype != KV_DTYPE_F32) return KV_ERR_ARG;
  // the last block may be partly filled: only there can a chosen context end
  if (first < 0 || last < 1 || keep < 1 || (long long)first + last > keep) return KV_ERR_ARG;
  if (n_q_heads % n_kv_heads != 0 || (head_dim != 64 && head_dim != 128)) return KV_ERR_SHAPE;
  if (max_ctx > kSelMaxCtx || (long long)keep * block_size > kSelMaxCtx || n_req > 65535 || n_kv_heads > 65535) return KV_ERR_SHAPE;
  if (n_req == 0) return KV_OK;
  if (q_dev == nullptr || bounds_dev == nullptr || bound_scales_dev == nullptr || block_tables_dev == nullptr ||
      context_lens_dev == nullptr || kept_dev == nullptr || kept_lens_dev == nullptr)
    return KV_ERR_ARG;
  const int size = dtype == KV_DTYPE_BF16 ? 2 : 4;
  if (((uintptr_t)q_dev & 15) || q_stride < 0 || q_stride * size % 16 != 0 || table_stride < 0 || ((uintptr_t)bounds_dev & 15)) return KV_ERR_ARG;
  for (const void *x : {(const void *)block_tables_dev, (const void *)context_lens_dev, (const void *)kept_dev, (const void *)kept_lens_dev})
    if ((uintptr_t)x & 3) return KV_ERR_ARG;
  const int max_blocks = select_max_blocks(max_ctx, block_size);
  if (table_stride < max_blocks) return KV_ERR_TABLE_SHORT;
  if (max_blocks > keep) {
    const long long need = (long long)n_req * n_kv_heads * max_blocks * 4;
    if (scratch_dev == nullptr || ((uintptr_t)scratch_dev & 15) || scratch_bytes < need) return KV_ERR_WORKSPACE;
  }
  const int device = current_device();
  if (device < 0) return KV_ERR_CUDA;
  SelectParams p;
  p.q = q_dev;
  p.q_stride = q_stride;
  p.table_stride = table_stride;
  p.n_req = n_req;
  p.heads = n_kv_heads;
  p.group = n_q_heads / n_kv_heads;
  p.num_blocks = num_blocks;
  p.block_size = block_size;
  p.max_ctx = max_ctx;
  p.max_blocks = max_blocks;
  p.first = first;
  p.last = last;
  p.keep = keep;
  p.codes = bounds_dev;
  p.scales = bound_scales_dev;
  p.tables = block_tables_dev;
  p.lens = context_lens_dev;
  p.keys = static_cast<uint32_t *>(scratch_dev);
  p.kept = kept_dev;
  p.kept_lens = kept_lens_dev;
  cudaStream_t st = (cudaStream_t)stream;
  if (head_dim == 128) return dtype == KV_DTYPE_F32 ? launch_select<128, float>(p, device, st) : launch_select<128, bf16>(p, device, st);
  return dtype == KV_DTYPE_F32 ? launch_select<64, float>(p, device, st) : launch_select<64, bf16>(p, device, st);
}

}  // extern "C"
