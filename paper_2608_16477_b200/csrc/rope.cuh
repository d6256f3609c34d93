// What the kernels that turn heads share: the plan and the sine and cosine of a pair (internal).
#pragma once
#include "common.cuh"

struct kv_rope {
  kv_rope_desc d;
  double theta[128];   // frequencies of the pairs
  double turns[128];   // theta / (2 pi)
};

namespace kvr {
namespace {

constexpr int kRopeMaxPairs = 128;

// (cos, sign * sin) of position * turns turns, times gain.  The angle is reduced to [-1/2, 1/2] turn in fp64; the product with
// gain is a rounding of its own, 2^-24 beside sincospi's ulp, and none where gain is 1: fp64 for it would be an operation more
// for each pair of every token.
__device__ __forceinline__ float2 rope_turn(int position, double turns, float gain, float sign) {
  const double a = (double)position * turns;
  float s, c;
  sincospif(2.0f * (float)(a - rint(a)), &s, &c);
  return make_float2(c * gain, s * (gain * sign));
}

// The turned members of a pair (a, b), w = (cos, sin).  Which product takes part in the fma is written out: kernels that turn the same
// head have to leave the same bits.
__device__ __forceinline__ float turned_first(float a, float b, float2 w) { return fmaf(a, w.x, -(b * w.y)); }
__device__ __forceinline__ float turned_second(float a, float b, float2 w) { return fmaf(a, w.y, b * w.x); }
// The same of interleaved pairs in the first 16 of 32 bytes of a head, where vectors are turned: the bits that these kernels have always
// left (the two differ by an ulp at most).
__device__ __forceinline__ float turned_neighbour(float a, float b, float2 w) { return fmaf(b, w.x, a * w.y); }

}  // namespace
}  // namespace kvr
