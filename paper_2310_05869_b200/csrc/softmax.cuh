// Softmax of rows whose scores and outputs are in TMEM: what the attention kernels of the serving entry points share.
#pragma once
#include "serving.cuh"
#include "tc_util.cuh"

namespace hyperattn {
namespace {

constexpr float kSumLimit = 32768.f;    // a tile whose weights sum to more has its reference moved (fp16 weights end at 2^16)
constexpr float kMostByArithmetic = 120.f;       // and one with a weight beyond 2 to that (which exp2_pair does not make; those up to it show in the sum)

// (NaN if one of them is)
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// 2^x of two numbers up to 127 by arithmetic: x = n + f with n the nearest integer, 2^f by a polynomial of degree 4 (its coefficients a least-maximum
// fit of the relative error over -1/2 .. 1/2: 2.7e-6), n added to the exponent.  Below -125 x counts as that, and what it gives is taken off every result: zero for
// those, no difference to others.  (ZERO; where results become fp16 it is zero anyway, and sums do not show it.)  Above 2^127 the exponent does not hold n,
// so the caller looks at the largest x, which goes to `most` (NaN if one is).  The exponential unit makes 16 a clock and SM, which is what a tile of scores
// takes longest for; so some of them are made here.
template <bool ZERO>
__device__ __forceinline__ uint64_t exp2_pair(uint64_t x2, float& most) {
  float x, y;
  unpack_f2(x2, x, y);
  most = max3(most, x, y);
  x2 = pack_f2(max3(x, -125.f, -125.f), max3(y, -125.f, -125.f));                       // (NaN stays, and becomes a huge number or NaN)
  const uint64_t t = fadd2(x2, pack_f2(12582912.f, 12582912.f));                      // 1.5 * 2^23 + n
  const uint64_t f = ffma2(fadd2(t, pack_f2(-12582912.f, -12582912.f)), pack_f2(-1.f, -1.f), x2);
  uint64_t p = ffma2(f, pack_f2(0.009570102207362652f, 0.009570102207362652f), pack_f2(0.05591786280274391f, 0.05591786280274391f));
  p = ffma2(f, p, pack_f2(0.240247443318367f, 0.240247443318367f));
  p = ffma2(f, p, pack_f2(0.6931217908859253f, 0.6931217908859253f));
  p = ffma2(f, p, pack_f2(0.9999992847442627f, 0.9999992847442627f));
  float p0, p1, t0, t1;
  unpack_f2(p, p0, p1);
  unpack_f2(t, t0, t1);
  const uint64_t w = pack_u2(__float_as_uint(p0) + (__float_as_uint(t0) << 23), __float_as_uint(p1) + (__float_as_uint(t1) << 23));
  constexpr float least = 0.9999992847442627f * 0x1p-125f;
  return ZERO ? fadd2(w, pack_f2(-least, -least)) : w;
}

// O of a row times alpha, in TMEM (rare).  All lanes together.
__device__ __noinline__ void rescale_o(uint32_t addr, int cols, float alpha) {
  uint32_t r[16];
  for (int c = 0; c < cols; c += 16) {
    tmem_ld16_issue(addr + c, r);
    tmem_ld16_wait(r);
#pragma unroll
    for (int e = 0; e < 16; ++e) r[e] = __float_as_uint(__uint_as_float(r[e]) * alpha);
    tmem_st16(addr + c, r);
  }
  tmem_wait_st();
}

}  // namespace
}  // namespace hyperattn
