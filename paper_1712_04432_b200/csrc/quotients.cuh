// Rows in 8 bits: s = max |x| / 127 in float, q = x / s rounded to the nearest integer (halves to even).  The scale of a row and the
// quotients of eight of its values, shared by the row quantiser and the norm that leaves its rows in 8 bits.
#pragma once
#include <stdint.h>

#include "pairs.cuh"

namespace mbd {

// The quotient, correctly rounded to an integer: a float quotient that is exactly half a step may have been rounded to it, the
// remainder tells.  (The scale is below 1e-30 here: the remainder is taken 2^64 times as large, all products being exact, since one of half
// the smallest denormal number would be rounded to zero.)
static __device__ __noinline__ float divide_to_integer(float x, float s) {
  constexpr float LARGE = 18446744073709551616.f;
  const float t = __fdiv_rn(x, s);
  float k = rintf(t);
  if (fabsf(t - k) == 0.5f) {
    const float rest = fmaf(-t * LARGE, s, x * LARGE);
    if (rest > 0.f) k = ceilf(t);
    if (rest < 0.f) k = floorf(t);
  }
  return fminf(fmaxf(k, -127.f), 127.f);
}

// The quotient with the reciprocal is off by 127 * 2^-23 at most (both roundings); one that is not nearer than NEAR to half a step
// rounds to the right integer.
constexpr float NEAR = 2e-5f;

// Eight quotients as bytes.  Adding 1.5 * 2^23 leaves a number's nearest integer (halves to even) in the low bits of its float.
__device__ __forceinline__ uint2 quotients(const f32x2* x, float s, float inv, bool tiny) {
  constexpr float MAGIC = 12582912.f;
  const f32x2 inv2 = pair(inv, inv), magic = pair(MAGIC, MAGIC), back = pair(-MAGIC, -MAGIC), minus = pair(-1.f, -1.f);
  uint32_t k[8];
  float t[8], worst = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const f32x2 t2 = mul2(x[j], inv2), r = add2(t2, magic);
    const float2 tf = floats(t2), rf = floats(r), off = floats(fma2(t2, minus, add2(r, back)));
    t[2 * j] = tf.x; t[2 * j + 1] = tf.y;
    k[2 * j] = __float_as_uint(rf.x); k[2 * j + 1] = __float_as_uint(rf.y);
    asm("max.abs.f32 %0, %0, %1, %2;" : "+f"(worst) : "f"(off.x), "f"(off.y));
  }
  if (tiny) {                                            // a scale whose reciprocal is no good
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float2 f = floats(x[j >> 1]);
      k[j] = s > 0.f ? static_cast<uint32_t>(static_cast<int>(divide_to_integer(j & 1 ? f.y : f.x, s))) : 0u;
    }
  } else if (worst > 0.5f - NEAR) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float low = floorf(t[j]), half = low + 0.5f;
      if (fabsf(t[j] - half) < NEAR) {                   // which side of the half step: x - half * s, of which the sign is exact
        const float2 f = floats(x[j >> 1]);
        const float rest = fmaf(-half, s, j & 1 ? f.y : f.x);
        k[j] = __float_as_uint((rest > 0.f ? low + 1.f : rest < 0.f ? low : rintf(half)) + MAGIC);
      }
    }
  }
  return make_uint2(__byte_perm(__byte_perm(k[0], k[1], 0x0040), __byte_perm(k[2], k[3], 0x0040), 0x5410),
                    __byte_perm(__byte_perm(k[4], k[5], 0x0040), __byte_perm(k[6], k[7], 0x0040), 0x5410));
}

struct Scale { float s, inv; bool tiny; };
__device__ __forceinline__ Scale scale_of(uint32_t bits) {
  const bool finite = bits < 0x7F800000u;                      // a row with an infinity or a NaN has no scale: it is NaN, and q is 0
  Scale r;
  r.s = finite ? __fdiv_rn(__uint_as_float(bits), 127.f) : __uint_as_float(0x7FC00000u);
  r.tiny = !(r.s >= 1e-30f);                                   // (zero, NaN, or so small that its reciprocal is not accurate)
  r.inv = r.tiny ? 0.f : __fdiv_rn(1.f, r.s);
  return r;
}

}  // namespace mbd
