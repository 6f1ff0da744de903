// One AdamW step over a list of tensors in one launch.  With g = grad * grad_scale (the library's gradients are sums over the
// batch, so grad_scale is 1 / B) and t the number of this step:
//     m <- b1 m + (1 - b1) g ,  v <- b2 v + (1 - b2) g^2
//     w <- w (1 - lr decay) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
// Moments are float, or 8 bits: blocks of 256 consecutive elements of a tensor share a float scale, the elements are e4m3
// numbers (a relative step of 2^-4 over 17 octaves, where an 8-bit integer has a fixed step), the largest of a block at
// 448.  Of v the root is held, which has half the octaves of v and is what the step divides by; a root that is not zero is never
// rounded to zero (smallest number of the type instead), so that a small m is not divided by eps alone.  The step itself is
// computed from the new moments before they are rounded.
//
// Bound by HBM: 30 bytes per element with float moments, bf16 weights, float masters and gradients, 18 with 8 bits, 8 with 8 bits and
// bf16 throughout.  58.6 M elements: 0.292 - 0.298 ms (5.9 - 6.0 TB/s, 90 - 92 % of the measured copy rate) and 0.206 ms (5.1 TB/s); 48 M elements in 240
// tensors, all bf16 and 8 bits: 0.103 ms (3.7 TB/s: there the instructions count, about 50 per element of them).  A warp owns 256
// consecutive elements, so that a block's maximum is one warp reduction; a thread block takes one contiguous range of the list
// (a stride over the whole grid was 1 % faster on a few large tensors and 28 % slower on many).
#include <math.h>

#include <algorithm>
#include <new>
#include <vector>

#include <cuda_fp8.h>

#include "../../include/mbd.h"
#include "epi.cuh"
#include "pairs.cuh"

namespace mbd {
namespace {

constexpr int BLOCK = 256;             // elements per warp and pass; also the elements that share a scale
constexpr int THREADS = 256, WARPS = THREADS / 32;

struct Tensor {
  void* p;
  float* master;
  const void* g;
  void* m;
  void* v;
  float* ms;
  float* vs;
  int64_t n;
  float decay;
  int flags;                           // see below
};
enum { P_BF16 = 1, G_BF16 = 2, MASTERED = 4, WIDE = 8 };

struct Clock {                         // device: steps taken, and the powers of the two rates
  double b1_t, b2_t;
  long long t;
  unsigned int seen;
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ float approx_root(float x) {
  float r;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float approx_reciprocal(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// ------------------------------------------------------------------------------------------------ four elements of a tensor
// Raw values as they are held; n: how many of the four are there, WHOLE: all, and aligned for one access.
constexpr int WHOLE = 8;

__device__ __forceinline__ uint4 read_floats(const char* base, int n) {
  const float* p = reinterpret_cast<const float*>(base);
  if (n == WHOLE) return *reinterpret_cast<const uint4*>(p);
  uint4 q;
  q.x = n > 0 ? __float_as_uint(p[0]) : 0u;
  q.y = n > 1 ? __float_as_uint(p[1]) : 0u;
  q.z = n > 2 ? __float_as_uint(p[2]) : 0u;
  q.w = n > 3 ? __float_as_uint(p[3]) : 0u;
  return q;
}
__device__ __forceinline__ uint4 read_bf16(const char* base, int n) {
  const uint16_t* p = reinterpret_cast<const uint16_t*>(base);
  uint4 q = make_uint4(0, 0, 0, 0);
  if (n == WHOLE) {
    const uint2 h = *reinterpret_cast<const uint2*>(p);
    q.x = h.x; q.y = h.y;
  } else {
    q.x = (n > 0 ? p[0] : 0u) | (n > 1 ? static_cast<uint32_t>(p[1]) << 16 : 0u);
    q.y = (n > 2 ? p[2] : 0u) | (n > 3 ? static_cast<uint32_t>(p[3]) << 16 : 0u);
  }
  return q;
}
__device__ __forceinline__ uint32_t read_codes(const char* base, int n) {
  const uint8_t* p = reinterpret_cast<const uint8_t*>(base);
  if (n == WHOLE) return *reinterpret_cast<const uint32_t*>(p);
  uint32_t q = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) if (i < n) q |= static_cast<uint32_t>(p[i]) << (8 * i);
  return q;
}
__device__ __forceinline__ void write_floats(char* base, int n, const f32x2* x) {
  float* p = reinterpret_cast<float*>(base);
  const float2 a = floats(x[0]), b = floats(x[1]);
  if (n == WHOLE) { __stcs(reinterpret_cast<float4*>(p), make_float4(a.x, a.y, b.x, b.y)); return; }
  if (n > 0) p[0] = a.x;
  if (n > 1) p[1] = a.y;
  if (n > 2) p[2] = b.x;
  if (n > 3) p[3] = b.y;
}
__device__ __forceinline__ void write_bf16(char* base, int n, const f32x2* x) {
  uint16_t* p = reinterpret_cast<uint16_t*>(base);
  const float2 a = floats(x[0]), b = floats(x[1]);
  const uint2 q = make_uint2(pack_bf16x2(a.x, a.y), pack_bf16x2(b.x, b.y));
  if (n == WHOLE) { *reinterpret_cast<uint2*>(p) = q; return; }
  if (n > 0) p[0] = static_cast<uint16_t>(q.x);
  if (n > 1) p[1] = static_cast<uint16_t>(q.x >> 16);
  if (n > 2) p[2] = static_cast<uint16_t>(q.y);
  if (n > 3) p[3] = static_cast<uint16_t>(q.y >> 16);
}
__device__ __forceinline__ void write_codes(char* base, int n, uint32_t q) {
  uint8_t* p = reinterpret_cast<uint8_t*>(base);
  if (n == WHOLE) { *reinterpret_cast<uint32_t*>(p) = q; return; }
#pragma unroll
  for (int i = 0; i < 4; ++i) if (i < n) p[i] = static_cast<uint8_t>(q >> (8 * i));
}
__device__ __forceinline__ void of_floats(const uint4& q, f32x2* x) {
  x[0] = pair(__uint_as_float(q.x), __uint_as_float(q.y));
  x[1] = pair(__uint_as_float(q.z), __uint_as_float(q.w));
}
__device__ __forceinline__ void of_bf16(const uint4& q, f32x2* x) {
  x[0] = pair(__uint_as_float(q.x << 16), __uint_as_float(q.x & 0xFFFF0000u));
  x[1] = pair(__uint_as_float(q.y << 16), __uint_as_float(q.y & 0xFFFF0000u));
}
__device__ __forceinline__ void of_codes(uint32_t q, f32x2* x) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float2 f = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(q >> (16 * h)), __NV_E4M3)));
    x[h] = pair(f.x, f.y);
  }
}
__device__ __forceinline__ uint32_t to_codes(f32x2 a, f32x2 b) {       // nearest, halves to even, NaN stays NaN
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(floats(a), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(floats(b), __NV_SATFINITE, __NV_E4M3);
  return lo | (hi << 16);
}

// ------------------------------------------------------------------------------------------------ moments in 8 bits
constexpr float E4M3_MAX = 448.f, E4M3_MIN = 0.001953125f;

__device__ __forceinline__ float warp_max(const f32x2* x) {            // the largest |x| of a warp's 8 x 32 values; NaN if there is one
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = floats(x[i]);
    asm("max.NaN.abs.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(f.x), "f"(f.y));
  }
  float r;
  asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(m));
  return r;
}

// x / 448, correctly rounded for ordinary x: the product with the rounded reciprocal, corrected once by its remainder.
__device__ __forceinline__ float over_448(float x) {
  const float q = x * (1.f / E4M3_MAX);
  return fmaf(fmaf(-E4M3_MAX, q, x), 1.f / E4M3_MAX, q);
}

// The block in 8 bits by exact roots and quotients; what is not finite is left out of the scale and held as NaN.
template <bool ROOT>
__device__ __forceinline__ float encode_exact(const f32x2* x, uint32_t* codes) {
  float y[8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 f = floats(x[i >> 1]);
    y[i] = i & 1 ? f.y : f.x;
    if (ROOT) y[i] = __fsqrt_rn(y[i]);
    const uint32_t b = __float_as_uint(y[i]) & 0x7FFFFFFFu;
    top = max(top, b < 0x7F800000u ? b : 0u);
  }
  const float scale = __fdiv_rn(__uint_as_float(__reduce_max_sync(0xffffffffu, top)), E4M3_MAX);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const bool finite = fabsf(y[i]) < INFINITY, some = y[i] > 0.f;
    y[i] = scale > 0.f ? __fdiv_rn(y[i], scale) : 0.f;
    if (ROOT && some) y[i] = fmaxf(y[i], E4M3_MIN);
    if (!finite) y[i] = NAN;
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) codes[h] = to_codes(pair(y[4 * h], y[4 * h + 1]), pair(y[4 * h + 2], y[4 * h + 3]));
  return scale;
}

// The same codes without a division or an exact root per element, which would be most of the kernel's instructions: `approx`
// (x, or its root within 2^-23) times the scale's reciprocal (within 2^-23) is within 2^-21 of the quotient with the two products'
// roundings.  Both ends of that interval are rounded to the type; where they agree, the quotient between them rounds to the same.  They do not in about one block of
// 100, or where the scale is no ordinary number: false, and the exact form above is due.
template <bool ROOT>
__device__ __forceinline__ bool encode(const f32x2* x, const f32x2* approx, float& scale, uint32_t* codes) {
  float top = warp_max(x);
  if (ROOT) top = __fsqrt_rn(top);
  scale = over_448(top);
  bool fine = scale > 1e-15f && scale < 1e30f;                         // (false for NaN, too)
  const float inv = approx_reciprocal(scale);
  constexpr float SLACK = 4.76837158203125e-7f;                        // 2^-21
  const float up = inv * (1.f + SLACK), down = inv * (1.f - SLACK);
  const f32x2 up2 = pair(up, up), down2 = pair(down, down);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t c = to_codes(mul2(approx[2 * h], up2), mul2(approx[2 * h + 1], up2));
    const uint32_t low = to_codes(mul2(approx[2 * h], down2), mul2(approx[2 * h + 1], down2));
    uint32_t differ = c ^ low;
    if (ROOT && ((low - 0x01010101u) & ~low & 0x80808080u)) {          // a zero among the codes
      differ = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 f = floats(x[2 * h + (i >> 1)]);
        const uint32_t up_code = (c >> (8 * i)) & 255u, low_code = (low >> (8 * i)) & 255u;
        if ((i & 1 ? f.y : f.x) > 0.f) {                               // lifted to the smallest number
          if (up_code == 0) c |= 1u << (8 * i);
          if (max(up_code, 1u) != max(low_code, 1u)) differ = 1;
        } else if (up_code != low_code) {
          differ = 1;
        }
      }
    }
    codes[h] = c;
    if (differ) fine = false;
  }
  return __all_sync(0xffffffffu, fine);
}

// ------------------------------------------------------------------------------------------------ the step
struct Rates {
  f32x2 grad, b1, c1, b2, c2, root, eps, step, one; // each twice
  float lr;
  bool exact_root;
};

// What a lane holds of a warp's block of 256: elements 4 l .. 4 l + 3 of either half.  There is a copy of the loop for each
// combination of types (TYPES: the bits of Tensor::flags that say which).
template <int BITS>
struct Raw {
  uint4 x[2], g[2];
  uint4 m[BITS == 32 ? 2 : 1], v[BITS == 32 ? 2 : 1];      // 8 bits: the codes of both halves in .x and .y
};

// Whole, aligned blocks come through shared memory, two of them on their way per warp without taking registers (holding even one
// block ahead in registers spilled, or left too few warps).  Bytes of a block: x and g 1 KB each (bf16: half of it used), the
// moments 1 KB or 256 bytes each.
constexpr int DEPTH = 3;
template <int BITS> constexpr int STAGE_BYTES = 2048 + 2 * (BITS == 32 ? 1024 : 256);

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); }

// A tensor's buffers; x: the weights that are read (the master, if there is one), p: where a master's rounding goes.
struct Place {
  const char* g;
  char *x, *p, *m, *v;
};

__host__ __device__ constexpr bool x_is_bf16(int flags) { return (flags & (P_BF16 | MASTERED)) == P_BF16; }

template <int BITS, int flags>
__device__ __forceinline__ void request(uint32_t stage, const Place& at, uint32_t block, int lane) {
  const uint32_t to = stage + 16 * lane;
  const uint64_t b16 = block * uint64_t(512) + 16 * lane, b32 = block * uint64_t(1024) + 16 * lane;
  if (flags & G_BF16) {
    copy16(to + 1024, at.g + b16);
  } else {
    copy16(to + 1024, at.g + b32); copy16(to + 1536, at.g + b32 + 512);
  }
  if (x_is_bf16(flags)) {
    copy16(to, at.x + b16);
  } else {
    copy16(to, at.x + b32); copy16(to + 512, at.x + b32 + 512);
  }
  if (BITS == 32) {
    copy16(to + 2048, at.m + b32); copy16(to + 2560, at.m + b32 + 512);
    copy16(to + 3 * 1024, at.v + b32); copy16(to + 3584, at.v + b32 + 512);
  } else {                             // the codes of m by the first 16 lanes, those of v by the others
    copy16(to + 2048, (lane < 16 ? at.m : at.v) + block * uint64_t(256) + 16 * (lane & 15));
  }
}

template <int BITS, int flags>
__device__ __forceinline__ void take(Raw<BITS>& r, const uint8_t* stage, int lane) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (flags & G_BF16) {
      const uint2 q = *reinterpret_cast<const uint2*>(stage + 1024 + 256 * h + 8 * lane);
      r.g[h] = make_uint4(q.x, q.y, 0, 0);
    } else {
      r.g[h] = *reinterpret_cast<const uint4*>(stage + 1024 + 512 * h + 16 * lane);
    }
    if (x_is_bf16(flags)) {
      const uint2 q = *reinterpret_cast<const uint2*>(stage + 256 * h + 8 * lane);
      r.x[h] = make_uint4(q.x, q.y, 0, 0);
    } else {
      r.x[h] = *reinterpret_cast<const uint4*>(stage + 512 * h + 16 * lane);
    }
    if (BITS == 32) {
      r.m[h] = *reinterpret_cast<const uint4*>(stage + 2048 + 512 * h + 16 * lane);
      r.v[h] = *reinterpret_cast<const uint4*>(stage + 3 * 1024 + 512 * h + 16 * lane);
    } else {
      (h ? r.m[0].y : r.m[0].x) = *reinterpret_cast<const uint32_t*>(stage + 2048 + 128 * h + 4 * lane);
      (h ? r.v[0].y : r.v[0].x) = *reinterpret_cast<const uint32_t*>(stage + 2304 + 128 * h + 4 * lane);
    }
  }
}

// A tensor's last block, or any of an unaligned tensor: element by element; `left`: elements from the lane's first one on.
__device__ __forceinline__ int present(int left) { return min(max(left, 0), 4); }

template <int BITS, int flags>
__device__ __forceinline__ void read_part(Raw<BITS>& r, const Place& at, uint32_t block, int left, int lane) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int n = present(left - 128 * h);
    const uint64_t e = block * uint64_t(BLOCK) + 128 * h + 4 * lane;
    r.g[h] = flags & G_BF16 ? read_bf16(at.g + 2 * e, n) : read_floats(at.g + 4 * e, n);
    r.x[h] = x_is_bf16(flags) ? read_bf16(at.x + 2 * e, n) : read_floats(at.x + 4 * e, n);
    if (BITS == 32) {
      r.m[h] = read_floats(at.m + 4 * e, n);
      r.v[h] = read_floats(at.v + 4 * e, n);
    } else {
      (h ? r.m[0].y : r.m[0].x) = read_codes(at.m + e, n);
      (h ? r.v[0].y : r.v[0].x) = read_codes(at.v + e, n);
    }
  }
}

template <int BITS, int flags>
__device__ __forceinline__ void update(const Raw<BITS>& raw, float& ms, float& vs, const Place& at, uint32_t block, int left,
                                       bool wide, float keep, int lane, const Rates& r) {
  f32x2 g[4], x[4], m[4], v[4], root[4];
  if (flags & G_BF16) { of_bf16(raw.g[0], g); of_bf16(raw.g[1], g + 2); }
  else { of_floats(raw.g[0], g); of_floats(raw.g[1], g + 2); }
  if (x_is_bf16(flags)) { of_bf16(raw.x[0], x); of_bf16(raw.x[1], x + 2); }
  else { of_floats(raw.x[0], x); of_floats(raw.x[1], x + 2); }
  if (BITS == 32) {
    of_floats(raw.m[0], m); of_floats(raw.m[BITS == 32 ? 1 : 0], m + 2);
    of_floats(raw.v[0], v); of_floats(raw.v[BITS == 32 ? 1 : 0], v + 2);
  } else {
    of_codes(raw.m[0].x, m); of_codes(raw.m[0].y, m + 2);
    of_codes(raw.v[0].x, v); of_codes(raw.v[0].y, v + 2);
  }
  const f32x2 ms2 = pair(ms, ms), vs2 = pair(vs, vs), keep2 = pair(keep, keep);
  // the moments: every product and sum rounded by itself, so that they are the formula's in plain float arithmetic, bit for bit, and
  // with them the 8-bit codes (one that falls on the other side of a middle is a sixteenth off).  The compiler joins a packed product and
  // a packed sum to a fused one; a sum as one * product + product, one known at run time only, it leaves alone.  The step taken from
  // the moments is good to a few units in its own last place.
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    g[i] = mul2(g[i], r.grad);
    if (BITS == 8) {
      m[i] = mul2(m[i], ms2);
      v[i] = mul2(v[i], vs2);
      v[i] = mul2(v[i], v[i]);
    }
    m[i] = fma2(mul2(m[i], r.b1), r.one, mul2(g[i], r.c1));
    v[i] = fma2(mul2(v[i], r.b2), r.one, mul2(mul2(g[i], g[i]), r.c2));
    const float2 vf = floats(v[i]);
    root[i] = pair(approx_root(vf.x), approx_root(vf.y));
  }
  if (r.exact_root) {                  // (approximate roots below 1e-19 are zero: that is seen next to a very small eps only)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 vf = floats(v[i]);
      root[i] = pair(__fsqrt_rn(vf.x), __fsqrt_rn(vf.y));
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 d = floats(fma2(root[i], r.root, r.eps));
    const f32x2 move = mul2(m[i], pair(approx_reciprocal(d.x), approx_reciprocal(d.y)));
    x[i] = fma2(move, r.step, mul2(x[i], keep2));
  }
  const uint64_t e = block * uint64_t(BLOCK) + 4 * lane;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int n = wide ? WHOLE : present(left - 128 * h);
    if (flags & P_BF16) write_bf16(at.p + 2 * e + 256 * h, n, x + 2 * h);
    if (!x_is_bf16(flags)) write_floats(at.x + 4 * e + 512 * h, n, x + 2 * h);
    if (BITS == 32) {
      write_floats(at.m + 4 * e + 512 * h, n, m + 2 * h);
      write_floats(at.v + 4 * e + 512 * h, n, v + 2 * h);
    }
  }
  if (BITS == 8) {
    uint32_t cm[2], cv[2];
    if (!encode<false>(m, m, ms, cm)) ms = encode_exact<false>(m, cm);
    if (!encode<true>(v, root, vs, cv)) vs = encode_exact<true>(v, cv);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int n = wide ? WHOLE : present(left - 128 * h);
      write_codes(at.m + e + 128 * h, n, cm[h]);
      write_codes(at.v + e + 128 * h, n, cv[h]);
    }
  }
}

static_assert(DEPTH == 3, "the loop below keeps two requests ahead");
template <int BITS> constexpr int RESIDENT = BITS == 32 ? 2 : 3;

// The chunks c0, c0 + WARPS, .. < stop of one tensor; a chunk is 2^lg consecutive blocks and one warp's.  Returns how many blocks it had.
// The scales of a chunk of eight are two accesses of 32 bytes (single words, a read and a write for each block, cost 30 us of 145 on
// 48 M elements); short lists have chunks of one block, for the sake of more warps.
template <int BITS, int flags>
__device__ __forceinline__ uint32_t share(const Tensor& w, uint32_t c0, uint32_t stop, int lg, const uint8_t* my, int lane, const Rates& rates) {
  constexpr int STAGE = STAGE_BYTES<BITS>;
  const uint32_t mask = (1u << lg) - 1u, slots = smem_u32(my);
  const Place at{static_cast<const char*>(w.g), static_cast<char*>(flags & MASTERED ? w.master : w.p), static_cast<char*>(w.p),
                 static_cast<char*>(w.m), static_cast<char*>(w.v)};
  const uint32_t blocks = static_cast<uint32_t>((w.n - 1) / BLOCK + 1), whole = w.flags & WIDE ? static_cast<uint32_t>(w.n / BLOCK) : 0u;
  const float keep = __fsub_rn(1.f, __fmul_rn(rates.lr, w.decay));
  // block i of this warp's share of the tensor; beyond `stop` chunks or `blocks` there is none
  const auto block_at = [&](uint32_t i) { return ((c0 + (i >> lg) * WARPS) << lg) + (i & mask); };
  const auto there = [&](uint32_t i, uint32_t b) { return c0 + (i >> lg) * WARPS < stop && b < blocks; };
  // a chunk's scales: those of m in lanes 0 .. 7, those of v in lanes 8 .. 15
  float* const scale_at = BITS == 8 ? (lane & 8 ? w.vs : w.ms) + (lane & 7) : nullptr;
  const auto mine = [&](uint32_t b) { return lane < 16 && static_cast<uint32_t>(lane & 7) <= mask && b + (lane & 7) < blocks; };
  float scales = 0.f, scales_ahead = 0.f;
  if (BITS == 8 && mine(c0 << lg)) scales_ahead = scale_at[c0 << lg];
#pragma unroll
  for (uint32_t i = 0; i < 2; ++i) {
    const uint32_t b = block_at(i);
    if (there(i, b) && b < whole) request<BITS, flags>(slots + i * STAGE, at, b, lane);
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  uint32_t slot = 0, i = 0;
  for (uint32_t b = block_at(0); there(i, b); b = block_at(++i)) {
    if (BITS == 8 && (i & mask) == 0) {
      scales = scales_ahead;
      const uint32_t next = block_at(i + mask + 1);
      if (there(i + mask + 1, next) && mine(next)) scales_ahead = scale_at[next];
    }
    asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 2) : "memory");
    __syncwarp();
    Raw<BITS> raw;
    const bool wide = b < whole;
    const int left = wide ? BLOCK : static_cast<int>(min(w.n - static_cast<int64_t>(b) * BLOCK, static_cast<int64_t>(BLOCK))) - 4 * lane;
    if (wide) take<BITS, flags>(raw, my + slot * STAGE, lane);
    else read_part<BITS, flags>(raw, at, b, left, lane);
    const uint32_t ahead = block_at(i + 2);
    __syncwarp();                    // every lane has read the slot that is written next (one step ago)
    if (there(i + 2, ahead) && ahead < whole) request<BITS, flags>(slots + (slot == 0 ? DEPTH - 1 : slot - 1) * STAGE, at, ahead, lane);
    asm volatile("cp.async.commit_group;" ::: "memory");
    const int k = i & mask;
    float ms = 0.f, vs = 0.f;
    if (BITS == 8) { ms = __shfl_sync(0xffffffffu, scales, k); vs = __shfl_sync(0xffffffffu, scales, 8 + k); }
    update<BITS, flags>(raw, ms, vs, at, b, left, wide, keep, lane, rates);
    if (BITS == 8) {
      if (lane == k) scales = ms;
      if (lane == 8 + k) scales = vs;
      if (static_cast<uint32_t>(k) == mask || b + 1 == blocks) {
        if (mine(b - k)) scale_at[b - k] = scales;
      }
    }
    if (++slot == DEPTH) slot = 0;
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  return i;
}

// first: the chunks of the tensors before each one.
template <int BITS>
__global__ void __launch_bounds__(THREADS, RESIDENT<BITS>)
adamw_kernel(const Tensor* __restrict__ tensors, const int* __restrict__ first, int count, int total, int lg, Clock* clock, double b1,
             double b2, float eps, double lr, float grad_scale, float one) {
  extern __shared__ __align__(128) uint8_t memory[];
  __shared__ Rates rates;
  const int lane = threadIdx.x & 31;
  const uint8_t* my = memory + (threadIdx.x >> 5) * DEPTH * STAGE_BYTES<BITS>;
  const int lo = static_cast<int>(static_cast<long long>(blockIdx.x) * total / gridDim.x);
  const int hi = static_cast<int>(static_cast<long long>(blockIdx.x + 1) * total / gridDim.x);
  int c = lo + (threadIdx.x >> 5);     // this warp's next chunk
  if (threadIdx.x == 0) {
    const double p1 = clock->b1_t * b1, p2 = clock->b2_t * b2;
    const auto both = [](double x) { return pair(static_cast<float>(x), static_cast<float>(x)); };
    rates = Rates{both(grad_scale), both(b1), both(1.0 - b1), both(b2), both(1.0 - b2), both(1.0 / sqrt(1.0 - p2)), both(eps),
                  both(-lr / (1.0 - p1)), both(one), static_cast<float>(lr), eps < 1e-12f};
  }
  // the tensor of chunk c: the last one that starts at or before it; every lane looks at a 32nd of what is left
  int t = 0;
  for (int left = count; left > 1;) {
    const int part = (left + 31) / 32, i = t + lane * part;
    const bool before = lane * part < left && first[i] <= c;
    const int last = 31 - __clz(__ballot_sync(0xffffffffu, before) | 1u);
    t += last * part;
    left = min(part, left - last * part);
  }
  __syncthreads();
  while (c < hi) {
    const int start = first[t], end = min(first[t + 1], hi);
    if (c >= end) { ++t; continue; }
    const Tensor w = tensors[t];
    const uint32_t c0 = c - start, stop = end - start;
    uint32_t blocks;
    switch (w.flags & (P_BF16 | G_BF16 | MASTERED)) {
      case 0: blocks = share<BITS, 0>(w, c0, stop, lg, my, lane, rates); break;
      case G_BF16: blocks = share<BITS, G_BF16>(w, c0, stop, lg, my, lane, rates); break;
      case P_BF16: blocks = share<BITS, P_BF16>(w, c0, stop, lg, my, lane, rates); break;
      case P_BF16 | G_BF16: blocks = share<BITS, P_BF16 | G_BF16>(w, c0, stop, lg, my, lane, rates); break;
      case P_BF16 | MASTERED: blocks = share<BITS, P_BF16 | MASTERED>(w, c0, stop, lg, my, lane, rates); break;
      default: blocks = share<BITS, P_BF16 | G_BF16 | MASTERED>(w, c0, stop, lg, my, lane, rates); break;
    }
    c += ((blocks + (1u << lg) - 1u) >> lg) * WARPS;       // (the first chunk of this warp's at or behind `end`)
    ++t;
  }
  // the block that comes here last moves the clock on: every other one has read it long ago
  if (threadIdx.x == 0) {
    __threadfence();
    if (atomicAdd(&clock->seen, 1u) == gridDim.x - 1) {
      clock->b1_t *= b1; clock->b2_t *= b2; clock->t += 1;
      clock->seen = 0;
    }
  }
}

template <int BITS> constexpr int smem_bytes() { return THREADS / 32 * DEPTH * STAGE_BYTES<BITS>; }

// The opt-in to more than 48 KB of shared memory (per device), and how many thread blocks an SM then holds.
template <int BITS>
cudaError_t ready(int* resident) {
  const cudaError_t e = cudaFuncSetAttribute(adamw_kernel<BITS>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes<BITS>());
  return e != cudaSuccess ? e : cudaOccupancyMaxActiveBlocksPerMultiprocessor(resident, adamw_kernel<BITS>, THREADS, smem_bytes<BITS>());
}

// The list's device as the current one, for the calls that wait for it or reach its memory; then the caller's again.
class OnDevice {
 public:
  explicit OnDevice(int dev) : ok_(cudaGetDevice(&before_) == cudaSuccess && (before_ == dev || cudaSetDevice(dev) == cudaSuccess)), back_(ok_ && before_ != dev) {}
  ~OnDevice() { if (back_) (void)cudaSetDevice(before_); }
  OnDevice(const OnDevice&) = delete;
  OnDevice& operator=(const OnDevice&) = delete;
  explicit operator bool() const { return ok_; }

 private:
  int before_ = 0;
  bool ok_, back_;
};

}  // namespace
}  // namespace mbd

using namespace mbd;

struct mbd_adamw {
  int dev = 0, grid = 0, count = 0, total = 0, lg = 0, bits = 32;
  double b1 = 0, b2 = 0;
  float eps = 0;
  char* block = nullptr;               // Clock, Tensor[count], int[count + 1]
  Clock* clock = nullptr;
  Tensor* tensors = nullptr;
  int* first = nullptr;
};

extern "C" mbd_status mbd_adamw_create(const mbd_adamw_tensor* tensors_host, int count, int state_bits, double beta1, double beta2, double eps,
                                       int64_t steps_done, mbd_adamw** out) {
  if (!tensors_host || !out || count < 1 || steps_done < 0 || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) ||
      !(eps >= 1e-30 && eps < 1.0)) return MBD_E_INVALID;
  if (state_bits != 32 && state_bits != 8) return MBD_E_UNSUPPORTED;
  struct Span { uintptr_t a, b; bool written; };
  try {
    std::vector<Tensor> table(count);
    std::vector<int> first(count + 1);
    std::vector<Span> spans;
    int64_t total = 0;
    for (int i = 0; i < count; ++i) {
      const mbd_adamw_tensor& t = tensors_host[i];
      if (t.n < 1 || !t.param_dev || !t.grad_dev || !t.m_dev || !t.v_dev || !(t.weight_decay >= 0.f && t.weight_decay < INFINITY)) return MBD_E_INVALID;
      if (t.master_dev && !t.param_bf16) return MBD_E_INVALID;             // float weights are their own master
      if (state_bits == 8 && (!t.m_scale_dev || !t.v_scale_dev)) return MBD_E_INVALID;
      const int64_t blocks = (t.n - 1) / BLOCK + 1;
      first[i] = static_cast<int>(total);
      if (t.n > (int64_t(1) << 46) || (total += blocks) > (1 << 30)) return MBD_E_UNSUPPORTED;
      const int64_t psize = t.param_bf16 ? 2 : 4, gsize = t.grad_bf16 ? 2 : 4, ssize = state_bits == 32 ? 4 : 1;
      const auto at = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
      if (at(t.param_dev) % psize || at(t.grad_dev) % gsize || at(t.m_dev) % ssize || at(t.v_dev) % ssize || at(t.master_dev) % 4 ||
          at(t.m_scale_dev) % 4 || at(t.v_scale_dev) % 4) return MBD_E_UNSUPPORTED;
      const auto span = [&](const void* p, int64_t bytes, bool written) { if (p) spans.push_back({at(p), at(p) + static_cast<uintptr_t>(bytes), written}); };
      span(t.param_dev, t.n * psize, true);
      span(t.master_dev, t.n * 4, true);
      span(t.grad_dev, t.n * gsize, false);
      span(t.m_dev, t.n * ssize, true);
      span(t.v_dev, t.n * ssize, true);
      if (state_bits == 8) { span(t.m_scale_dev, blocks * 4, true); span(t.v_scale_dev, blocks * 4, true); }
      Tensor& d = table[i];
      d.p = t.param_dev; d.master = t.master_dev; d.g = t.grad_dev; d.m = t.m_dev; d.v = t.v_dev;
      d.ms = state_bits == 8 ? t.m_scale_dev : nullptr;
      d.vs = state_bits == 8 ? t.v_scale_dev : nullptr;
      d.n = t.n;
      d.decay = t.weight_decay;
      const bool wide = (at(t.param_dev) | at(t.master_dev) | at(t.grad_dev) | at(t.m_dev) | at(t.v_dev)) % 16 == 0;
      d.flags = (t.param_bf16 ? P_BF16 : 0) | (t.grad_bf16 ? G_BF16 : 0) | (t.master_dev ? MASTERED : 0) | (wide ? WIDE : 0);
    }
    first[count] = static_cast<int>(total);
    // a buffer that is written may be named once: two entries on it would race
    std::sort(spans.begin(), spans.end(), [](const Span& x, const Span& y) { return x.a < y.a; });
    uintptr_t end = 0, end_written = 0;
    for (const Span& s : spans) {
      if (s.a < end_written || (s.written && s.a < end)) return MBD_E_INVALID;
      end = std::max(end, s.b);
      if (s.written) end_written = std::max(end_written, s.b);
    }
    mbd_adamw* h = new (std::nothrow) mbd_adamw;
    if (!h) return MBD_E_ALLOC;
    h->count = count; h->bits = state_bits;
    h->b1 = beta1; h->b2 = beta2; h->eps = static_cast<float>(eps);
    const size_t bytes = 64 + sizeof(Tensor) * count + sizeof(int) * (count + 1);
    mbd_status st = MBD_OK;
    int sms = 0, resident = 0;
    if (cudaGetDevice(&h->dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, h->dev) != cudaSuccess ||
        (state_bits == 32 ? ready<32>(&resident) : ready<8>(&resident)) != cudaSuccess) st = MBD_E_CUDA;
    else if (cudaMalloc(reinterpret_cast<void**>(&h->block), bytes) != cudaSuccess) { h->block = nullptr; st = MBD_E_ALLOC; }
    if (st == MBD_OK) {
      // one wave: every thread block takes its share of the list
      const int64_t warps = THREADS / 32, most = static_cast<int64_t>(sms) * std::max(resident, 1);
      h->lg = total >= 8 * 4 * most * warps ? 3 : 0;                      // (chunks of eight where every warp has a few of them)
      int64_t chunks = 0;
      for (int i = 0; i < count; ++i) {
        const int64_t blocks = first[i + 1] - first[i];
        first[i] = static_cast<int>(chunks);
        chunks += (blocks + (1 << h->lg) - 1) >> h->lg;
      }
      first[count] = h->total = static_cast<int>(chunks);
      h->grid = static_cast<int>(std::min((chunks + warps - 1) / warps, most));
      h->clock = reinterpret_cast<Clock*>(h->block);
      h->tensors = reinterpret_cast<Tensor*>(h->block + 64);
      h->first = reinterpret_cast<int*>(h->block + 64 + sizeof(Tensor) * count);
      if (cudaMemcpy(h->tensors, table.data(), sizeof(Tensor) * count, cudaMemcpyHostToDevice) != cudaSuccess ||
          cudaMemcpy(h->first, first.data(), sizeof(int) * (count + 1), cudaMemcpyHostToDevice) != cudaSuccess) st = MBD_E_CUDA;
      else st = mbd_adamw_set_steps(h, steps_done);
    }
    if (st != MBD_OK) {
      (void)cudaGetLastError();
      if (h->block) cudaFree(h->block);
      delete h;
      return st;
    }
    *out = h;
    return MBD_OK;
  } catch (...) {                      // out of host memory
    return MBD_E_ALLOC;
  }
}

extern "C" mbd_status mbd_adamw_destroy(mbd_adamw* opt) {
  if (!opt) return MBD_E_INVALID;
  if (opt->block) cudaFree(opt->block);
  delete opt;
  return MBD_OK;
}

extern "C" mbd_status mbd_adamw_set_steps(mbd_adamw* opt, int64_t steps_done) {
  if (!opt || steps_done < 0) return MBD_E_INVALID;
  Clock c{};
  c.b1_t = pow(opt->b1, static_cast<double>(steps_done));
  c.b2_t = pow(opt->b2, static_cast<double>(steps_done));
  c.t = steps_done;
  // (the second wait is for the copy itself, and for those of a new list: from pageable memory it may return before it has landed, and
  // the next step's stream need not wait for it)
  const OnDevice on(opt->dev);
  if (!on || cudaDeviceSynchronize() != cudaSuccess || cudaMemcpy(opt->clock, &c, sizeof(c), cudaMemcpyHostToDevice) != cudaSuccess ||
      cudaDeviceSynchronize() != cudaSuccess) { (void)cudaGetLastError(); return MBD_E_CUDA; }
  return MBD_OK;
}

extern "C" mbd_status mbd_adamw_get_steps(mbd_adamw* opt, int64_t* steps_done_host) {
  if (!opt || !steps_done_host) return MBD_E_INVALID;
  Clock c{};
  const OnDevice on(opt->dev);
  if (!on || cudaDeviceSynchronize() != cudaSuccess || cudaMemcpy(&c, opt->clock, sizeof(c), cudaMemcpyDeviceToHost) != cudaSuccess) { (void)cudaGetLastError(); return MBD_E_CUDA; }
  *steps_done_host = c.t;
  return MBD_OK;
}

extern "C" mbd_status mbd_adamw_step(mbd_adamw* opt, double lr, double grad_scale, void* cuda_stream) {
  if (!opt || !(lr >= 0.0 && lr < 1e30) || !(fabs(grad_scale) < 1e30)) return MBD_E_INVALID;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { (void)cudaGetLastError(); return MBD_E_CUDA; }
  if (dev != opt->dev) return MBD_E_STATE;                     // the list's device has to be the current one
  const dim3 grid(static_cast<unsigned>(opt->grid)), block(THREADS);
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = opt->bits == 32
      ? launch_pdl(adamw_kernel<32>, grid, block, smem_bytes<32>(), stream, 0, static_cast<const Tensor*>(opt->tensors), static_cast<const int*>(opt->first), opt->count, opt->total, opt->lg, opt->clock, opt->b1, opt->b2, opt->eps, lr, static_cast<float>(grad_scale), 1.f)
      : launch_pdl(adamw_kernel<8>, grid, block, smem_bytes<8>(), stream, 0, static_cast<const Tensor*>(opt->tensors), static_cast<const int*>(opt->first), opt->count, opt->total, opt->lg, opt->clock, opt->b1, opt->b2, opt->eps, lr, static_cast<float>(grad_scale), 1.f);
  if (e != cudaSuccess) { (void)cudaGetLastError(); return MBD_E_CUDA; }
  return MBD_OK;
}
