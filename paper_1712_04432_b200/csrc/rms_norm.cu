// Root-mean-square norm of rows, with the residual's addition in front and rows in 16, 32 or 8 bits behind, and its gradients.
//
//   h = x (+ residual, rounded to the residual's type),  r = 1 / sqrt(mean(h^2) + eps),  y = h r g
//   in 8 bits: u = h g in float, s = max |u| / 127, q = u / s rounded to an integer, scale = s r.  r is the same for all of a row, so it goes
//   into the scale: q needs the row's largest |u| only and does not depend on the order in which the squares are added.
//   backward: m = mean(dy g h r),  dh = r (dy g - h r m) (+ the gradient that arrives along the residual),  dg = sum over rows of dy h r
//
// Each tensor passes once: the row stays in registers between the sum and the result, the gain and the columns' sums of dg
// in the registers of the threads that own the columns (blocks take row after row).  HBM bounds large calls, latency small ones.
// Where blocks keep something from row to row, rows come through shared memory by asynchronous copies some rows ahead: a warp waits for
// its own copies only, and how much is under way does not depend on registers.
#include <math_constants.h>

#include <atomic>

#include "../../include/mbd.h"
#include "quotients.cuh"
#include "vec8.cuh"

namespace mbd {
namespace {

struct Norm {
  const void *x, *res;
  const float* gain;
  void *h, *y;
  int8_t* q;
  float* scale;
  int64_t ldx, ldres, ldh, ldy, ldq, R;
  float eps;
  int K, y_bf16, n, stages;              // n: threads per row, a power of 2
};

// Squares beyond float's range (|h| above 1e19 / sqrt(K)) are added up again with the row taken 2^-80 times as large.
constexpr float SMALLER = 8.271806125530277e-25f;   // 2^-80

// 1 / sqrt(sum / K + eps): the approximation and one step of Newton's method, about an ulp.
__device__ __forceinline__ float root(float sum, float inv_K, float eps) {
  const float x = fmaf(sum, inv_K, eps), r = rsqrtf(x);
  if (!(x < 1e38f)) return r;                             // (infinite, or next to it, or NaN)
  return fmaf(0.5f * r, fmaf(-x * r, r, 1.f), r);
}

// Sums and maxima over the n threads of a row; everybody gets them.  A row has a warp, or whole warps that meet at a barrier of
// their own; `turn` alternates so that one barrier per exchange is enough.
struct Exchange { float a[2][32], b[2][32]; uint32_t m[2][32]; };
template <bool B, bool M>
__device__ __forceinline__ void over_row(Exchange& e, int& turn, int n, float& a, float& b, uint32_t& m) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    a += __shfl_xor_sync(0xffffffffu, a, d);
    if (B) b += __shfl_xor_sync(0xffffffffu, b, d);
  }
  if (M) m = __reduce_max_sync(0xffffffffu, m);
  if (n <= 32) return;
  const int w = threadIdx.x >> 5, l = threadIdx.x & 31, warps = n >> 5, row = threadIdx.x / n, first = row * warps;
  if (l == 0) {
    e.a[turn][w] = a;
    if (B) e.b[turn][w] = b;
    if (M) e.m[turn][w] = m;
  }
  asm volatile("bar.sync %0, %1;" :: "r"(1 + row), "r"(n) : "memory");
  a = l < warps ? e.a[turn][first + l] : 0.f;
  if (B) b = l < warps ? e.b[turn][first + l] : 0.f;
  if (M) m = __reduce_max_sync(0xffffffffu, l < warps ? e.m[turn][first + l] : 0u);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    a += __shfl_xor_sync(0xffffffffu, a, d);
    if (B) b += __shfl_xor_sync(0xffffffffu, b, d);
  }
  turn ^= 1;
}

// ---- rows on their way through shared memory: each warp of a row copies its own columns and reads them back.
// WIDE: in pieces of 16 bytes; else (floats) of 4.  Columns behind the row's end are zero from the start and are not copied.
__device__ __forceinline__ void copies_sent() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copies_landed(int ahead) {            // all but the last `ahead` rows' copies of this thread
  if (ahead == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
  else if (ahead == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
  else asm volatile("cp.async.wait_group 3;" ::: "memory");
}
constexpr int MOST_STAGES = 4;
constexpr int FORWARD_THREADS = 768, BACKWARD_THREADS = 512;   // of a block that takes many rows

// Eight floats are two pieces of 16 bytes side by side: a thread that copied both would ask for each 32-byte sector twice (8192 x 2048 floats backward
// 73 instead of 48 us), so the lanes of a warp copy the warp's 1024 bytes in order and read the pieces that others brought; every second
// group of eight pieces is swapped in pairs, which keeps the reads apart in the banks.
__device__ __forceinline__ uint32_t piece_at(int p) { return (p ^ (p >> 3 & 1)) * 16; }

template <int N, int NV, bool WIDE, typename T>
__device__ __forceinline__ void send_row(uint32_t buffer, const T* row, int t, int K) {
  if constexpr (WIDE && sizeof(T) == 4) {
    const int lane = t & 31, first = t & ~31;
    const T* from = row + 8 * first + 4 * lane;
    const uint32_t to = buffer + first * 32 + piece_at(lane);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (8 * (first + j * N) + 128 * h + 4 * lane < K)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to + j * N * 32 + h * 512), "l"(from + 8 * j * N + 128 * h) : "memory");
  } else {
    constexpr int UNIT = WIDE ? 16 : 4, PIECES = WIDE ? 1 : 8;
    const uint32_t to = buffer + t * UNIT;
    const T* from = row + column<WIDE>(t, 0, N, 0);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int h = 0; h < PIECES; ++h)
        if (column<WIDE>(t, j, N, 0) + (WIDE ? 0 : h * N) < K) {
          const T* at = from + (WIDE ? 8 * j * N : (8 * j + h) * N);
          if (WIDE) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to + j * N * UNIT), "l"(at) : "memory");
          else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" :: "r"(to + (j * PIECES + h) * N * UNIT), "l"(at) : "memory");
        }
  }
}
// Address of value i of vector j of thread t (i: the first of a piece).
template <int N, bool WIDE, typename T> __device__ __forceinline__ uint32_t value_at(uint32_t buffer, int t, int j, int i) {
  if (WIDE && sizeof(T) == 4) return buffer + ((t & ~31) + j * N) * 32 + piece_at(2 * (t & 31) + (i >> 2)) + (i & 3) * 4;
  if (WIDE) return buffer + (j * N + t) * 16 + i * 2;
  return buffer + ((8 * j + i) * N + t) * 4;
}
// (volatile, as the gain below: what is read twice is not held in registers between)
template <int N, bool WIDE> __device__ __forceinline__ void take8(uint32_t buffer, int t, int j, Raw8<__nv_bfloat16>& r) {
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]) : "r"(value_at<N, WIDE, __nv_bfloat16>(buffer, t, j, 0)));
}
template <int N, bool WIDE> __device__ __forceinline__ void take8(uint32_t buffer, int t, int j, Raw8<float>& r) {
  if (WIDE) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                   : "=f"(r.f[4 * h]), "=f"(r.f[4 * h + 1]), "=f"(r.f[4 * h + 2]), "=f"(r.f[4 * h + 3]) : "r"(value_at<N, true, float>(buffer, t, j, 4 * h)));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) asm volatile("ld.shared.f32 %0, [%1];" : "=f"(r.f[i]) : "r"(value_at<N, false, float>(buffer, t, j, i)));
  }
}
// Eight values back into their places.
template <int N, bool WIDE> __device__ __forceinline__ void put8(uint32_t buffer, int t, int j, const Raw8<__nv_bfloat16>& r) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" :: "r"(value_at<N, WIDE, __nv_bfloat16>(buffer, t, j, 0)), "r"(r.w[0]), "r"(r.w[1]), "r"(r.w[2]), "r"(r.w[3]) : "memory");
}
template <int N, bool WIDE> __device__ __forceinline__ void put8(uint32_t buffer, int t, int j, const Raw8<float>& r) {
#pragma unroll
  for (int i = 0; i < 8; ++i) asm volatile("st.shared.f32 [%0], %1;" :: "r"(value_at<N, WIDE, float>(buffer, t, j, i)), "f"(r.f[i]) : "memory");
}

// Zeros where this thread's columns lie behind the row's end.
template <int N, int NV, bool WIDE, typename T> __device__ __forceinline__ void clear_row(uint32_t buffer, int t, int K) {
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < 8; i += 4 / static_cast<int>(sizeof(T)))
      if (column<WIDE>(t, j, N, i) >= K) asm volatile("st.shared.b32 [%0], %1;" :: "r"(value_at<N, WIDE, T>(buffer, t, j, i)), "r"(0) : "memory");
}

// The gain in shared memory, in the order in which the threads of a row read it.
template <int N, int NV, bool WIDE>
__device__ __forceinline__ void keep_gain(float* kept, const float* gain, int K) {
  for (int c = threadIdx.x; c < NV * 8 * N; c += blockDim.x) {
    const int j = c / (8 * N), rest = c - j * 8 * N;
    const int at = WIDE ? (((2 * j + (rest >> 2 & 1)) * N + (rest >> 3)) * 4 + (rest & 3)) : c;
    kept[at] = c < K ? (gain ? gain[c] : 1.f) : 0.f;
  }
}
// (volatile: it is read anew for each row, not held in registers)
template <int N, bool WIDE> __device__ __forceinline__ void kept_gain(const float* kept, int t, int j, f32x2* g) {
  const uint32_t at = static_cast<uint32_t>(__cvta_generic_to_shared(kept)) + (WIDE ? (2 * j * N + t) * 16 : (t + 8 * j * N) * 4);
  if (WIDE) {
#pragma unroll
    for (int h = 0; h < 2; ++h) asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(g[2 * h]), "=l"(g[2 * h + 1]) : "r"(at + h * N * 16));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a, b;
      asm volatile("ld.shared.f32 %0, [%1];" : "=f"(a) : "r"(at + 2 * i * N * 4));
      asm volatile("ld.shared.f32 %0, [%1];" : "=f"(b) : "r"(at + (2 * i + 1) * N * 4));
      g[i] = pair(a, b);
    }
  }
}
__device__ __forceinline__ float both(f32x2 x) {
  const float2 v = floats(x);
  return v.x + v.y;
}

template <bool WIDE>
__device__ __forceinline__ void gain8(const float* gain, int t, int j, int n, int K, f32x2* g) {
  float v[8];
  if (WIDE && gain && (reinterpret_cast<uintptr_t>(gain) & 15u) == 0) {
    const int c = column<true>(t, j, n, 0);
    const float4 a = c < K ? *reinterpret_cast<const float4*>(gain + c) : make_float4(0.f, 0.f, 0.f, 0.f);
    const float4 b = c < K ? *reinterpret_cast<const float4*>(gain + c + 4) : make_float4(0.f, 0.f, 0.f, 0.f);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = column<WIDE>(t, j, n, i);
      v[i] = c >= K ? 0.f : gain ? gain[c] : 1.f;
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) g[i] = pair(v[2 * i], v[2 * i + 1]);
}

// h of one vector, from what was loaded; with a residual it is rounded to the residual's type.
template <typename TX, typename TR, bool RES>
__device__ __forceinline__ Raw8<TR> stream8(const Raw8<TX>& x, const Raw8<TR>& res) {
  Raw8<TR> h;
  float v[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = floats(RES ? add2(x.two(i), res.two(i)) : x.two(i));
    v[2 * i] = f.x;
    v[2 * i + 1] = f.y;
  }
  h.set(v);
  return h;
}

// One vector of the result in 16 or 32 bits, and in 8.
template <bool WIDE, typename TY, typename TR>
__device__ __forceinline__ void result8(TY* y, int t, int j, int n, int K, const Raw8<TR>& h, const f32x2* g, f32x2 inv2) {
  float v[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = floats(mul2(mul2(h.two(i), inv2), g[i]));
    v[2 * i] = f.x;
    v[2 * i + 1] = f.y;
  }
  Raw8<TY> o;
  o.set(v);
  store8<WIDE>(y, t, j, n, K, o);
}
template <bool WIDE, typename TR>
__device__ __forceinline__ void bytes8(int8_t* q, int t, int j, int n, int K, const Raw8<TR>& h, const f32x2* g, const Scale& c) {
  f32x2 u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) u[i] = mul2(h.two(i), g[i]);
  const uint2 w = quotients(u, c.s, c.inv, c.tiny);
  if (WIDE) {
    if (column<true>(t, j, n, 0) < K) *reinterpret_cast<uint2*>(q + column<true>(t, j, n, 0)) = w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int k = column<false>(t, j, n, i);
      if (k < K) q[k] = static_cast<int8_t>((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
    }
  }
}
// NV vectors of all results of row r; gain(j, g): the gain of vector j.
template <int NV, bool WIDE, typename TR, typename G>
__device__ __forceinline__ void results(const Norm& p, int64_t r, int t, int n, const Raw8<TR>* h, float inv, const Scale& c, G&& gain) {
  const f32x2 inv2 = pair(inv, inv);
  if (p.y && p.y_bf16) {
    __nv_bfloat16* y = static_cast<__nv_bfloat16*>(p.y) + r * p.ldy;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      f32x2 g[4];
      gain(j, g);
      result8<WIDE>(y, t, j, n, p.K, h[j], g, inv2);
    }
  } else if (p.y) {
    float* y = static_cast<float*>(p.y) + r * p.ldy;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      f32x2 g[4];
      gain(j, g);
      result8<WIDE>(y, t, j, n, p.K, h[j], g, inv2);
    }
  }
  if (p.q) {
    int8_t* q = p.q + r * p.ldq;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      f32x2 g[4];
      gain(j, g);
      bytes8<WIDE>(q, t, j, n, p.K, h[j], g, c);
    }
  }
}
// The largest |h g| so far, by its bits (their order is that of the magnitudes, infinities and NaN last).
template <typename TR> __device__ __forceinline__ uint32_t largest8(const Raw8<TR>& h, const f32x2* g, uint32_t so_far) {
  float top = __uint_as_float(so_far);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 u = floats(mul2(h.two(i), g[i]));
    asm("max.NaN.abs.f32 %0, %0, %1, %2;" : "+f"(top) : "f"(u.x), "f"(u.y));
  }
  return __float_as_uint(top) & 0x7FFFFFFFu;
}
template <typename TR> __device__ __forceinline__ Raw8<TR> smaller8(const Raw8<TR>& h) {
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = h.at(i) * SMALLER;
  Raw8<TR> r;
  r.set(v);
  return r;
}

// A few rows: one per block, a vector a thread (16 x 1024 bf16 to 8 bits, with residual: 2.0 us, one round trip and a barrier).
template <typename TX, typename TR, bool RES, bool WIDE>
__global__ void __launch_bounds__(1024) rms_norm_few_kernel(const __grid_constant__ Norm p) {
  __shared__ Exchange ex;
  const int n = p.n, t = threadIdx.x;
  const int64_t r = blockIdx.x;
  int turn = 0;
  pdl_trigger();
  pdl_wait();
  Raw8<TX> x;
  Raw8<TR> res;
  load8<WIDE>(static_cast<const TX*>(p.x) + r * p.ldx, t, 0, n, p.K, x);
  if (RES) load8<WIDE>(static_cast<const TR*>(p.res) + r * p.ldres, t, 0, n, p.K, res);
  f32x2 g[4];
  gain8<WIDE>(p.gain, t, 0, n, p.K, g);
  const Raw8<TR> h = stream8<TX, TR, RES>(x, res);
  f32x2 sum2 = pair(0.f, 0.f);
#pragma unroll
  for (int i = 0; i < 4; ++i) sum2 = fma2(h.two(i), h.two(i), sum2);
  float sum = both(sum2), none = 0.f;
  uint32_t top = p.q ? largest8(h, g, 0u) : 0u;
  over_row<false, true>(ex, turn, n, sum, none, top);
  if (RES && p.h) store8<WIDE>(static_cast<TR*>(p.h) + r * p.ldh, t, 0, n, p.K, h);
  float inv = root(sum, __fdiv_rn(1.f, static_cast<float>(p.K)), p.eps);
  if (sum == CUDART_INF_F) {
    const Raw8<TR> z = smaller8(h);
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = fmaf(z.at(i), z.at(i), sum);
    uint32_t unused = 0;
    over_row<false, false>(ex, turn, n, sum, none, unused);
    inv = root(sum, __fdiv_rn(1.f, static_cast<float>(p.K)), 0.f) * SMALLER;
  }
  Scale c{};
  if (p.q) c = scale_of(top);
  results<1, WIDE>(p, r, t, n, &h, inv, c, [&](int, f32x2* to) {
#pragma unroll
    for (int i = 0; i < 4; ++i) to[i] = g[i];
  });
  if (p.q && t == 0) p.scale[r] = c.s * inv;
}

// More rows, N threads and NV vectors each, 128 threads a block at least: nothing is held from one row to the next, the rows of other blocks hide
// the wait for a row.  HBM bounds it (8192 x 4096 bf16 with residual 43 us, 6.2 TB/s; torch copies
// such tensors at 6.0 and adds them at 6.7).
template <typename TX, typename TR, bool RES, int N, int NV, bool WIDE>
__global__ void __launch_bounds__(N < 128 ? 128 : N) rms_norm_direct_kernel(const __grid_constant__ Norm p) {
  __shared__ Exchange ex;
  const int t = threadIdx.x & (N - 1);
  const int64_t r = blockIdx.x * static_cast<int64_t>(blockDim.x / N) + threadIdx.x / N;
  int turn = 0;
  pdl_trigger();
  pdl_wait();
  if (r >= p.R) return;
  Raw8<TX> x[NV];
  Raw8<TR> res[NV], h[NV];
  const TX* x_row = static_cast<const TX*>(p.x) + r * p.ldx;
  const TR* res_row = static_cast<const TR*>(p.res) + r * p.ldres;
#pragma unroll
  for (int j = 0; j < NV; ++j) load8<WIDE>(x_row, t, j, N, p.K, x[j]);
  if (RES) {
#pragma unroll
    for (int j = 0; j < NV; ++j) load8<WIDE>(res_row, t, j, N, p.K, res[j]);
  }
  f32x2 sum2 = pair(0.f, 0.f);
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    h[j] = stream8<TX, TR, RES>(x[j], res[j]);
#pragma unroll
    for (int i = 0; i < 4; ++i) sum2 = fma2(h[j].two(i), h[j].two(i), sum2);
  }
  if (RES && p.h) {
    TR* out = static_cast<TR*>(p.h) + r * p.ldh;
#pragma unroll
    for (int j = 0; j < NV; ++j) store8<WIDE>(out, t, j, N, p.K, h[j]);
  }
  if (p.q) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      f32x2 g[4];
      gain8<WIDE>(p.gain, t, j, N, p.K, g);
      top = largest8(h[j], g, top);
    }
  }
  float sum = both(sum2), none = 0.f;
  over_row<false, true>(ex, turn, N, sum, none, top);
#pragma unroll
  for (int j = 0; j < NV; ++j) h[j].repack();
  const float inv_K = __fdiv_rn(1.f, static_cast<float>(p.K));
  float inv = root(sum, inv_K, p.eps);
  if (sum == CUDART_INF_F) {
    sum = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const Raw8<TR> z = smaller8(h[j]);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(z.at(i), z.at(i), sum);
    }
    uint32_t unused = 0;
    over_row<false, false>(ex, turn, N, sum, none, unused);
    inv = root(sum, inv_K, 0.f) * SMALLER;
  }
  Scale c{};
  if (p.q) {
    c = scale_of(top);
    if (t == 0) p.scale[r] = c.s * inv;
  }
  results<NV, WIDE>(p, r, t, N, h, inv, c, [&](int j, f32x2* g) { gain8<WIDE>(p.gain, t, j, N, p.K, g); });
}

// Many rows with little traffic each (no residual, or results in 8 bits): one block per SM, blockDim.x / N rows at a time, which come through
// shared memory, p.stages rows deep; the gain lies there too.  8192 x 4096 bf16 25 us (5.4 TB/s), in 8 bits 33 us: instructions bound that one.
template <typename TX, typename TR, bool RES, int N, int NV>
__global__ void __launch_bounds__(FORWARD_THREADS) rms_norm_ring_kernel(const __grid_constant__ Norm p) {
  constexpr bool WIDE = true;
  __shared__ Exchange ex;
  extern __shared__ __align__(16) char memory[];
  constexpr int X_BYTES = NV * 8 * static_cast<int>(sizeof(TX)) * N, STAGE = X_BYTES + (RES ? NV * 8 * static_cast<int>(sizeof(TR)) * N : 0);
  const int t = threadIdx.x & (N - 1), mine = threadIdx.x / N, rows = blockDim.x / N;
  const int64_t step = static_cast<int64_t>(gridDim.x) * rows, first = blockIdx.x * static_cast<int64_t>(rows) + mine;
  float* gain = reinterpret_cast<float*>(memory);
  char* ring = memory + NV * 32 * N + mine * p.stages * STAGE;
  const uint32_t ring_at = static_cast<uint32_t>(__cvta_generic_to_shared(ring));
  const float inv_K = __fdiv_rn(1.f, static_cast<float>(p.K));
  int turn = 0;
  for (int s = 0; s < p.stages; ++s) {
    clear_row<N, NV, WIDE, TX>(ring_at + s * STAGE, t, p.K);
    if (RES) clear_row<N, NV, WIDE, TR>(ring_at + s * STAGE + X_BYTES, t, p.K);
  }
  pdl_trigger();
  pdl_wait();
  const TX* x_row = static_cast<const TX*>(p.x) + first * p.ldx;
  const TR* res_row = RES ? static_cast<const TR*>(p.res) + first * p.ldres : nullptr;
  const int64_t x_step = step * p.ldx, res_step = step * p.ldres;
  auto send = [&](int64_t r, int s) {                      // the next row that has not been sent
    if (r < p.R) {
      send_row<N, NV, WIDE>(ring_at + s * STAGE, x_row, t, p.K);
      x_row += x_step;
      if (RES) {
        send_row<N, NV, WIDE>(ring_at + s * STAGE + X_BYTES, res_row, t, p.K);
        res_row += res_step;
      }
    }
    copies_sent();
  };
  for (int s = 0; s < p.stages - 1; ++s) send(first + s * step, s);
  keep_gain<N, NV, WIDE>(gain, p.gain, p.K);
  __syncthreads();
  int s = 0;
  for (int64_t r = first; r < p.R; r += step) {
    Raw8<TR> h[NV];
    f32x2 sum2 = pair(0.f, 0.f);
    uint32_t top = 0;
    __syncwarp();                                          // (the warp is done with the stage of the row before)
    send(r + (p.stages - 1) * step, s == 0 ? p.stages - 1 : s - 1);
    copies_landed(p.stages - 1);
    __syncwarp();
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      Raw8<TX> x;
      Raw8<TR> res;
      take8<N, WIDE>(ring_at + s * STAGE, t, j, x);
      if (RES) take8<N, WIDE>(ring_at + s * STAGE + X_BYTES, t, j, res);
      h[j] = stream8<TX, TR, RES>(x, res);
#pragma unroll
      for (int i = 0; i < 4; ++i) sum2 = fma2(h[j].two(i), h[j].two(i), sum2);
    }
    if (RES && p.h) {
      TR* out = static_cast<TR*>(p.h) + r * p.ldh;
#pragma unroll
      for (int j = 0; j < NV; ++j) store8<WIDE>(out, t, j, N, p.K, h[j]);
    }
    if (p.q) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        f32x2 g[4];
        kept_gain<N, WIDE>(gain, t, j, g);
        top = largest8(h[j], g, top);
      }
    }
    float sum = both(sum2), none = 0.f;
    if (p.q) over_row<false, true>(ex, turn, N, sum, none, top);
    else over_row<false, false>(ex, turn, N, sum, none, top);
#pragma unroll
    for (int j = 0; j < NV; ++j) h[j].repack();
    float inv = root(sum, inv_K, p.eps);
    if (sum == CUDART_INF_F) {
      sum = 0.f;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const Raw8<TR> z = smaller8(h[j]);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fmaf(z.at(i), z.at(i), sum);
      }
      uint32_t unused = 0;
      over_row<false, false>(ex, turn, N, sum, none, unused);
      inv = root(sum, inv_K, 0.f) * SMALLER;
    }
    Scale c{};
    if (p.q) {
      c = scale_of(top);
      if (t == 0) p.scale[r] = c.s * inv;
    }
    results<NV, WIDE>(p, r, t, N, h, inv, c, [&](int j, f32x2* g) { kept_gain<N, WIDE>(gain, t, j, g); });
    s = s == p.stages - 1 ? 0 : s + 1;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

// A row too long for registers: read a second time.
template <typename TX, typename TR, bool RES, bool WIDE>
__global__ void __launch_bounds__(1024) rms_norm_long_kernel(const __grid_constant__ Norm p) {
  __shared__ Exchange ex;
  const int n = p.n, t = threadIdx.x;
  const int vectors = (p.K + 8 * n - 1) / (8 * n);
  const int64_t r = blockIdx.x;
  int turn = 0;
  pdl_trigger();
  pdl_wait();
  // second: h is there if it is stored (x or the residual may be gone: h may lie in their place)
  auto stream = [&](int j, bool second) {
    Raw8<TX> x;
    Raw8<TR> res, h;
    if (RES && second && p.h) {
      load8<WIDE>(static_cast<const TR*>(p.h) + r * p.ldh, t, j, n, p.K, h);
      return h;
    }
    load8<WIDE>(static_cast<const TX*>(p.x) + r * p.ldx, t, j, n, p.K, x);
    if (RES) load8<WIDE>(static_cast<const TR*>(p.res) + r * p.ldres, t, j, n, p.K, res);
    h = stream8<TX, TR, RES>(x, res);
    if (RES && !second && p.h) store8<WIDE>(static_cast<TR*>(p.h) + r * p.ldh, t, j, n, p.K, h);
    return h;
  };
  float sum = 0.f, none = 0.f;
  f32x2 g[4];
  uint32_t top = 0, unused = 0;
#pragma unroll 2
  for (int j = 0; j < vectors; ++j) {
    const Raw8<TR> h = stream(j, false);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = fmaf(h.at(i), h.at(i), sum);
    if (p.q) {
      gain8<WIDE>(p.gain, t, j, n, p.K, g);
      top = largest8(h, g, top);
    }
  }
  over_row<false, true>(ex, turn, n, sum, none, top);
  float inv = root(sum, __fdiv_rn(1.f, static_cast<float>(p.K)), p.eps);
  if (sum == CUDART_INF_F) {
    sum = 0.f;
    for (int j = 0; j < vectors; ++j) {
      const Raw8<TR> h = stream(j, true);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(h.at(i) * SMALLER, h.at(i) * SMALLER, sum);
    }
    over_row<false, false>(ex, turn, n, sum, none, unused);
    inv = root(sum, __fdiv_rn(1.f, static_cast<float>(p.K)), 0.f) * SMALLER;
  }
  const Scale c = scale_of(top);
  for (int j = 0; j < vectors; ++j) {
    const Raw8<TR> h = stream(j, true);
    gain8<WIDE>(p.gain, t, j, n, p.K, g);
    if (p.y && p.y_bf16) result8<WIDE>(static_cast<__nv_bfloat16*>(p.y) + r * p.ldy, t, j, n, p.K, h, g, pair(inv, inv));
    else if (p.y) result8<WIDE>(static_cast<float*>(p.y) + r * p.ldy, t, j, n, p.K, h, g, pair(inv, inv));
    if (p.q) bytes8<WIDE>(p.q + r * p.ldq, t, j, n, p.K, h, g, c);
  }
  if (p.q && t == 0) p.scale[r] = c.s * inv;
}

// ---- backward ---------------------------------------------------------------------------------------------------------
struct Grad {
  const void *dy, *h, *dres;
  const float* gain;
  void* dx;
  float* part;               // [gridDim.x][K]: each block's sums of dg; null where they are not asked for
  int64_t lddy, ldh, lddres, lddx, R;
  float eps;
  int K, n, stages, acc_shared;         // acc_shared (long rows): the block's sums lie in shared memory
};

// One block per SM, blockDim.x / N rows at a time through shared memory (RING; floats of any alignment too, bf16 in whole vectors); a row is read
// from there twice, so that registers hold the sums of dg and little else.  8192 x 4096 bf16 with d_residual: 44 us (6.1 TB/s) without d_gain, 49
// with it: the kernel below cannot start before the last block ends.  Two vectors a thread to 4096 columns, four beyond (8192 columns 47 us, by two
// 53); 768 threads in fewer registers were slower on short batches (4099 x 1000 bf16 13.6 us, 10.8 with 512).
template <typename TD, typename TH, int N, int NV, bool RING, bool WIDE>
__global__ void __launch_bounds__(BACKWARD_THREADS) rms_norm_backward_kernel(const __grid_constant__ Grad p) {
  __shared__ Exchange ex;
  extern __shared__ __align__(16) char memory[];          // gain and ring; at the end the sums of dg
  constexpr int D_BYTES = NV * 8 * static_cast<int>(sizeof(TD)) * N, H_BYTES = NV * 8 * static_cast<int>(sizeof(TH)) * N;
  const int t = threadIdx.x & (N - 1), own = threadIdx.x / N, rows = blockDim.x / N, stage = D_BYTES + (p.dres ? 2 : 1) * H_BYTES;
  const int64_t step = static_cast<int64_t>(gridDim.x) * rows, first = blockIdx.x * static_cast<int64_t>(rows) + own;
  float* gain = reinterpret_cast<float*>(memory);
  char* ring = memory + NV * 32 * N + own * p.stages * stage;
  const uint32_t ring_at = static_cast<uint32_t>(__cvta_generic_to_shared(ring));
  const float inv_K = __fdiv_rn(1.f, static_cast<float>(p.K));
  int turn = 0;
  if constexpr (RING) {
    for (int s = 0; s < p.stages; ++s) {
      clear_row<N, NV, WIDE, TD>(ring_at + s * stage, t, p.K);
      clear_row<N, NV, WIDE, TH>(ring_at + s * stage + D_BYTES, t, p.K);
      if (p.dres) clear_row<N, NV, WIDE, TH>(ring_at + s * stage + D_BYTES + H_BYTES, t, p.K);
    }
  }
  pdl_trigger();
  pdl_wait();
  const TD* d_row = static_cast<const TD*>(p.dy) + first * p.lddy;
  const TH* h_row = static_cast<const TH*>(p.h) + first * p.ldh;
  const TH* res_row = p.dres ? static_cast<const TH*>(p.dres) + first * p.lddres : nullptr;
  const int64_t d_step = step * p.lddy, h_step = step * p.ldh, res_step = step * p.lddres;
  auto send = [&](int64_t r, int s) {                      // the next row that has not been sent
    if (r < p.R) {
      const uint32_t at = ring_at + s * stage;
      send_row<N, NV, WIDE>(at, d_row, t, p.K);
      send_row<N, NV, WIDE>(at + D_BYTES, h_row, t, p.K);
      d_row += d_step;
      h_row += h_step;
      if (p.dres) {
        send_row<N, NV, WIDE>(at + D_BYTES + H_BYTES, res_row, t, p.K);
        res_row += res_step;
      }
    }
    copies_sent();
  };
  if constexpr (RING) {
    for (int s = 0; s < p.stages - 1; ++s) send(first + s * step, s);
  }
  f32x2 acc[NV][4];
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[j][i] = pair(0.f, 0.f);
  keep_gain<N, NV, WIDE>(gain, p.gain, p.K);
  __syncthreads();
  int s = 0;
  for (int64_t r = first; r < p.R; r += step) {
    if constexpr (RING) {
      __syncwarp();
      send(r + (p.stages - 1) * step, s == 0 ? p.stages - 1 : s - 1);
      copies_landed(p.stages - 1);
      __syncwarp();
    }
    Raw8<TD> held_d[RING ? 1 : NV];
    Raw8<TH> held_z[RING ? 1 : NV];                      // a row that comes through shared memory is read from there again
    auto row8 = [&](int j, Raw8<TD>& d, Raw8<TH>& z) {
      if constexpr (RING) {
        take8<N, WIDE>(ring_at + s * stage, t, j, d);
        take8<N, WIDE>(ring_at + s * stage + D_BYTES, t, j, z);
      } else {
        d = held_d[j];
        z = held_z[j];
        d.repack();
        z.repack();
      }
    };
    f32x2 sum2 = pair(0.f, 0.f), dot2 = pair(0.f, 0.f);
    uint32_t unused = 0;
    if constexpr (!RING) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        load8<WIDE>(d_row, t, j, N, p.K, held_d[j]);
        load8<WIDE>(h_row, t, j, N, p.K, held_z[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      Raw8<TD> d;
      Raw8<TH> z;
      f32x2 g[4];
      row8(j, d, z);
      kept_gain<N, WIDE>(gain, t, j, g);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sum2 = fma2(z.two(i), z.two(i), sum2);
        dot2 = fma2(mul2(d.two(i), g[i]), z.two(i), dot2);
      }
    }
    float sum = both(sum2), dot = both(dot2);
    over_row<true, false>(ex, turn, N, sum, dot, unused);
    float small = 1.f, inv = root(sum, inv_K, p.eps);
    if (sum == CUDART_INF_F) {
      sum = dot = 0.f;
      small = SMALLER;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        Raw8<TD> d;
        Raw8<TH> z;
        f32x2 g[4];
        row8(j, d, z);
        kept_gain<N, WIDE>(gain, t, j, g);
        z = smaller8(z);
        if constexpr (RING) put8<N, WIDE>(ring_at + s * stage + D_BYTES, t, j, z);
        else held_z[j] = z;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 v = floats(z.two(i)), dg = floats(mul2(d.two(i), g[i]));
          sum = fmaf(v.x, v.x, fmaf(v.y, v.y, sum));
          dot = fmaf(dg.x, v.x, fmaf(dg.y, v.y, dot));
        }
      }
      over_row<true, false>(ex, turn, N, sum, dot, unused);
      inv = root(sum, inv_K, 0.f);
    }
    const float mean = dot * inv_K * inv, outer = inv * small;
    TH* out = static_cast<TH*>(p.dx) + r * p.lddx;
    const f32x2 inv2 = pair(inv, inv), minus_mean = pair(-mean, -mean), outer2 = pair(outer, outer);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      Raw8<TD> d;
      Raw8<TH> z, dres;
      row8(j, d, z);
      if (!p.dres) dres.clear();
      else if constexpr (RING) take8<N, WIDE>(ring_at + s * stage + D_BYTES + H_BYTES, t, j, dres);
      else load8<WIDE>(res_row, t, j, N, p.K, dres);
      f32x2 g[4];
      kept_gain<N, WIDE>(gain, t, j, g);
      float v[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x2 unit = mul2(z.two(i), inv2);
        const float2 f = floats(fma2(outer2, fma2(unit, minus_mean, mul2(d.two(i), g[i])), dres.two(i)));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
        acc[j][i] = fma2(d.two(i), unit, acc[j][i]);
      }
      Raw8<TH> o;
      o.set(v);
      store8<WIDE>(out, t, j, N, p.K, o);
    }
    if constexpr (!RING) {
      d_row += d_step;
      h_row += h_step;
      res_row += res_step;
    }
    s = s == p.stages - 1 ? 0 : s + 1;
  }
  if constexpr (RING) asm volatile("cp.async.wait_all;" ::: "memory");
  if (!p.part) return;
  // the rows' sums meet in shared memory, each thread's columns in the order of its vectors
  float* out = p.part + static_cast<int64_t>(blockIdx.x) * p.K;
  float* sums = reinterpret_cast<float*>(memory);
  __syncthreads();                                       // (gain and ring are done with)
  if (WIDE) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float2 a = floats(acc[j][2 * h]), b = floats(acc[j][2 * h + 1]);
        *reinterpret_cast<float4*>(sums + own * NV * 8 * N + ((2 * j + h) * N + t) * 4) = make_float4(a.x, a.y, b.x, b.y);
      }
  } else {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 v = floats(acc[j][i >> 1]);
        sums[own * NV * 8 * N + column<false>(t, j, N, i)] = i & 1 ? v.y : v.x;
      }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < NV * 2 * N; i += blockDim.x) {
    float4 total = *reinterpret_cast<const float4*>(sums + 4 * i);
    for (int k = 1; k < rows; ++k) {
      const float4 v = *reinterpret_cast<const float4*>(sums + k * NV * 8 * N + 4 * i);
      total = make_float4(total.x + v.x, total.y + v.y, total.z + v.z, total.w + v.w);
    }
    const int c = WIDE ? 8 * (i % N + i / (2 * N) * N) + 4 * (i / N & 1) : 4 * i;
    const float v[4] = {total.x, total.y, total.z, total.w};
#pragma unroll
    for (int m = 0; m < 4; ++m)
      if (c + m < p.K) out[c + m] = v[m];
  }
}

// Rows too long for registers: read a second time, two vectors at a time on their way, the block's sums of dg in shared memory or, longer
// than that, in its row of `part`.
template <typename TD, typename TH, bool WIDE>
__global__ void __launch_bounds__(1024) rms_norm_backward_long_kernel(const __grid_constant__ Grad p) {
  constexpr int TWO = 2;
  __shared__ Exchange ex;
  extern __shared__ float shared_acc[];
  const int n = p.n, t = threadIdx.x;
  const int vectors = (p.K + 8 * n - 1) / (8 * n);
  const float inv_K = __fdiv_rn(1.f, static_cast<float>(p.K));
  int turn = 0;
  pdl_trigger();
  pdl_wait();
  float* out = p.part ? p.part + static_cast<int64_t>(blockIdx.x) * p.K : nullptr;
  const bool shared = p.part && p.acc_shared;
  // where a thread's sum lies: apart in the banks, or in its column
  auto place = [&](int j, int i) { return shared ? (8 * j + i) * n + t : column<WIDE>(t, j, n, i); };
  float* acc = shared ? shared_acc : out;
  if (acc)
    for (int j = 0; j < vectors; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (column<WIDE>(t, j, n, i) < p.K) acc[place(j, i)] = 0.f;
  for (int64_t r = blockIdx.x; r < p.R; r += gridDim.x) {
    const TD* dy = static_cast<const TD*>(p.dy) + r * p.lddy;
    const TH* h = static_cast<const TH*>(p.h) + r * p.ldh;
    float small = 1.f, inv = 0.f, sum, dot;
    uint32_t unused = 0;
    for (int pass = 0; pass < 2; ++pass) {
      sum = dot = 0.f;
      for (int j0 = 0; j0 < vectors; j0 += TWO) {
        Raw8<TD> d[TWO];
        Raw8<TH> z[TWO];
        f32x2 g[4];
#pragma unroll
        for (int u = 0; u < TWO; ++u) {                    // (vectors behind the last are zeros)
          load8<WIDE>(dy, t, j0 + u, n, p.K, d[u]);
          load8<WIDE>(h, t, j0 + u, n, p.K, z[u]);
        }
#pragma unroll
        for (int u = 0; u < TWO; ++u) {
          gain8<WIDE>(p.gain, t, j0 + u, n, p.K, g);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 v = floats(mul2(z[u].two(i), pair(small, small))), dg = floats(mul2(d[u].two(i), g[i]));
            sum = fmaf(v.x, v.x, fmaf(v.y, v.y, sum));
            dot = fmaf(dg.x, v.x, fmaf(dg.y, v.y, dot));
          }
        }
      }
      over_row<true, false>(ex, turn, n, sum, dot, unused);
      inv = root(sum, inv_K, pass ? 0.f : p.eps);
      if (sum != CUDART_INF_F) break;
      small = SMALLER;
    }
    const float mean = dot * inv_K * inv, outer = inv * small;
    TH* to = static_cast<TH*>(p.dx) + r * p.lddx;
    for (int j0 = 0; j0 < vectors; j0 += TWO) {
      Raw8<TD> d[TWO];
      Raw8<TH> z[TWO], dres[TWO];
#pragma unroll
      for (int u = 0; u < TWO; ++u) {
        load8<WIDE>(dy, t, j0 + u, n, p.K, d[u]);
        load8<WIDE>(h, t, j0 + u, n, p.K, z[u]);
        if (p.dres) load8<WIDE>(static_cast<const TH*>(p.dres) + r * p.lddres, t, j0 + u, n, p.K, dres[u]);
        else dres[u].clear();
      }
#pragma unroll
      for (int u = 0; u < TWO; ++u) {
        const int j = j0 + u;
        f32x2 g[4];
        float v[8];
        Raw8<TH> o;
        gain8<WIDE>(p.gain, t, j, n, p.K, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float unit = z[u].at(i) * small * inv;
          const float2 gi = floats(g[i >> 1]);
          v[i] = fmaf(outer, fmaf(-unit, mean, d[u].at(i) * (i & 1 ? gi.y : gi.x)), dres[u].at(i));
          if (acc && column<WIDE>(t, j, n, i) < p.K) {
            const int at = place(j, i);
            acc[at] = fmaf(d[u].at(i), unit, acc[at]);
          }
        }
        o.set(v);
        store8<WIDE>(to, t, j, n, p.K, o);
      }
    }
  }
  if (shared)
    for (int j = 0; j < vectors; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int c = column<WIDE>(t, j, n, i);
        if (c < p.K) out[c] = acc[place(j, i)];
      }
}

// dg = the blocks' sums, added in the order of the blocks within 32 strands: all loads of a thread are under way at once.  Its blocks are small
// enough to wait beside the blocks of the kernel above.
__global__ void __launch_bounds__(256) gain_sums_kernel(const float* part, int slots, int K, float* d_gain) {
  __shared__ float strand[32][33];
  const int l = threadIdx.x & 31, w = threadIdx.x >> 5, first = blockIdx.x * 32;
  const int q = threadIdx.x & 7, row = threadIdx.x >> 3, c = first + 4 * q;      // four columns of every 32nd row
  pdl_trigger();
  pdl_wait();
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (K % 4 == 0 && (reinterpret_cast<uintptr_t>(part) & 15u) == 0) {
    if (c < K) {
#pragma unroll 5
      for (int k = row; k < slots; k += 32) {
        const float4 v = *reinterpret_cast<const float4*>(part + static_cast<int64_t>(k) * K + c);
        s = make_float4(s.x + v.x, s.y + v.y, s.z + v.z, s.w + v.w);
      }
    }
  } else {
#pragma unroll 2
    for (int k = row; k < slots; k += 32) {
      const float* at = part + static_cast<int64_t>(k) * K + c;
      s.x += c < K ? at[0] : 0.f;
      s.y += c + 1 < K ? at[1] : 0.f;
      s.z += c + 2 < K ? at[2] : 0.f;
      s.w += c + 3 < K ? at[3] : 0.f;
    }
  }
  strand[row][4 * q] = s.x; strand[row][4 * q + 1] = s.y; strand[row][4 * q + 2] = s.z; strand[row][4 * q + 3] = s.w;
  __syncthreads();
#pragma unroll
  for (int m = 0; m < 4; ++m) {                            // warp w: columns 4 w .. of the block's, their strands in the lanes
    float v = strand[l][4 * w + m];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    if (l == 0 && first + 4 * w + m < K) d_gain[first + 4 * w + m] = v;
  }
}

// ---- launches ---------------------------------------------------------------------------------------------------------
constexpr int MEMORY = 216 * 1024;         // most shared memory of a block

int pow2_threads(int64_t want, int most) {
  int n = 32;
  while (n < want && n < most) n *= 2;
  return n;
}

// A kernel's shared memory beyond the 48 KB that need no leave: asked for once per device.
template <auto KERNEL> cudaError_t allow(size_t bytes) {
  if (bytes <= 47 * 1024) return cudaSuccess;
  static std::atomic<uint64_t> asked{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || (dev < 64 && (asked.load(std::memory_order_relaxed) >> dev & 1u))) return e;
  e = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, MEMORY);
  if (e == cudaSuccess && dev < 64) asked.fetch_or(uint64_t{1} << dev, std::memory_order_relaxed);
  return e;
}

// How rows of K values go through one block per SM: N threads and NV vectors a row, `rows` rows at a time, `stages` deep (0: not
// through shared memory); row_bytes: what a thread's eight columns take in all tensors that come that way.
constexpr int64_t LONGEST = 16384;
struct Shape { int n, nv, rows, stages; size_t bytes; };
Shape shape_of(int64_t K, int row_bytes, bool ring, int threads, int64_t two_vectors) {
  Shape s{};
  s.nv = K <= two_vectors ? 2 : 4;
  s.n = pow2_threads((K + 8 * s.nv - 1) / (8 * s.nv), 512);
  const size_t gain = static_cast<size_t>(s.nv) * 32 * s.n, row = static_cast<size_t>(s.nv) * row_bytes * s.n;
  s.rows = threads / s.n;
  if (s.n > 32 && s.rows > 15) s.rows = 15;                // barriers of a block: 0 .. 15, and 0 is everybody's
  s.bytes = gain;
  if (!ring) return s;
  while (s.rows > 1 && gain + 2 * row * s.rows > MEMORY) --s.rows;
  while (s.stages < MOST_STAGES && gain + (s.stages + 1) * row * s.rows <= MEMORY) ++s.stages;
  if (s.stages < 2) s.stages = 0;
  else s.bytes = gain + s.stages * row * s.rows;
  return s;
}

template <auto KERNEL, typename P> cudaError_t launch_shape(P p, const Shape& s, size_t bytes, int64_t grid, cudaStream_t stream) {
  const cudaError_t e = allow<KERNEL>(bytes);
  if (e != cudaSuccess) return e;
  p.n = s.n;
  p.stages = s.stages;
  return launch_pdl(KERNEL, dim3(static_cast<unsigned>(grid)), dim3(s.n * s.rows), bytes, stream, 1, p);
}

// How rows of K values go directly: N threads and NV vectors.
template <typename TX, typename TR, bool RES, bool WIDE>
cudaError_t launch_direct(Norm p, cudaStream_t stream) {
  const int nv = p.K <= 512 ? 2 : p.K <= 1024 ? 4 : p.K <= 4096 ? 2 : 4;      // (a warp to itself is worth more vectors; 8 warps are enough)
  p.n = pow2_threads((p.K + 8 * nv - 1) / (8 * nv), 256);
  const int threads = p.n < 128 ? 128 : p.n, rows = threads / p.n;
  const dim3 grid(static_cast<unsigned>((p.R + rows - 1) / rows)), block(threads);
  switch (nv * 1024 + p.n) {
    case 2 * 1024 + 32: return launch_pdl(rms_norm_direct_kernel<TX, TR, RES, 32, 2, WIDE>, grid, block, 0, stream, 1, p);
    case 2 * 1024 + 128: return launch_pdl(rms_norm_direct_kernel<TX, TR, RES, 128, 2, WIDE>, grid, block, 0, stream, 1, p);
    case 2 * 1024 + 256: return launch_pdl(rms_norm_direct_kernel<TX, TR, RES, 256, 2, WIDE>, grid, block, 0, stream, 1, p);
    case 4 * 1024 + 32: return launch_pdl(rms_norm_direct_kernel<TX, TR, RES, 32, 4, WIDE>, grid, block, 0, stream, 1, p);
    default: return launch_pdl(rms_norm_direct_kernel<TX, TR, RES, 256, 4, WIDE>, grid, block, 0, stream, 1, p);
  }
}

template <typename TX, typename TR, bool RES>
cudaError_t launch_ring(const Norm& p, const Shape& s, int sms, cudaStream_t stream) {
  const int64_t want = (p.R + s.rows - 1) / s.rows, grid = want < sms ? want : sms;
  switch (s.nv * 1024 + s.n) {
    case 2 * 1024 + 32: return launch_shape<rms_norm_ring_kernel<TX, TR, RES, 32, 2>>(p, s, s.bytes, grid, stream);
    case 4 * 1024 + 32: return launch_shape<rms_norm_ring_kernel<TX, TR, RES, 32, 4>>(p, s, s.bytes, grid, stream);
    case 4 * 1024 + 64: return launch_shape<rms_norm_ring_kernel<TX, TR, RES, 64, 4>>(p, s, s.bytes, grid, stream);
    case 4 * 1024 + 128: return launch_shape<rms_norm_ring_kernel<TX, TR, RES, 128, 4>>(p, s, s.bytes, grid, stream);
    case 4 * 1024 + 256: return launch_shape<rms_norm_ring_kernel<TX, TR, RES, 256, 4>>(p, s, s.bytes, grid, stream);
    default: return launch_shape<rms_norm_ring_kernel<TX, TR, RES, 512, 4>>(p, s, s.bytes, grid, stream);
  }
}

// Few rows go one per block, for the latency.  Others go directly where their traffic hides what a row costs besides (8 bytes a value: 8192 x
// 4096 bf16 with residual 43 us, by the ring 48; 8192 x 2048 floats with one 42, 48), or where they are too few to fill the ring (2000 x 4096 without
// a residual 9.4 us, 10.4; 1000 x 1024 with one 2.5, 4.6); through the ring where there is less traffic (8192 x 4096 bf16 without a residual 25 us,
// directly 32; in 8 bits with one 43, 48).
template <typename TX, typename TR, bool RES, bool WIDE>
cudaError_t launch_norm(Norm p, int sms, cudaStream_t stream) {
  if (p.K <= 8192) {
    if (p.R < 2 * sms) {
      p.n = pow2_threads((p.K + 7) / 8, 1024);
      return launch_pdl(rms_norm_few_kernel<TX, TR, RES, WIDE>, dim3(static_cast<unsigned>(p.R)), dim3(p.n), 0, stream, 1, p);
    }
    const int bytes = static_cast<int>(sizeof(TX) + (RES ? (p.h ? 2 : 1) * sizeof(TR) : 0)) + (p.y ? (p.y_bf16 ? 2 : 4) : 0);
    if (!WIDE || (bytes >= 8 && !p.q) || p.R * p.K <= 10000000) return launch_direct<TX, TR, RES, WIDE>(p, stream);
  }
  if constexpr (WIDE) {
    const Shape s = shape_of(p.K, 8 * static_cast<int>(sizeof(TX) + (RES ? sizeof(TR) : 0)), true, FORWARD_THREADS, 512);
    if (p.K <= LONGEST && s.stages) return launch_ring<TX, TR, RES>(p, s, sms, stream);
  }
  p.n = 1024;
  return launch_pdl(rms_norm_long_kernel<TX, TR, RES, WIDE>, dim3(static_cast<unsigned>(p.R)), dim3(1024), 0, stream, 1, p);
}

template <typename TD, typename TH, bool RING, bool WIDE>
cudaError_t launch_rows(const Grad& p, const Shape& s, int64_t grid, cudaStream_t stream) {
  const size_t joined = p.part ? static_cast<size_t>(s.rows) * s.nv * 8 * s.n * 4 : 0, bytes = s.bytes > joined ? s.bytes : joined;
  switch (s.nv * 1024 + s.n) {
    case 2 * 1024 + 32: return launch_shape<rms_norm_backward_kernel<TD, TH, 32, 2, RING, WIDE>>(p, s, bytes, grid, stream);
    case 2 * 1024 + 64: return launch_shape<rms_norm_backward_kernel<TD, TH, 64, 2, RING, WIDE>>(p, s, bytes, grid, stream);
    case 2 * 1024 + 128: return launch_shape<rms_norm_backward_kernel<TD, TH, 128, 2, RING, WIDE>>(p, s, bytes, grid, stream);
    case 2 * 1024 + 256: return launch_shape<rms_norm_backward_kernel<TD, TH, 256, 2, RING, WIDE>>(p, s, bytes, grid, stream);
    case 4 * 1024 + 32: return launch_shape<rms_norm_backward_kernel<TD, TH, 32, 4, RING, WIDE>>(p, s, bytes, grid, stream);
    case 4 * 1024 + 64: return launch_shape<rms_norm_backward_kernel<TD, TH, 64, 4, RING, WIDE>>(p, s, bytes, grid, stream);
    case 4 * 1024 + 128: return launch_shape<rms_norm_backward_kernel<TD, TH, 128, 4, RING, WIDE>>(p, s, bytes, grid, stream);
    case 4 * 1024 + 256: return launch_shape<rms_norm_backward_kernel<TD, TH, 256, 4, RING, WIDE>>(p, s, bytes, grid, stream);
    default: return launch_shape<rms_norm_backward_kernel<TD, TH, 512, 4, RING, WIDE>>(p, s, bytes, grid, stream);
  }
}

template <typename TD, typename TH, bool WIDE>
cudaError_t launch_backward(Grad p, int sms, float* d_gain, cudaStream_t stream) {
  constexpr bool RING = WIDE || (sizeof(TD) == 4 && sizeof(TH) == 4);
  const Shape s = shape_of(p.K, 8 * static_cast<int>(sizeof(TD) + (p.dres ? 2 : 1) * sizeof(TH)), RING, BACKWARD_THREADS, 4096);
  int64_t grid = (p.R + s.rows - 1) / s.rows;
  cudaError_t e;
  if (p.K > LONGEST || (RING && !s.stages)) {
    p.n = 1024;
    grid = p.R < sms ? p.R : sms;
    size_t bytes = (static_cast<size_t>(p.K) + 8191) / 8192 * 8192 * 4;
    p.acc_shared = p.part && bytes <= MEMORY;
    if (!p.acc_shared) bytes = 0;
    if ((e = allow<rms_norm_backward_long_kernel<TD, TH, WIDE>>(bytes)) != cudaSuccess) return e;
    e = launch_pdl(rms_norm_backward_long_kernel<TD, TH, WIDE>, dim3(static_cast<unsigned>(grid)), dim3(1024), bytes, stream, 1, p);
  } else {
    if (grid > sms) grid = sms;
    e = launch_rows<TD, TH, RING, WIDE>(p, s, grid, stream);
  }
  if (e != cudaSuccess || !p.part) return e;
  return launch_pdl(gain_sums_kernel, dim3(static_cast<unsigned>((p.K + 31) / 32)), dim3(256), 0, stream, 1, static_cast<const float*>(p.part),
                    static_cast<int>(grid), p.K, d_gain);
}

mbd_status device(int* sms) {
  int dev = 0;
  if (cudaGetDevice(&dev) == cudaSuccess && cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess) return MBD_OK;
  (void)cudaGetLastError();
  return MBD_E_CUDA;
}

mbd_status done(cudaError_t e) {
  if (e == cudaSuccess) return MBD_OK;
  (void)cudaGetLastError();
  return MBD_E_CUDA;
}

}  // namespace
}  // namespace mbd

using namespace mbd;
typedef __nv_bfloat16 bf16;

extern "C" mbd_status mbd_rms_norm(int64_t R, int64_t K, const void* X_dev, int x_bf16, int64_t ldx, const void* residual_dev, int residual_bf16,
                                   int64_t ldres, const float* gain_dev, double eps, void* H_dev, int64_t ldh, void* Y_dev, int y_bf16,
                                   int64_t ldy, int8_t* Q_dev, int64_t ldq, float* scale_dev, void* cuda_stream) {
  if (R < 0 || K < 1 || !(eps >= 1e-30 && eps < 1.0)) return MBD_E_INVALID;
  if (R == 0) return MBD_OK;
  if (!X_dev || (!Y_dev && !Q_dev) || (H_dev && !residual_dev) || (Q_dev && !scale_dev)) return MBD_E_INVALID;
  const int held = residual_bf16 ? 2 : 4;
  const Rows x{X_dev, R, K, ldx, x_bf16 ? 2 : 4}, res{residual_dev, R, K, ldres, held}, h{H_dev, R, K, ldh, held}, y{Y_dev, R, K, ldy, y_bf16 ? 2 : 4},
      q{Q_dev, R, K, ldq, 1}, scale{Q_dev ? scale_dev : nullptr, 1, R, R, 4}, gain{gain_dev, 1, K, K, 4};
  for (const Rows* t : {&x, &res, &h, &y, &q})
    if (t->base && R > 1 && t->ld < K) return MBD_E_INVALID;
  if (R > INT32_MAX || K > INT32_MAX - 65536) return MBD_E_UNSUPPORTED;
  for (const Rows* t : {&x, &res, &h, &y, &scale, &gain})
    if (t->misplaced()) return MBD_E_UNSUPPORTED;
  // results are apart from each other and from the inputs; h and y may take the place of an input of their type
  const bool x_as_h = !x_bf16 == !residual_bf16, x_as_y = !x_bf16 == !y_bf16, res_as_y = !residual_bf16 == !y_bf16;
  if (!apart(h, y) || !apart(h, q) || !apart(h, scale) || !apart(h, gain) || !apart(y, q) || !apart(y, scale) || !apart(y, gain) ||
      !apart(q, scale) || !apart(q, gain) || !apart(q, x) || !apart(q, res) || !apart(scale, x) || !apart(scale, res) || !apart(scale, gain) ||
      !apart_or_same(h, res) || !(x_as_h ? apart_or_same(h, x) : apart(h, x)) || !(x_as_y ? apart_or_same(y, x) : apart(y, x)) ||
      !(res_as_y ? apart_or_same(y, res) : apart(y, res))) return MBD_E_INVALID;
  int sms = 0;
  const mbd_status st = device(&sms);
  if (st != MBD_OK) return st;
  Norm p{X_dev, residual_dev, gain_dev, H_dev, Y_dev, Q_dev, scale_dev, ldx, ldres, ldh, ldy, ldq, R, static_cast<float>(eps), static_cast<int>(K), y_bf16 != 0, 0, 0};
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const bool wide = K % 8 == 0 && x.wide() && res.wide() && h.wide() && y.wide() && q.wide();
  cudaError_t e;
  if (!residual_dev)
    e = x_bf16 ? (wide ? launch_norm<bf16, bf16, false, true>(p, sms, stream) : launch_norm<bf16, bf16, false, false>(p, sms, stream))
               : (wide ? launch_norm<float, float, false, true>(p, sms, stream) : launch_norm<float, float, false, false>(p, sms, stream));
  else if (residual_bf16)
    e = x_bf16 ? (wide ? launch_norm<bf16, bf16, true, true>(p, sms, stream) : launch_norm<bf16, bf16, true, false>(p, sms, stream))
               : (wide ? launch_norm<float, bf16, true, true>(p, sms, stream) : launch_norm<float, bf16, true, false>(p, sms, stream));
  else
    e = x_bf16 ? (wide ? launch_norm<bf16, float, true, true>(p, sms, stream) : launch_norm<bf16, float, true, false>(p, sms, stream))
               : (wide ? launch_norm<float, float, true, true>(p, sms, stream) : launch_norm<float, float, true, false>(p, sms, stream));
  return done(e);
}

extern "C" mbd_status mbd_rms_norm_backward(int64_t R, int64_t K, const void* dY_dev, int dy_bf16, int64_t lddy, const void* H_dev, int h_bf16,
                                            int64_t ldh, const float* gain_dev, double eps, const void* d_residual_dev, int64_t lddres,
                                            void* dX_dev, int64_t lddx, float* d_gain_dev, float* scratch_dev, void* cuda_stream) {
  if (R < 0 || K < 1 || !(eps >= 1e-30 && eps < 1.0)) return MBD_E_INVALID;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const Rows d_gain{d_gain_dev, 1, K, K, 4}, gain{gain_dev, 1, K, K, 4};
  if (R == 0) {                                             // a sum over no rows
    if (!d_gain_dev) return MBD_OK;
    if (d_gain.misplaced()) return MBD_E_UNSUPPORTED;
    return done(cudaMemsetAsync(d_gain_dev, 0, static_cast<size_t>(K) * 4, stream));
  }
  if (!dY_dev || !H_dev || !dX_dev || (d_gain_dev && !scratch_dev)) return MBD_E_INVALID;
  const int held = h_bf16 ? 2 : 4;
  const int64_t slots = R < MBD_NORM_SCRATCH_ROWS ? R : MBD_NORM_SCRATCH_ROWS;
  const Rows dy{dY_dev, R, K, lddy, dy_bf16 ? 2 : 4}, h{H_dev, R, K, ldh, held}, dres{d_residual_dev, R, K, lddres, held}, dx{dX_dev, R, K, lddx, held},
      scratch{d_gain_dev ? scratch_dev : nullptr, slots, K, K, 4};
  for (const Rows* t : {&dy, &h, &dres, &dx})
    if (t->base && R > 1 && t->ld < K) return MBD_E_INVALID;
  if (R > INT32_MAX || K > INT32_MAX - 65536) return MBD_E_UNSUPPORTED;
  for (const Rows* t : {&dy, &h, &dres, &dx, &d_gain, &scratch, &gain})
    if (t->misplaced()) return MBD_E_UNSUPPORTED;
  if (!apart_or_same(dx, h) || !apart_or_same(dx, dres) || !(dy.size == held ? apart_or_same(dx, dy) : apart(dx, dy)) || !apart(dx, gain)) return MBD_E_INVALID;
  for (const Rows* out : {&d_gain, &scratch})
    for (const Rows* t : {&dy, &h, &dres, &dx, &gain})
      if (!apart(*out, *t)) return MBD_E_INVALID;
  if (!apart(d_gain, scratch)) return MBD_E_INVALID;
  int sms = 0;
  const mbd_status st = device(&sms);
  if (st != MBD_OK) return st;
  if (sms > MBD_NORM_SCRATCH_ROWS) sms = MBD_NORM_SCRATCH_ROWS;
  const Grad p{dY_dev, H_dev, d_residual_dev, gain_dev, dX_dev, d_gain_dev ? scratch_dev : nullptr, lddy, ldh, lddres, lddx, R, static_cast<float>(eps), static_cast<int>(K), 0, 0, 0};
  const bool wide = K % 8 == 0 && dy.wide() && h.wide() && dres.wide() && dx.wide();
  cudaError_t e;
  if (dy_bf16 && h_bf16) e = wide ? launch_backward<bf16, bf16, true>(p, sms, d_gain_dev, stream) : launch_backward<bf16, bf16, false>(p, sms, d_gain_dev, stream);
  else if (dy_bf16) e = wide ? launch_backward<bf16, float, true>(p, sms, d_gain_dev, stream) : launch_backward<bf16, float, false>(p, sms, d_gain_dev, stream);
  else if (h_bf16) e = wide ? launch_backward<float, bf16, true>(p, sms, d_gain_dev, stream) : launch_backward<float, bf16, false>(p, sms, d_gain_dev, stream);
  else e = wide ? launch_backward<float, float, true>(p, sms, d_gain_dev, stream) : launch_backward<float, float, false>(p, sms, d_gain_dev, stream);
  return done(e);
}
