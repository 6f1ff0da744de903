// Root-mean-square norm of rows, with the residual's addition in front and rows in 16, 32 or 8 bits behind, and its gradients.
//
//   h = x (+ residual, rounded to the residual's type),  r = 1 / sqrt(mean(h^2) + eps),  y = h r g
//   in 8 bits: u = h g in float, s = max |u| / 127, q = u / s rounded to an integer, scale = s r.  r is the same for all of a row, so it goes
//   into the scale: q needs the row's largest |u| only and does not depend on the order in which the squares are added.
//   backward: m = mean(dy g h r),  dh = r (dy g - h r m) (+ the gradient that arrives along the residual),  dg = sum over rows of dy h r
//
// Each tensor passes once: the row stays in registers between the sum and the result, the gain and the columns' sums of dg
// in the registers of the threads that own the columns (blocks take row after row).  HBM bounds large calls, latency small ones.
#include <math_constants.h>

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
  int64_t ldx, ldres, ldh, ldy, ldq, R, K;
  float eps;
  int y_bf16, n;              // n: threads per row, a power of 2
};

// Squares beyond float's range (|h| above 1e19 / sqrt(K)) are added up again with the row taken 2^-80 times as large.
constexpr float SMALLER = 8.271806125530277e-25f;   // 2^-80

__device__ __forceinline__ float root(float sum, float K, float eps) { return __frcp_rn(__fsqrt_rn(__fdiv_rn(sum, K) + eps)); }

// Sums and maxima over the n threads of a row; everybody gets them.  n > 32: the block is one row; `turn` alternates so that one
// barrier per exchange is enough.
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
  const int w = threadIdx.x >> 5, l = threadIdx.x & 31, warps = n >> 5;
  if (l == 0) {
    e.a[turn][w] = a;
    if (B) e.b[turn][w] = b;
    if (M) e.m[turn][w] = m;
  }
  __syncthreads();
  a = l < warps ? e.a[turn][l] : 0.f;
  if (B) b = l < warps ? e.b[turn][l] : 0.f;
  if (M) m = __reduce_max_sync(0xffffffffu, l < warps ? e.m[turn][l] : 0u);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    a += __shfl_xor_sync(0xffffffffu, a, d);
    if (B) b += __shfl_xor_sync(0xffffffffu, b, d);
  }
  turn ^= 1;
}

template <bool WIDE>
__device__ __forceinline__ void gain8(const float* gain, int t, int64_t j, int n, int64_t K, float* g) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t c = column<WIDE>(t, j, n, i);
    g[i] = c >= K ? 0.f : gain ? gain[c] : 1.f;
  }
}

// h of one vector, from what was loaded; with a residual it is rounded to the residual's type.
template <typename TX, typename TR, bool RES>
__device__ __forceinline__ Raw8<TR> stream8(const Raw8<TX>& x, const Raw8<TR>& res) {
  Raw8<TR> h;
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = RES ? x.at(i) + res.at(i) : x.at(i);
  h.set(v);
  return h;
}

template <bool WIDE, typename TR>
__device__ __forceinline__ void results8(const Norm& p, int64_t r, int t, int64_t j, const Raw8<TR>& h, const float* g, float inv, const Scale& c) {
  if (p.y) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = h.at(i) * inv * g[i];
    store8<WIDE>(p.y, p.y_bf16, r * p.ldy, t, j, p.n, p.K, v);
  }
  if (p.q) {
    f32x2 u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = pair(h.at(2 * i) * g[2 * i], h.at(2 * i + 1) * g[2 * i + 1]);
    const uint2 w = quotients(u, c.s, c.inv, c.tiny);
    int8_t* q = p.q + r * p.ldq;
    if (WIDE) {
      if (column<true>(t, j, p.n, 0) < p.K) *reinterpret_cast<uint2*>(q + column<true>(t, j, p.n, 0)) = w;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t k = column<false>(t, j, p.n, i);
        if (k < p.K) q[k] = static_cast<int8_t>((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
      }
    }
  }
}

// Rows in registers, NV vectors a thread.  AHEAD: the next row is on its way while this one is worked on.
template <typename TX, typename TR, bool RES, int NV, int MAXT, bool AHEAD, bool WIDE>
__global__ void __launch_bounds__(MAXT) rms_norm_kernel(const __grid_constant__ Norm p) {
  __shared__ Exchange ex;
  const int n = p.n, t = threadIdx.x & (n - 1), rows = blockDim.x / n;
  const int64_t step = static_cast<int64_t>(gridDim.x) * rows;
  int turn = 0;
  pdl_trigger();
  pdl_wait();
  float g[NV][8];
#pragma unroll
  for (int j = 0; j < NV; ++j) gain8<WIDE>(p.gain, t, j, n, p.K, g[j]);
  Raw8<TX> x[NV];
  Raw8<TR> res[NV];
  auto fetch = [&](int64_t r) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      x[j].clear();
      res[j].clear();
      if (r < p.R) {
        load8<WIDE>(static_cast<const TX*>(p.x) + r * p.ldx, t, j, n, p.K, x[j]);
        if (RES) load8<WIDE>(static_cast<const TR*>(p.res) + r * p.ldres, t, j, n, p.K, res[j]);
      }
    }
  };
  int64_t r = blockIdx.x * static_cast<int64_t>(rows) + threadIdx.x / n;
  if (AHEAD) fetch(r);
  for (int64_t base = blockIdx.x * static_cast<int64_t>(rows); base < p.R; base += step, r += step) {
    if (!AHEAD) fetch(r);
    Raw8<TR> h[NV];
    float sum = 0.f, none = 0.f;
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      h[j] = stream8<TX, TR, RES>(x[j], res[j]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        sum = fmaf(h[j].at(i), h[j].at(i), sum);
        if (p.q) top = max(top, __float_as_uint(h[j].at(i) * g[j][i]) & 0x7FFFFFFFu);
      }
      if (RES && p.h && r < p.R) store8<WIDE>(static_cast<TR*>(p.h) + r * p.ldh, t, j, n, p.K, h[j]);
    }
    if (AHEAD) fetch(r + step);
    over_row<false, true>(ex, turn, n, sum, none, top);
    float inv = root(sum, static_cast<float>(p.K), p.eps);
    if (sum == CUDART_INF_F) {
      sum = 0.f;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fmaf(h[j].at(i) * SMALLER, h[j].at(i) * SMALLER, sum);
      uint32_t unused = 0;
      over_row<false, false>(ex, turn, n, sum, none, unused);
      inv = root(sum, static_cast<float>(p.K), 0.f) * SMALLER;
    }
    const Scale c = scale_of(top);
    if (r < p.R) {
#pragma unroll
      for (int j = 0; j < NV; ++j) results8<WIDE>(p, r, t, j, h[j], g[j], inv, c);
      if (p.q && t == 0) p.scale[r] = c.s * inv;
    }
  }
}

// A row too long for registers: read a second time.
template <typename TX, typename TR, bool RES, bool WIDE>
__global__ void __launch_bounds__(1024) rms_norm_long_kernel(const __grid_constant__ Norm p) {
  __shared__ Exchange ex;
  const int n = p.n, t = threadIdx.x;
  const int64_t vectors = (p.K + 8 * n - 1) / (8 * n), r = blockIdx.x;
  int turn = 0;
  pdl_trigger();
  pdl_wait();
  // second: h is there if it is stored (x or the residual may be gone: h may lie in their place)
  auto stream = [&](int64_t j, bool second) {
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
  float sum = 0.f, none = 0.f, g[8];
  uint32_t top = 0, unused = 0;
  for (int64_t j = 0; j < vectors; ++j) {
    const Raw8<TR> h = stream(j, false);
    gain8<WIDE>(p.gain, t, j, n, p.K, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      sum = fmaf(h.at(i), h.at(i), sum);
      top = max(top, __float_as_uint(h.at(i) * g[i]) & 0x7FFFFFFFu);
    }
  }
  over_row<false, true>(ex, turn, n, sum, none, top);
  float inv = root(sum, static_cast<float>(p.K), p.eps);
  if (sum == CUDART_INF_F) {
    sum = 0.f;
    for (int64_t j = 0; j < vectors; ++j) {
      const Raw8<TR> h = stream(j, true);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(h.at(i) * SMALLER, h.at(i) * SMALLER, sum);
    }
    over_row<false, false>(ex, turn, n, sum, none, unused);
    inv = root(sum, static_cast<float>(p.K), 0.f) * SMALLER;
  }
  const Scale c = scale_of(top);
  for (int64_t j = 0; j < vectors; ++j) {
    const Raw8<TR> h = stream(j, true);
    gain8<WIDE>(p.gain, t, j, n, p.K, g);
    results8<WIDE>(p, r, t, j, h, g, inv, c);
  }
  if (p.q && t == 0) p.scale[r] = c.s * inv;
}

// ---- backward ---------------------------------------------------------------------------------------------------------
struct Grad {
  const void *dy, *h, *dres;
  const float* gain;
  void* dx;
  float* part;               // [gridDim.x][K]: each block's sums of dg; null where they are not asked for
  int64_t lddy, ldh, lddres, lddx, R, K;
  float eps;
  int n, acc_shared;         // acc_shared (long rows): the block's sums lie in shared memory
};

template <typename TD, typename TH, int NV, int MAXT, bool AHEAD, bool WIDE>
__global__ void __launch_bounds__(MAXT) rms_norm_backward_kernel(const __grid_constant__ Grad p) {
  __shared__ Exchange ex;
  extern __shared__ float joined[];          // several rows at a time: [rows][K]
  const int n = p.n, t = threadIdx.x & (n - 1), rows = blockDim.x / n;
  const int64_t step = static_cast<int64_t>(gridDim.x) * rows;
  int turn = 0;
  pdl_trigger();
  pdl_wait();
  float g[NV][8], acc[NV][8];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    gain8<WIDE>(p.gain, t, j, n, p.K, g[j]);
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[j][i] = 0.f;
  }
  Raw8<TD> dy[NV];
  Raw8<TH> h[NV];
  auto fetch = [&](int64_t r) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      dy[j].clear();
      h[j].clear();
      if (r < p.R) {
        load8<WIDE>(static_cast<const TD*>(p.dy) + r * p.lddy, t, j, n, p.K, dy[j]);
        load8<WIDE>(static_cast<const TH*>(p.h) + r * p.ldh, t, j, n, p.K, h[j]);
      }
    }
  };
  int64_t r = blockIdx.x * static_cast<int64_t>(rows) + threadIdx.x / n;
  if (AHEAD) fetch(r);
  for (int64_t base = blockIdx.x * static_cast<int64_t>(rows); base < p.R; base += step, r += step) {
    if (!AHEAD) fetch(r);
    Raw8<TD> d[NV];
    Raw8<TH> z[NV], dres[NV];
    float sum = 0.f, dot = 0.f;
    uint32_t unused = 0;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      d[j] = dy[j];
      z[j] = h[j];
      if (p.dres && r < p.R) load8<WIDE>(static_cast<const TH*>(p.dres) + r * p.lddres, t, j, n, p.K, dres[j]);
      else dres[j].clear();
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        sum = fmaf(z[j].at(i), z[j].at(i), sum);
        dot = fmaf(d[j].at(i) * g[j][i], z[j].at(i), dot);
      }
    }
    if (AHEAD) fetch(r + step);
    over_row<true, false>(ex, turn, n, sum, dot, unused);
    float small = 1.f, inv = root(sum, static_cast<float>(p.K), p.eps);
    if (sum == CUDART_INF_F) {
      sum = dot = 0.f;
      small = SMALLER;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float v = z[j].at(i) * SMALLER;
          sum = fmaf(v, v, sum);
          dot = fmaf(d[j].at(i) * g[j][i], v, dot);
        }
      over_row<true, false>(ex, turn, n, sum, dot, unused);
      inv = root(sum, static_cast<float>(p.K), 0.f);
    }
    const float mean = __fdiv_rn(dot, static_cast<float>(p.K)) * inv, outer = inv * small;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float unit = z[j].at(i) * small * inv;
        v[i] = fmaf(outer, fmaf(-unit, mean, d[j].at(i) * g[j][i]), dres[j].at(i));
        acc[j][i] = fmaf(d[j].at(i), unit, acc[j][i]);
      }
      if (r < p.R) {
        Raw8<TH> o;
        o.set(v);
        store8<WIDE>(static_cast<TH*>(p.dx) + r * p.lddx, t, j, n, p.K, o);
      }
    }
  }
  if (!p.part) return;
  float* out = p.part + blockIdx.x * p.K;
  if (rows == 1) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t c = column<WIDE>(t, j, n, i);
        if (c < p.K) out[c] = acc[j][i];
      }
    return;
  }
  float* mine = joined + (threadIdx.x / n) * p.K;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t c = column<WIDE>(t, j, n, i);
      if (c < p.K) mine[c] = acc[j][i];
    }
  __syncthreads();
  for (int64_t c = threadIdx.x; c < p.K; c += blockDim.x) {
    float s = 0.f;
    for (int k = 0; k < rows; ++k) s += joined[k * p.K + c];
    out[c] = s;
  }
}

// Rows too long for registers: read a second time, the block's sums of dg in shared memory or, longer than that, in its row of `part`.
template <typename TD, typename TH, bool WIDE>
__global__ void __launch_bounds__(1024) rms_norm_backward_long_kernel(const __grid_constant__ Grad p) {
  __shared__ Exchange ex;
  extern __shared__ float shared_acc[];
  const int n = p.n, t = threadIdx.x;
  const int64_t vectors = (p.K + 8 * n - 1) / (8 * n);
  int turn = 0;
  pdl_trigger();
  pdl_wait();
  float* out = p.part ? p.part + blockIdx.x * p.K : nullptr;
  float* acc = p.part && p.acc_shared ? shared_acc : out;
  if (acc)
    for (int64_t j = 0; j < vectors; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t c = column<WIDE>(t, j, n, i);
        if (c < p.K) acc[c] = 0.f;
      }
  for (int64_t r = blockIdx.x; r < p.R; r += gridDim.x) {
    const TD* dy = static_cast<const TD*>(p.dy) + r * p.lddy;
    const TH* h = static_cast<const TH*>(p.h) + r * p.ldh;
    float small = 1.f, inv = 0.f, sum, dot, g[8];
    uint32_t unused = 0;
    for (int pass = 0; pass < 2; ++pass) {
      sum = dot = 0.f;
      for (int64_t j = 0; j < vectors; ++j) {
        Raw8<TD> d;
        Raw8<TH> z;
        load8<WIDE>(dy, t, j, n, p.K, d);
        load8<WIDE>(h, t, j, n, p.K, z);
        gain8<WIDE>(p.gain, t, j, n, p.K, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float v = z.at(i) * small;
          sum = fmaf(v, v, sum);
          dot = fmaf(d.at(i) * g[i], v, dot);
        }
      }
      over_row<true, false>(ex, turn, n, sum, dot, unused);
      inv = root(sum, static_cast<float>(p.K), pass ? 0.f : p.eps);
      if (sum != CUDART_INF_F) break;
      small = SMALLER;
    }
    const float mean = __fdiv_rn(dot, static_cast<float>(p.K)) * inv, outer = inv * small;
    for (int64_t j = 0; j < vectors; ++j) {
      Raw8<TD> d;
      Raw8<TH> z, dres, o;
      float v[8];
      load8<WIDE>(dy, t, j, n, p.K, d);
      load8<WIDE>(h, t, j, n, p.K, z);
      if (p.dres) load8<WIDE>(static_cast<const TH*>(p.dres) + r * p.lddres, t, j, n, p.K, dres);
      else dres.clear();
      gain8<WIDE>(p.gain, t, j, n, p.K, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float unit = z.at(i) * small * inv;
        v[i] = fmaf(outer, fmaf(-unit, mean, d.at(i) * g[i]), dres.at(i));
        const int64_t c = column<WIDE>(t, j, n, i);
        if (acc && c < p.K) acc[c] = fmaf(d.at(i), unit, acc[c]);
      }
      o.set(v);
      store8<WIDE>(static_cast<TH*>(p.dx) + r * p.lddx, t, j, n, p.K, o);
    }
  }
  if (acc && acc != out)
    for (int64_t j = 0; j < vectors; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t c = column<WIDE>(t, j, n, i);
        if (c < p.K) out[c] = acc[c];
      }
}

// dg = the blocks' sums, added in the order of the blocks within eight strands.
__global__ void __launch_bounds__(256) gain_sums_kernel(const float* part, int slots, int64_t K, float* d_gain) {
  __shared__ float strand[8][33];
  const int l = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int64_t c = blockIdx.x * 32ll + l;
  pdl_trigger();
  pdl_wait();
  float s = 0.f;
  if (c < K) {
#pragma unroll 4
    for (int k = w; k < slots; k += 8) s += part[k * K + c];
  }
  strand[w][l] = s;
  __syncthreads();
  if (w == 0 && c < K) {
    s = strand[0][l];
#pragma unroll
    for (int k = 1; k < 8; ++k) s += strand[k][l];
    d_gain[c] = s;
  }
}

// ---- launches ---------------------------------------------------------------------------------------------------------
constexpr int64_t IN_REGISTERS = 8192, IN_REGISTERS_SLOWLY = 32768;   // longest rows of the two forms

int pow2_threads(int64_t want, int most) {
  int n = 32;
  while (n < want && n < most) n *= 2;
  return n;
}

template <typename TX, typename TR, bool RES, bool WIDE>
cudaError_t launch_norm(Norm p, int sms, cudaStream_t stream) {
  if (p.K > IN_REGISTERS_SLOWLY) {
    p.n = 1024;
    return launch_pdl(rms_norm_long_kernel<TX, TR, RES, WIDE>, dim3(static_cast<unsigned>(p.R)), dim3(1024), 0, stream, 1, p);
  }
  if (p.K > IN_REGISTERS) {
    p.n = 1024;
    const int64_t grid = p.R < 2 * sms ? p.R : 2 * sms;
    return launch_pdl(rms_norm_kernel<TX, TR, RES, 4, 1024, false, WIDE>, dim3(static_cast<unsigned>(grid)), dim3(1024), 0, stream, 1, p);
  }
  if (p.R < 2 * sms) {                       // few rows: a vector a thread, for the latency
    p.n = pow2_threads((p.K + 7) / 8, 1024);
    return launch_pdl(rms_norm_kernel<TX, TR, RES, 1, 1024, false, WIDE>, dim3(static_cast<unsigned>(p.R)), dim3(p.n), 0, stream, 1, p);
  }
  p.n = pow2_threads((p.K + 15) / 16, 512);
  const int rows = p.n == 32 ? 4 : 1, threads = p.n * rows;
  const int64_t want = (p.R + rows - 1) / rows, most = static_cast<int64_t>(sms) * (1024 / threads < 16 ? 1024 / threads : 16);
  return launch_pdl(rms_norm_kernel<TX, TR, RES, 2, 512, true, WIDE>, dim3(static_cast<unsigned>(want < most ? want : most)), dim3(threads), 0, stream, 1, p);
}

template <typename TD, typename TH, bool WIDE>
cudaError_t launch_backward(Grad p, int sms, float* d_gain, cudaStream_t stream) {
  int64_t grid;
  cudaError_t e;
  if (p.K > IN_REGISTERS) {
    p.n = 1024;
    grid = p.R < sms ? p.R : sms;
    const size_t bytes = static_cast<size_t>(p.K) * 4;
    p.acc_shared = p.part && bytes <= 200 * 1024;
    const auto kernel = rms_norm_backward_long_kernel<TD, TH, WIDE>;
    if (p.acc_shared && bytes > 40 * 1024 &&
        (e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024)) != cudaSuccess) return e;
    e = launch_pdl(kernel, dim3(static_cast<unsigned>(grid)), dim3(1024), p.acc_shared ? bytes : 0, stream, 1, p);
  } else {
    p.n = pow2_threads((p.K + 15) / 16, 512);
    const int rows = p.n == 32 ? 4 : 1, threads = p.n * rows;
    const int64_t want = (p.R + rows - 1) / rows, most = static_cast<int64_t>(sms) * (512 / threads < 4 ? 512 / threads : 4);
    grid = want < most ? want : most;
    e = launch_pdl(rms_norm_backward_kernel<TD, TH, 2, 512, true, WIDE>, dim3(static_cast<unsigned>(grid)), dim3(threads),
                   rows > 1 ? static_cast<size_t>(rows) * p.K * 4 : 0, stream, 1, p);
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
  Norm p{X_dev, residual_dev, gain_dev, H_dev, Y_dev, Q_dev, scale_dev, ldx, ldres, ldh, ldy, ldq, R, K, static_cast<float>(eps), y_bf16 != 0, 0};
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
  if (sms > MBD_NORM_SCRATCH_ROWS / 4) sms = MBD_NORM_SCRATCH_ROWS / 4;
  const Grad p{dY_dev, H_dev, d_residual_dev, gain_dev, dX_dev, d_gain_dev ? scratch_dev : nullptr, lddy, ldh, lddres, lddx, R, K, static_cast<float>(eps), 0, 0};
  const bool wide = K % 8 == 0 && dy.wide() && h.wide() && dres.wide() && dx.wide();
  cudaError_t e;
  if (dy_bf16 && h_bf16) e = wide ? launch_backward<bf16, bf16, true>(p, sms, d_gain_dev, stream) : launch_backward<bf16, bf16, false>(p, sms, d_gain_dev, stream);
  else if (dy_bf16) e = wide ? launch_backward<bf16, float, true>(p, sms, d_gain_dev, stream) : launch_backward<bf16, float, false>(p, sms, d_gain_dev, stream);
  else if (h_bf16) e = wide ? launch_backward<float, bf16, true>(p, sms, d_gain_dev, stream) : launch_backward<float, bf16, false>(p, sms, d_gain_dev, stream);
  else e = wide ? launch_backward<float, float, true>(p, sms, d_gain_dev, stream) : launch_backward<float, float, false>(p, sms, d_gain_dev, stream);
  return done(e);
}
