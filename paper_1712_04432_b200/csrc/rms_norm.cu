// Root-mean-square norm of rows, with the residual's addition in front and rows in 16, 32 or 8 bits behind.
//
//   h = x (+ residual, rounded to the residual's type),  r = 1 / sqrt(mean(h^2) + eps),  y = h r g
//   in 8 bits: u = h g in float, s = max |u| / 127, q = u / s rounded to an integer, scale = s r.  r is the same for all of a row, so it goes
//   into the scale: q needs the row's largest |u| only and does not depend on the order in which the squares are added.
//
// Each tensor passes once: the row stays in registers between the sum and the result.  HBM bounds large calls, latency small ones.
#include "quotients.cuh"
#include "rms_norm.cuh"

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

// h of one vector, from what was loaded; with a residual it is rounded to the residual's type.
template <typename TX, typename TR, bool RES>
__device__ __forceinline__ Raw8<TR> stream8(const Raw8<TX>& x, const Raw8<TR>& res) {
  if constexpr (!RES && sizeof(TX) == sizeof(TR)) return x;
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
// shared memory, p.stages rows deep; the gain lies there too.  8192 x 4096 bf16 24 us (5.5 TB/s), in 8 bits 31 us: instructions bound that one.
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

// A row too long for registers and, in two stages, for shared memory: read a second time (1024 x 16384 bf16 with a residual in floats 44 us, 4.6 TB/s of
// what passes once; through the ring, one row a block, 2048 x 16384 bf16 take 35 us, 3.9 TB/s, with a residual 60, 4.5 TB/s).
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
// a residual 9.4 us, 10.4; 1000 x 1024 with one 2.5, 4.6); through the ring where there is less traffic (8192 x 4096 bf16 without a residual 24 us,
// directly 32; in 8 bits with one 43, 48).  Rows of more than 8192 values go through the ring if they fit, or else are read twice.
template <typename TX, typename TR, bool RES, bool WIDE>
cudaError_t launch_norm(Norm p, int sms, cudaStream_t stream) {
  constexpr bool RING = !RES || (sizeof(TX) == 2 && sizeof(TR) == 2);         // (a residual in or with floats is always much traffic)
  if (p.K <= 8192) {
    if (p.R < 2 * sms) {
      p.n = pow2_threads((p.K + 7) / 8, 1024);
      return launch_pdl(rms_norm_few_kernel<TX, TR, RES, WIDE>, dim3(static_cast<unsigned>(p.R)), dim3(p.n), 0, stream, 1, p);
    }
    const int bytes = static_cast<int>(sizeof(TX) + (RES ? (p.h ? 2 : 1) * sizeof(TR) : 0)) + (p.y ? (p.y_bf16 ? 2 : 4) : 0);
    if (!WIDE || !RING || (bytes >= 8 && !p.q) || p.R * p.K <= 10000000) return launch_direct<TX, TR, RES, WIDE>(p, stream);
  }
  if constexpr (WIDE && RING) {
    const Shape s = shape_of(p.K, 8 * static_cast<int>(sizeof(TX) + (RES ? sizeof(TR) : 0)), true, FORWARD_THREADS, 512);
    if (p.K <= LONGEST && s.stages) return launch_ring<TX, TR, RES>(p, s, sms, stream);
  }
  p.n = 1024;
  return launch_pdl(rms_norm_long_kernel<TX, TR, RES, WIDE>, dim3(static_cast<unsigned>(p.R)), dim3(1024), 0, stream, 1, p);
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
