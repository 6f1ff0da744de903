// Gradients of the root-mean-square norm of rows.
//
//   m = mean(dy g h r),  dh = r (dy g - h r m) (+ the gradient that arrives along the residual),  dg = sum over rows of dy h r,  r = 1 / sqrt(mean(h^2) + eps)
//
// Each tensor passes once.  The columns' sums of dg lie in the registers of the threads that own the columns, blocks taking row after row, which
// come through shared memory by asynchronous copies some rows ahead: a warp waits for its own copies only, and how much is under way does
// not depend on registers.  HBM bounds large calls, latency small ones.
#include "rms_norm.cuh"

namespace mbd {
namespace {

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
    if constexpr (!RING) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        load8<WIDE>(d_row, t, j, N, p.K, held_d[j]);
        load8<WIDE>(h_row, t, j, N, p.K, held_z[j]);
      }
    }
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

// Rows too long for registers, or of which two stages do not fit into shared memory (beyond 8192 columns all but bf16 without d_residual): read a second
// time, two vectors at a time on their way, the block's sums of dg in shared memory or, longer than that, in its row of `part`.  2048 x 16384 bf16 with
// d_residual 94 us, 2.9 TB/s of what passes once; 1024 x 16384 floats without 81, 2.5 TB/s; by the kernel above 2048 x 16384 bf16 without 60, 3.4 TB/s.
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

template <typename TD, typename TH, bool RING, bool WIDE>
cudaError_t launch_rows(const Grad& p, const Shape& s, int64_t grid, cudaStream_t stream) {
  const size_t joined = p.part ? static_cast<size_t>(s.rows) * s.nv * 8 * s.n * 4 : 0, bytes = s.bytes > joined ? s.bytes : joined;
  switch (s.nv * 1024 + s.n) {
    case 2 * 1024 + 32: return launch_shape<rms_norm_backward_kernel<TD, TH, 32, 2, RING, WIDE>>(p, s, bytes, grid, stream);
    case 2 * 1024 + 64: return launch_shape<rms_norm_backward_kernel<TD, TH, 64, 2, RING, WIDE>>(p, s, bytes, grid, stream);
    case 2 * 1024 + 128: return launch_shape<rms_norm_backward_kernel<TD, TH, 128, 2, RING, WIDE>>(p, s, bytes, grid, stream);
    case 2 * 1024 + 256: return launch_shape<rms_norm_backward_kernel<TD, TH, 256, 2, RING, WIDE>>(p, s, bytes, grid, stream);
    case 4 * 1024 + 256: return launch_shape<rms_norm_backward_kernel<TD, TH, 256, 4, RING, WIDE>>(p, s, bytes, grid, stream);
    default: break;
  }
  if constexpr (!RING || sizeof(TD) + sizeof(TH) == 4)        // (two stages of such rows with floats among them are more than a block has)
    return launch_shape<rms_norm_backward_kernel<TD, TH, 512, 4, RING, WIDE>>(p, s, bytes, grid, stream);
  return cudaErrorInvalidValue;
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

}  // namespace
}  // namespace mbd

using namespace mbd;
typedef __nv_bfloat16 bf16;

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
