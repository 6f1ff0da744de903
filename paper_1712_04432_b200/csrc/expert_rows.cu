// The rows of a batch to the experts and back, around the products grouped by expert.  places[t, j] is the row, among the rows sorted by
// expert, of token t's j-th slot; a place outside [0, rows) is an empty slot.
//
//   dispatch          out[places[t, j]] = x[t]                     (the bits as they are, with the rows' scales if there are any)
//   combine           out[t] = residual[t] + sum_j w[t, j] y[places[t, j]]           in float, j ascending, one rounding
//   combine backward  dy[places[t, j]] = w[t, j] d_out[t],   dw[t, j] = <d_out[t], y[places[t, j]]>
//   dispatch backward is combine without weights.
//
// All of them go by token: the token's row passes once and its k rows elsewhere once each, whole rows at a time, so the order of the
// places costs nothing.  HBM bounds them.
#include "../../include/mbd.h"
#include "vec8.cuh"

namespace mbd {
namespace {

typedef __nv_bfloat16 bf16;

struct Dispatch {
  const unsigned char* x;
  unsigned char* out;
  const float* scale;
  float* out_scale;
  const int32_t* places;
  int64_t ldx, ldo, row;       // bytes
  int64_t T, rows;
  int k, n;                    // n: threads per token
};

template <typename V> __device__ __forceinline__ V get(const unsigned char* p) { return *reinterpret_cast<const V*>(p); }

// V: the widest type that all addresses, strides and the row's length are multiples of.  Four of them a thread on their way at once: 8192 tokens to two
// places, 4096 bf16 columns, 32 us (6.3 TB/s).
template <typename V>
__global__ void __launch_bounds__(256) dispatch_kernel(const __grid_constant__ Dispatch p) {
  constexpr int AT_ONCE = 4;
  pdl_trigger();
  pdl_wait();
  const int n = p.n, l = threadIdx.x & (n - 1);
  const int64_t t = (blockIdx.x * static_cast<int64_t>(blockDim.x) + threadIdx.x) / n;
  if (t >= p.T) return;
  const int32_t* places = p.places + t * p.k;
  const unsigned char* x = p.x + t * p.ldx;
  const int64_t count = p.row / static_cast<int64_t>(sizeof(V));
  for (int64_t first = l; first < count; first += AT_ONCE * n) {
    V v[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i)
      if (first + i * n < count) v[i] = get<V>(x + (first + i * n) * sizeof(V));
    for (int j = 0; j < p.k; ++j) {
      const int64_t at = places[j];
      if (at < 0 || at >= p.rows) continue;
      unsigned char* to = p.out + at * p.ldo;
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i)
        if (first + i * n < count) *reinterpret_cast<V*>(to + (first + i * n) * sizeof(V)) = v[i];
    }
  }
  if (p.scale)
    for (int j = l; j < p.k; j += n) {
      const int64_t at = places[j];
      if (at >= 0 && at < p.rows) p.out_scale[at] = p.scale[t];
    }
}

constexpr int MAX_K = 32;
constexpr int NARROW = 128;    // threads a token where rows move element by element: offsets between a thread's columns are constants then

struct Combine {
  const void* y;
  const int32_t* places;
  const float* weights;
  const void* res;
  void* out;
  int64_t ldy, ldres, ldo, T, rows;
  int K, k, n;
};

// NV vectors of a thread and two slots are on their way together: the row of places, then 3 NV loads, then the sums.  For more than four slots
// (8192 tokens of 8, 1024 columns: 31 us, 4.9 TB/s) and for rows that move element by element.
template <typename TY, typename TO, int NV, bool WIDE>
__global__ void __launch_bounds__(512) combine_kernel(const __grid_constant__ Combine p) {
  pdl_trigger();
  pdl_wait();
  const int n = WIDE ? p.n : NARROW, l = threadIdx.x & (n - 1);
  const int64_t t = (blockIdx.x * static_cast<int64_t>(blockDim.x) + threadIdx.x) / n;
  if (t >= p.T) return;
  const int32_t* places = p.places + t * p.k;
  const float* weights = p.weights ? p.weights + t * p.k : nullptr;
  const TO* res_row = p.res ? static_cast<const TO*>(p.res) + t * p.ldres : nullptr;
  TO* out_row = static_cast<TO*>(p.out) + t * p.ldo;
  const int vectors = (p.K + 8 * n - 1) / (8 * n);
  for (int c = 0; c < vectors; c += NV) {
    f32x2 sum[NV][4];
    Raw8<TO> res[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      res[v].clear();
      if (res_row) load8<WIDE>(res_row, l, c + v, n, p.K, res[v]);
    }
    for (int j = 0; j < p.k; j += 2) {
      const int64_t a = places[j], b = j + 1 < p.k ? places[j + 1] : -1;
      const bool there_a = a >= 0 && a < p.rows, there_b = b >= 0 && b < p.rows;
      const float wa = there_a && weights ? weights[j] : 1.f, wb = there_b && weights ? weights[j + 1] : 1.f;
      Raw8<TY> ya[NV], yb[NV];
      if (there_a) {
#pragma unroll
        for (int v = 0; v < NV; ++v) load8<WIDE>(static_cast<const TY*>(p.y) + a * p.ldy, l, c + v, n, p.K, ya[v]);
      }
      if (there_b) {
#pragma unroll
        for (int v = 0; v < NV; ++v) load8<WIDE>(static_cast<const TY*>(p.y) + b * p.ldy, l, c + v, n, p.K, yb[v]);
      }
      if (j == 0) {
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int i = 0; i < 4; ++i) sum[v][i] = res[v].two(i);
      }
      if (there_a) {                                       // (an empty slot adds nothing, whatever its weight)
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int i = 0; i < 4; ++i) sum[v][i] = fma2(pair(wa, wa), ya[v].two(i), sum[v][i]);
      }
      if (there_b) {
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int i = 0; i < 4; ++i) sum[v][i] = fma2(pair(wb, wb), yb[v].two(i), sum[v][i]);
      }
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float f[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 s = floats(sum[v][i]);
        f[2 * i] = s.x;
        f[2 * i + 1] = s.y;
      }
      Raw8<TO> o;
      o.set(f);
      store8<WIDE>(out_row, l, c + v, n, p.K, o);
    }
  }
}

// Up to SLOTS slots in whole vectors, all of a thread's loads under way at once and no sums held between them (8192 tokens of two
// slots, 4096 bf16 columns: 42 us, by the kernel above 51).
template <typename TY, typename TO, int NV, int SLOTS>
__global__ void __launch_bounds__(512) combine_slots_kernel(const __grid_constant__ Combine p) {
  pdl_trigger();
  pdl_wait();
  const int n = p.n, l = threadIdx.x & (n - 1);
  const int64_t t = (blockIdx.x * static_cast<int64_t>(blockDim.x) + threadIdx.x) / n;
  if (t >= p.T) return;
  const TO* res_row = p.res ? static_cast<const TO*>(p.res) + t * p.ldres : nullptr;
  TO* out_row = static_cast<TO*>(p.out) + t * p.ldo;
  const TY* row[SLOTS];
  float w[SLOTS];
#pragma unroll
  for (int j = 0; j < SLOTS; ++j) {
    const int64_t at = j < p.k ? p.places[t * p.k + j] : -1;
    row[j] = at >= 0 && at < p.rows ? static_cast<const TY*>(p.y) + at * p.ldy : nullptr;
    w[j] = row[j] && p.weights ? p.weights[t * p.k + j] : 1.f;
  }
  const int vectors = (p.K + 8 * n - 1) / (8 * n);
  for (int c = 0; c < vectors; c += NV) {
    Raw8<TO> res[NV];
    Raw8<TY> y[SLOTS][NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      res[v].clear();
      if (res_row) load8<true>(res_row, l, c + v, n, p.K, res[v]);
    }
#pragma unroll
    for (int j = 0; j < SLOTS; ++j)
      if (row[j]) {
#pragma unroll
        for (int v = 0; v < NV; ++v) load8<true>(row[j], l, c + v, n, p.K, y[j][v]);
      }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      f32x2 sum[4];
      float f[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[i] = res[v].two(i);
#pragma unroll
      for (int j = 0; j < SLOTS; ++j)
        if (row[j]) {                                      // (an empty slot adds nothing, whatever its weight)
#pragma unroll
          for (int i = 0; i < 4; ++i) sum[i] = fma2(pair(w[j], w[j]), y[j][v].two(i), sum[i]);
        }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 s = floats(sum[i]);
        f[2 * i] = s.x;
        f[2 * i + 1] = s.y;
      }
      Raw8<TO> o;
      o.set(f);
      store8<true>(out_row, l, c + v, n, p.K, o);
    }
  }
}

struct CombineGrad {
  const void* d_out;
  const void* y;
  const int32_t* places;
  const float* weights;
  void* dy;
  float* dw;
  int64_t ldd, ldy, lddy, T, rows;
  int K, k, n;                    // n >= 32 threads per token, n / 32 warps; n > 32: the block has one token
};

// The rows of SLOTS slots are on their way together; each thread adds up its part of their dot products over the whole row, the threads meet
// once per SLOTS slots.  8192 tokens of two slots, 4096 bf16 columns: 58 us (5.8 TB/s).  (Four slots at a time took as long as two: 5003 tokens
// of four, 1000 columns, 18 us.)
template <typename TD, typename TY, int NV, bool WIDE>
__global__ void __launch_bounds__(512) combine_backward_kernel(const __grid_constant__ CombineGrad p) {
  constexpr int SLOTS = 2;
  __shared__ float dots[16][MAX_K];
  pdl_trigger();
  pdl_wait();
  const int n = WIDE ? p.n : NARROW, l = threadIdx.x & (n - 1), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t t = (blockIdx.x * static_cast<int64_t>(blockDim.x) + threadIdx.x) / n;
  if (t >= p.T) return;                                  // (the same for a warp, and for a block that has one token)
  const TD* d_row = static_cast<const TD*>(p.d_out) + t * p.ldd;
  const int vectors = (p.K + 8 * n - 1) / (8 * n);
  const int64_t place = lane < p.k ? p.places[t * p.k + lane] : -1;
  const float weight = lane < p.k ? p.weights[t * p.k + lane] : 0.f;
  float dot = 0.f;                                       // lane j: this warp's part of slot j
  Raw8<TD> d[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) load8<WIDE>(d_row, l, v, n, p.K, d[v]);
  for (int j0 = 0; j0 < p.k; j0 += SLOTS) {
    int64_t at[SLOTS];
    float w[SLOTS];
    bool there[SLOTS];
    f32x2 s[SLOTS];
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
      at[j] = __shfl_sync(0xffffffffu, place, (j0 + j) & 31);
      w[j] = __shfl_sync(0xffffffffu, weight, (j0 + j) & 31);
      there[j] = j0 + j < p.k && at[j] >= 0 && at[j] < p.rows;
      s[j] = pair(0.f, 0.f);
    }
    for (int c = 0; c < vectors; c += NV) {
      if (vectors > NV) {                                // a row longer than the registers: read again for each group of slots
#pragma unroll
        for (int v = 0; v < NV; ++v) load8<WIDE>(d_row, l, c + v, n, p.K, d[v]);
      }
      Raw8<TY> y[SLOTS][NV];
      if (p.dw) {
#pragma unroll
        for (int j = 0; j < SLOTS; ++j)
          if (there[j]) {
#pragma unroll
            for (int v = 0; v < NV; ++v) load8<WIDE>(static_cast<const TY*>(p.y) + at[j] * p.ldy, l, c + v, n, p.K, y[j][v]);
          }
      }
#pragma unroll
      for (int j = 0; j < SLOTS; ++j)
        if (there[j]) {
          TY* to = static_cast<TY*>(p.dy) + at[j] * p.lddy;
#pragma unroll
          for (int v = 0; v < NV; ++v) {
            float f[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float2 o = floats(mul2(pair(w[j], w[j]), d[v].two(i)));
              f[2 * i] = o.x;
              f[2 * i + 1] = o.y;
              if (p.dw) s[j] = fma2(d[v].two(i), y[j][v].two(i), s[j]);
            }
            Raw8<TY> o;
            o.set(f);
            store8<WIDE>(to, l, c + v, n, p.K, o);
          }
        }
    }
    if (p.dw) {
#pragma unroll
      for (int j = 0; j < SLOTS; ++j) {
        const float2 f = floats(s[j]);
        float total = f.x + f.y;
#pragma unroll
        for (int m = 16; m > 0; m >>= 1) total += __shfl_xor_sync(0xffffffffu, total, m);
        if (lane == j0 + j) dot = total;
      }
    }
  }
  if (!p.dw) return;
  if (n > 32) {
    dots[warp][lane] = dot;
    __syncthreads();
    if (warp > 0) return;
    dot = dots[0][lane];
    for (int w = 1; w < n >> 5; ++w) dot += dots[w][lane];
  }
  if (lane < p.k) p.dw[t * p.k + lane] = dot;
}

// ---- launches ---------------------------------------------------------------------------------------------------------
int threads_for(int64_t work_items, int most) {
  int n = 32;
  while (n < work_items && n < most) n *= 2;
  return n;
}

template <typename V> cudaError_t launch(Dispatch p, cudaStream_t stream) {
  p.n = threads_for(p.row / static_cast<int64_t>(sizeof(V)) / 4, 256);
  const int threads = p.n < 128 ? 128 : p.n;
  const int64_t grid = (p.T * p.n + threads - 1) / threads;
  return launch_pdl(dispatch_kernel<V>, dim3(static_cast<unsigned>(grid)), dim3(threads), 0, stream, 1, p);
}

// Vectors of a thread: few tokens have one, for the latency; many have so many that about 200 bytes of a thread are on their way, but 32
// threads have something to do.
constexpr int64_t FEW = 512;
int vectors_for(int64_t T, int64_t K, int bytes) {
  if (T < FEW || K < 512) return 1;
  return bytes == 2 && K >= 1024 ? 4 : 2;
}

template <typename TY, typename TO> cudaError_t launch(Combine p, bool wide, cudaStream_t stream) {
  constexpr int MORE = sizeof(TY) == 2 ? 4 : 2;
  int nv = vectors_for(p.T, p.K, sizeof(TY));
  if (p.k > 2 && nv == 4) nv = 2;
  p.n = wide ? threads_for((p.K + 8 * nv - 1) / (8 * nv), nv == 1 ? 512 : 256) : NARROW;
  const int threads = p.n < 128 ? 128 : p.n;
  const dim3 grid(static_cast<unsigned>((p.T * p.n + threads - 1) / threads)), block(threads);
  if (!wide) return launch_pdl(combine_kernel<TY, TO, 1, false>, grid, block, 0, stream, 1, p);
  if (p.k <= 2) {
    if (nv == 1) return launch_pdl(combine_slots_kernel<TY, TO, 1, 2>, grid, block, 0, stream, 1, p);
    if (nv == 2) return launch_pdl(combine_slots_kernel<TY, TO, 2, 2>, grid, block, 0, stream, 1, p);
    return launch_pdl(combine_slots_kernel<TY, TO, MORE, 2>, grid, block, 0, stream, 1, p);
  }
  if (p.k <= 4) {
    if (nv == 1) return launch_pdl(combine_slots_kernel<TY, TO, 1, 4>, grid, block, 0, stream, 1, p);
    return launch_pdl(combine_slots_kernel<TY, TO, MORE / 2, 4>, grid, block, 0, stream, 1, p);
  }
  if (nv == 1) return launch_pdl(combine_kernel<TY, TO, 1, true>, grid, block, 0, stream, 1, p);
  return launch_pdl(combine_kernel<TY, TO, 2, true>, grid, block, 0, stream, 1, p);
}

template <typename TD, typename TY> cudaError_t launch(CombineGrad p, bool wide, cudaStream_t stream) {
  const int nv = vectors_for(p.T, p.K, 4);               // (two already: results leave as fast as rows come)
  p.n = wide ? threads_for((p.K + 8 * nv - 1) / (8 * nv), nv == 1 ? 512 : 256) : NARROW;
  const int threads = p.n == 32 ? 128 : p.n;
  const dim3 grid(static_cast<unsigned>((p.T * p.n + threads - 1) / threads)), block(threads);
  if (!wide) return launch_pdl(combine_backward_kernel<TD, TY, 1, false>, grid, block, 0, stream, 1, p);
  if (nv == 1) return launch_pdl(combine_backward_kernel<TD, TY, 1, true>, grid, block, 0, stream, 1, p);
  return launch_pdl(combine_backward_kernel<TD, TY, 2, true>, grid, block, 0, stream, 1, p);
}

mbd_status done(cudaError_t e) {
  if (e == cudaSuccess) return MBD_OK;
  (void)cudaGetLastError();
  return MBD_E_CUDA;
}

// Sizes all three share.  rows: of the tensor sorted by expert.
mbd_status sizes(int64_t T, int k, int64_t K, int64_t rows) {
  if (T < 0 || K < 1 || k < 1 || rows < 0) return MBD_E_INVALID;
  if (k > MAX_K || T > INT32_MAX || rows > INT32_MAX || K > INT32_MAX - 65536) return MBD_E_UNSUPPORTED;
  return MBD_OK;
}

}  // namespace
}  // namespace mbd

using namespace mbd;

extern "C" mbd_status mbd_expert_dispatch(int64_t T, int k, int64_t K, int element_bytes, const void* X_dev, int64_t ldx, const float* scale_dev,
                                          const int32_t* places_dev, int64_t rows, void* out_dev, int64_t ldo, float* out_scale_dev,
                                          void* cuda_stream) {
  if (element_bytes != 1 && element_bytes != 2 && element_bytes != 4) return MBD_E_INVALID;
  const mbd_status st = sizes(T, k, K, rows);
  if (st != MBD_OK) return st;
  if (T == 0 || rows == 0) return MBD_OK;
  if (!X_dev || !places_dev || !out_dev || !scale_dev != !out_scale_dev) return MBD_E_INVALID;
  if ((T > 1 && ldx < K) || (rows > 1 && ldo < K)) return MBD_E_INVALID;
  const Rows x{X_dev, T, K, ldx, element_bytes}, out{out_dev, rows, K, ldo, element_bytes}, places{places_dev, 1, T * k, T * k, 4},
      scale{scale_dev, 1, T, T, 4}, out_scale{out_scale_dev, 1, rows, rows, 4};
  for (const Rows* t : {&x, &out, &places, &scale, &out_scale})
    if (t->misplaced()) return MBD_E_UNSUPPORTED;
  for (const Rows* t : {&x, &places, &scale})
    if (!apart(out, *t) || !apart(out_scale, *t)) return MBD_E_INVALID;
  if (!apart(out, out_scale)) return MBD_E_INVALID;
  const Dispatch p{static_cast<const unsigned char*>(X_dev), static_cast<unsigned char*>(out_dev), scale_dev, out_scale_dev, places_dev,
                   ldx * element_bytes, ldo * element_bytes, K * element_bytes, T, rows, k, 0};
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const uint64_t all = reinterpret_cast<uintptr_t>(X_dev) | reinterpret_cast<uintptr_t>(out_dev) | static_cast<uint64_t>(p.row) |
                       (T > 1 ? static_cast<uint64_t>(p.ldx) : 0u) | (rows > 1 ? static_cast<uint64_t>(p.ldo) : 0u);
  return done(all % 16 == 0 ? launch<uint4>(p, stream) : all % 8 == 0 ? launch<uint2>(p, stream) : all % 4 == 0 ? launch<uint32_t>(p, stream)
              : all % 2 == 0 ? launch<uint16_t>(p, stream) : launch<uint8_t>(p, stream));
}

extern "C" mbd_status mbd_expert_combine(int64_t T, int k, int64_t K, const void* Y_dev, int y_bf16, int64_t ldy, int64_t rows,
                                         const int32_t* places_dev, const float* weights_dev, const void* residual_dev, int64_t ldres,
                                         void* out_dev, int out_bf16, int64_t ldo, void* cuda_stream) {
  const mbd_status st = sizes(T, k, K, rows);
  if (st != MBD_OK) return st;
  if (T == 0) return MBD_OK;
  if ((!Y_dev && rows > 0) || !places_dev || !out_dev) return MBD_E_INVALID;
  if ((rows > 1 && ldy < K) || (T > 1 && (ldo < K || (residual_dev && ldres < K)))) return MBD_E_INVALID;
  const int osize = out_bf16 ? 2 : 4;
  const Rows y{rows > 0 ? Y_dev : nullptr, rows, K, ldy, y_bf16 ? 2 : 4}, res{residual_dev, T, K, ldres, osize}, out{out_dev, T, K, ldo, osize},
      places{places_dev, 1, T * k, T * k, 4}, weights{weights_dev, 1, T * k, T * k, 4};
  for (const Rows* t : {&y, &res, &out, &places, &weights})
    if (t->misplaced()) return MBD_E_UNSUPPORTED;
  if (!apart(out, y) || !apart(out, places) || !apart(out, weights) || !apart_or_same(out, res)) return MBD_E_INVALID;
  const Combine p{Y_dev, places_dev, weights_dev, residual_dev, out_dev, ldy, ldres, ldo, T, rows, static_cast<int>(K), k, 0};
  const bool wide = K % 8 == 0 && y.wide() && res.wide() && out.wide();
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  return done(y_bf16 ? (out_bf16 ? launch<bf16, bf16>(p, wide, stream) : launch<bf16, float>(p, wide, stream))
                     : (out_bf16 ? launch<float, bf16>(p, wide, stream) : launch<float, float>(p, wide, stream)));
}

extern "C" mbd_status mbd_expert_combine_backward(int64_t T, int k, int64_t K, const void* d_out_dev, int d_out_bf16, int64_t ldd,
                                                  const void* Y_dev, int y_bf16, int64_t ldy, int64_t rows, const int32_t* places_dev,
                                                  const float* weights_dev, void* dY_dev, int64_t lddy, float* d_weights_dev, void* cuda_stream) {
  const mbd_status st = sizes(T, k, K, rows);
  if (st != MBD_OK) return st;
  if (T == 0) return MBD_OK;
  if (!d_out_dev || !places_dev || !weights_dev || (rows > 0 && (!dY_dev || (d_weights_dev && !Y_dev)))) return MBD_E_INVALID;
  if ((T > 1 && ldd < K) || (rows > 1 && (lddy < K || (d_weights_dev && ldy < K)))) return MBD_E_INVALID;
  const int ysize = y_bf16 ? 2 : 4;
  const Rows d{d_out_dev, T, K, ldd, d_out_bf16 ? 2 : 4}, y{d_weights_dev && rows > 0 ? Y_dev : nullptr, rows, K, ldy, ysize},
      dy{rows > 0 ? dY_dev : nullptr, rows, K, lddy, ysize}, places{places_dev, 1, T * k, T * k, 4}, weights{weights_dev, 1, T * k, T * k, 4},
      dw{d_weights_dev, 1, T * k, T * k, 4};
  for (const Rows* t : {&d, &y, &dy, &places, &weights, &dw})
    if (t->misplaced()) return MBD_E_UNSUPPORTED;
  if (!apart_or_same(dy, y)) return MBD_E_INVALID;
  for (const Rows* t : {&d, &places, &weights})
    if (!apart(dy, *t) || !apart(dw, *t)) return MBD_E_INVALID;
  if (!apart(dw, y) || !apart(dw, dy)) return MBD_E_INVALID;
  const CombineGrad p{d_out_dev, Y_dev, places_dev, weights_dev, dY_dev, d_weights_dev, ldd, ldy, lddy, T, rows, static_cast<int>(K), k, 0};
  const bool wide = K % 8 == 0 && d.wide() && y.wide() && dy.wide();
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  return done(d_out_bf16 ? (y_bf16 ? launch<bf16, bf16>(p, wide, stream) : launch<bf16, float>(p, wide, stream))
                         : (y_bf16 ? launch<float, bf16>(p, wide, stream) : launch<float, float>(p, wide, stream)));
}
