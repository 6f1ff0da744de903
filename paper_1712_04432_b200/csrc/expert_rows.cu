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

// V: the widest type that all addresses, strides and the row's length are multiples of.
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

struct Combine {
  const void* y;
  const int32_t* places;
  const float* weights;
  const void* res;
  void* out;
  int64_t ldy, ldres, ldo, T, rows;
  int K, k, n;
};

template <typename TY, typename TO, bool WIDE>
__global__ void __launch_bounds__(256) combine_kernel(const __grid_constant__ Combine p) {
  constexpr int AT_ONCE = 4;
  pdl_trigger();
  pdl_wait();
  const int n = p.n, l = threadIdx.x & (n - 1);
  const int64_t t = (blockIdx.x * static_cast<int64_t>(blockDim.x) + threadIdx.x) / n;
  if (t >= p.T) return;
  const int32_t* places = p.places + t * p.k;
  const float* weights = p.weights ? p.weights + t * p.k : nullptr;
  const int vectors = (p.K + 8 * n - 1) / (8 * n);
  for (int c = 0; c < vectors; ++c) {
    float sum[8];
    Raw8<TO> res;
    res.clear();
    if (p.res) load8<WIDE>(static_cast<const TO*>(p.res) + t * p.ldres, l, c, n, p.K, res);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = res.at(i);
    for (int j0 = 0; j0 < p.k; j0 += AT_ONCE) {
      Raw8<TY> y[AT_ONCE];
      float w[AT_ONCE];
      bool there[AT_ONCE];
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) {
        const int64_t at = j0 + j < p.k ? places[j0 + j] : -1;
        there[j] = at >= 0 && at < p.rows;
        w[j] = there[j] && weights ? weights[j0 + j] : 1.f;
        if (there[j]) load8<WIDE>(static_cast<const TY*>(p.y) + at * p.ldy, l, c, n, p.K, y[j]);
      }
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j)
        if (there[j])                                    // an empty slot adds nothing, whatever its weight
#pragma unroll
          for (int i = 0; i < 8; ++i) sum[i] = fmaf(w[j], y[j].at(i), sum[i]);
    }
    Raw8<TO> o;
    o.set(sum);
    store8<WIDE>(static_cast<TO*>(p.out) + t * p.ldo, l, c, n, p.K, o);
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

constexpr int MAX_K = 32;

template <typename TD, typename TY, bool WIDE>
__global__ void __launch_bounds__(256) combine_backward_kernel(const __grid_constant__ CombineGrad p) {
  __shared__ float dots[8][MAX_K];
  pdl_trigger();
  pdl_wait();
  const int n = p.n, l = threadIdx.x & (n - 1), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t t = (blockIdx.x * static_cast<int64_t>(blockDim.x) + threadIdx.x) / n;
  const bool live = t < p.T;                             // (the same for a warp, and for a block that has one token)
  float dot = 0.f;                                       // lane j: this warp's part of slot j
  if (live) {
    const int vectors = (p.K + 8 * n - 1) / (8 * n);
    const int64_t place = lane < p.k ? p.places[t * p.k + lane] : -1;
    const float weight = lane < p.k ? p.weights[t * p.k + lane] : 0.f;
    for (int c = 0; c < vectors; ++c) {
      Raw8<TD> d;
      load8<WIDE>(static_cast<const TD*>(p.d_out) + t * p.ldd, l, c, n, p.K, d);
      for (int j = 0; j < p.k; ++j) {
        const int64_t at = __shfl_sync(0xffffffffu, place, j);
        if (at < 0 || at >= p.rows) continue;
        const float w = __shfl_sync(0xffffffffu, weight, j);
        Raw8<TY> y, o;
        float v[8], s = 0.f;
        if (p.dw) {
          load8<WIDE>(static_cast<const TY*>(p.y) + at * p.ldy, l, c, n, p.K, y);
#pragma unroll
          for (int i = 0; i < 8; ++i) s = fmaf(d.at(i), y.at(i), s);
#pragma unroll
          for (int m = 16; m > 0; m >>= 1) s += __shfl_xor_sync(0xffffffffu, s, m);
          if (lane == j) dot += s;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = w * d.at(i);
        o.set(v);
        store8<WIDE>(static_cast<TY*>(p.dy) + at * p.lddy, l, c, n, p.K, o);
      }
    }
  }
  if (!p.dw || !live) return;
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

template <typename TY, typename TO> cudaError_t launch(Combine p, bool wide, cudaStream_t stream) {
  p.n = threads_for((p.K + 7) / 8, 256);
  const int threads = p.n < 128 ? 128 : p.n;
  const dim3 grid(static_cast<unsigned>((p.T * p.n + threads - 1) / threads)), block(threads);
  return wide ? launch_pdl(combine_kernel<TY, TO, true>, grid, block, 0, stream, 1, p) : launch_pdl(combine_kernel<TY, TO, false>, grid, block, 0, stream, 1, p);
}

template <typename TD, typename TY> cudaError_t launch(CombineGrad p, bool wide, cudaStream_t stream) {
  p.n = threads_for((p.K + 7) / 8, 256);
  const int threads = p.n == 32 ? 128 : p.n;
  const dim3 grid(static_cast<unsigned>((p.T * p.n + threads - 1) / threads)), block(threads);
  return wide ? launch_pdl(combine_backward_kernel<TD, TY, true>, grid, block, 0, stream, 1, p)
              : launch_pdl(combine_backward_kernel<TD, TY, false>, grid, block, 0, stream, 1, p);
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
