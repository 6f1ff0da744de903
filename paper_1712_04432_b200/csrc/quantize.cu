// Rows in 8 bits: s = max |x| / 127 in float, q = x / s rounded to the nearest integer (halves to even), one scale per row --
// a token of a batch, or an output channel of a weight matrix -- for the products of 8-bit integers.
//
// A row stays in registers between its maximum and its quotients, so a call reads each value once: 3 bytes of traffic per
// bf16 value.  That leaves about 16 instructions per value at the full rate of HBM, too few for a correctly rounded division each, so
// the quotient is first taken with the reciprocal (off by less than 2 units in the last place, 2^-15 at 127) and the division
// is done where that lies within 2^-14 of half a step.
#include "../../include/mbd.h"
#include "epi.cuh"

namespace mbd {
namespace {

constexpr int PER = 4;                 // vectors of 8 values a thread keeps

template <typename T> struct Vec8;
template <> struct Vec8<__nv_bfloat16> {
  uint4 q;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { q = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void set(int i, __nv_bfloat16 x) { reinterpret_cast<__nv_bfloat16*>(&q)[i] = x; }
  __device__ __forceinline__ float get(int i) const {
    const uint32_t w = (&q.x)[i >> 1];
    return __uint_as_float(i & 1 ? w & 0xFFFF0000u : w << 16);
  }
};
template <> struct Vec8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = *reinterpret_cast<const float4*>(p); b = *reinterpret_cast<const float4*>(p + 4); }
  __device__ __forceinline__ void set(int i, float x) { (i < 4 ? &a.x : &b.x)[i & 3] = x; }
  __device__ __forceinline__ float get(int i) const { return (i < 4 ? &a.x : &b.x)[i & 3]; }
};

template <typename T>
__device__ __forceinline__ Vec8<T> fetch(const T* row, int64_t i, int64_t K, bool wide) {
  Vec8<T> v;
  if (wide && i + 8 <= K) { v.load(row + i); return v; }
#pragma unroll
  for (int j = 0; j < 8; ++j) v.set(j, i + j < K ? row[i + j] : T(0.f));
  return v;
}

template <typename T>
__device__ __forceinline__ uint32_t max_bits(const Vec8<T>& v, uint32_t m) {         // |x| in rising order of its bits
#pragma unroll
  for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(v.get(j)) & 0x7FFFFFFFu);
  return m;
}

// The quotient, correctly rounded: a float quotient that is exactly half a step may have been rounded to it, the remainder tells.
__device__ __noinline__ float divide_to_integer(float x, float s) {
  const float t = __fdiv_rn(x, s);
  float k = rintf(t);
  if (fabsf(t - k) == 0.5f) {
    const float rest = fmaf(-t, s, x);
    if (rest > 0.f) k = ceilf(t);
    if (rest < 0.f) k = floorf(t);
  }
  return fminf(fmaxf(k, -127.f), 127.f);
}

template <typename T>
__device__ __forceinline__ void put(int8_t* row, int64_t i, int64_t K, bool wide, const Vec8<T>& v, float s, float inv, bool tiny) {
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float x = v.get(j);
    float k;
    if (tiny) {
      k = s > 0.f ? divide_to_integer(x, s) : 0.f;
    } else {
      const float t = x * inv;
      k = rintf(t);
      if (fabsf(t - k) > 0.5f - 6.103515625e-5f) k = divide_to_integer(x, s);
    }
    w[j >> 2] |= (static_cast<uint32_t>(static_cast<int>(k)) & 0xFFu) << (8 * (j & 3));
  }
  if (wide && i + 8 <= K) { *reinterpret_cast<uint2*>(row + i) = make_uint2(w[0], w[1]); return; }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (i + j < K) row[i + j] = static_cast<int8_t>(w[j >> 2] >> (8 * (j & 3)));
}

// One row per block.  KEEP: the row fits the block's registers; otherwise it is read a second time.
template <typename T, bool KEEP>
__global__ void __launch_bounds__(1024)
quantize_rows_kernel(const T* __restrict__ X, int64_t ldx, int64_t K, int8_t* __restrict__ Q, int64_t ldq, float* __restrict__ scale,
                     int wide_in, int wide_out) {
  __shared__ uint32_t warp_max[32];
  const int tid = threadIdx.x, n = blockDim.x;
  pdl_trigger();
  pdl_wait();
  const T* row = X + blockIdx.x * ldx;
  int8_t* out = Q + blockIdx.x * ldq;
  uint32_t m = 0;
  Vec8<T> v[KEEP ? PER : 1];
  if (KEEP) {
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int64_t i = 8 * static_cast<int64_t>(tid + j * n);
      if (i < K) v[j] = fetch(row, i, K, wide_in);
    }
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (8 * static_cast<int64_t>(tid + j * n) < K) m = max_bits(v[j], m);
  } else {
    for (int64_t i = 8 * static_cast<int64_t>(tid); i < K; i += 8 * n) m = max_bits(fetch(row, i, K, wide_in), m);
  }
  m = __reduce_max_sync(0xffffffffu, m);
  if (n > 32) {
    if ((tid & 31) == 0) warp_max[tid >> 5] = m;
    __syncthreads();
    m = __reduce_max_sync(0xffffffffu, (tid & 31) < (n >> 5) ? warp_max[tid & 31] : 0u);
  }
  const bool finite = m < 0x7F800000u;                         // a row with an infinity or a NaN has no scale: it is NaN, and q is 0
  const float s = finite ? __fdiv_rn(__uint_as_float(m), 127.f) : __uint_as_float(0x7FC00000u);
  const bool tiny = !(s >= 1e-30f);                            // (zero, NaN, or so small that its reciprocal is not accurate)
  const float inv = tiny ? 0.f : __fdiv_rn(1.f, s);
  if (tid == 0) scale[blockIdx.x] = s;
  if (KEEP) {
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int64_t i = 8 * static_cast<int64_t>(tid + j * n);
      if (i < K) put(out, i, K, wide_out, v[j], s, inv, tiny);
    }
  } else {
    for (int64_t i = 8 * static_cast<int64_t>(tid); i < K; i += 8 * n) put(out, i, K, wide_out, fetch(row, i, K, wide_in), s, inv, tiny);
  }
}

template <typename T>
cudaError_t launch(const void* X, int64_t R, int64_t K, int64_t ldx, int8_t* Q, int64_t ldq, float* scale, int sms, cudaStream_t stream) {
  const int wide_in = (reinterpret_cast<uintptr_t>(X) & 15u) == 0 && ldx % (16 / static_cast<int>(sizeof(T))) == 0;
  const int wide_out = (reinterpret_cast<uintptr_t>(Q) & 7u) == 0 && ldq % 8 == 0;
  const int64_t vectors = (K + 7) / 8;
  // few rows: as many threads as a row has vectors, for its latency; many rows: each thread its full share of registers
  const int64_t want = R < 2 * sms ? vectors : (vectors + PER - 1) / PER;
  int threads = 32;
  while (threads < want && threads < 1024) threads *= 2;
  const dim3 grid(static_cast<unsigned>(R)), block(threads);
  const T* x = static_cast<const T*>(X);
  if (vectors <= static_cast<int64_t>(threads) * PER) return launch_pdl(quantize_rows_kernel<T, true>, grid, block, 0, stream, 1, x, ldx, K, Q, ldq, scale, wide_in, wide_out);
  return launch_pdl(quantize_rows_kernel<T, false>, grid, block, 0, stream, 1, x, ldx, K, Q, ldq, scale, wide_in, wide_out);
}

}  // namespace
}  // namespace mbd

using namespace mbd;

extern "C" mbd_status mbd_quantize_rows(const void* X_dev, int x_bf16, int64_t R, int64_t K, int64_t ldx, int8_t* Q_dev, int64_t ldq,
                                        float* scale_dev, int sync, void* cuda_stream) {
  if (R < 0 || K < 1 || ldx < K || ldq < K) return MBD_E_INVALID;
  if (R == 0) return MBD_OK;
  if (!X_dev || !Q_dev || !scale_dev) return MBD_E_INVALID;
  if (R > INT32_MAX) return MBD_E_UNSUPPORTED;
  if ((reinterpret_cast<uintptr_t>(X_dev) & (x_bf16 ? 1u : 3u)) || (reinterpret_cast<uintptr_t>(scale_dev) & 3u)) return MBD_E_UNSUPPORTED;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
      (x_bf16 ? launch<__nv_bfloat16>(X_dev, R, K, ldx, Q_dev, ldq, scale_dev, sms, stream)
              : launch<float>(X_dev, R, K, ldx, Q_dev, ldq, scale_dev, sms, stream)) != cudaSuccess ||
      (sync && cudaStreamSynchronize(stream) != cudaSuccess)) {
    (void)cudaGetLastError();
    return MBD_E_CUDA;
  }
  return MBD_OK;
}
