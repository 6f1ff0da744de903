// Rows in 8 bits: s = max |x| / 127 in float, q = x / s rounded to the nearest integer (halves to even), one scale per row --
// a token of a batch, or an output channel of a weight matrix -- for the products of 8-bit integers.
//
// A call reads each value once: 3 bytes of traffic per bf16 value.  That leaves about 16 instructions per value at the full rate of
// HBM, too few for a division each, so the quotient is taken with the reciprocal, and where it lies next to half a step the sign of
// x - half * s decides.  Conversions to integers run at a quarter of the rate of sums, so rounding is a sum.
#include "../../include/mbd.h"
#include "epi.cuh"
#include "quotients.cuh"

namespace mbd {
namespace {

constexpr int PER = 4;                 // most vectors of 8 values a thread keeps

template <typename T> struct Vec8;
template <> struct Vec8<__nv_bfloat16> {
  uint4 q;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { q = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void part(const __nv_bfloat16* p, int n) {
    const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
    q.x = (n > 0 ? h[0] : 0u) | (n > 1 ? static_cast<uint32_t>(h[1]) << 16 : 0u);
    q.y = (n > 2 ? h[2] : 0u) | (n > 3 ? static_cast<uint32_t>(h[3]) << 16 : 0u);
    q.z = (n > 4 ? h[4] : 0u) | (n > 5 ? static_cast<uint32_t>(h[5]) << 16 : 0u);
    q.w = (n > 6 ? h[6] : 0u) | (n > 7 ? static_cast<uint32_t>(h[7]) << 16 : 0u);
  }
  __device__ __forceinline__ void pairs(f32x2* x) const {
    x[0] = pair(__uint_as_float(q.x << 16), __uint_as_float(q.x & 0xFFFF0000u));
    x[1] = pair(__uint_as_float(q.y << 16), __uint_as_float(q.y & 0xFFFF0000u));
    x[2] = pair(__uint_as_float(q.z << 16), __uint_as_float(q.z & 0xFFFF0000u));
    x[3] = pair(__uint_as_float(q.w << 16), __uint_as_float(q.w & 0xFFFF0000u));
  }
  // the largest |x| so far, by its bits (their order is that of the magnitudes, infinities and NaN last): two 16-bit maxima per word
  __device__ __forceinline__ uint32_t largest(uint32_t m) const {
    m = __vmaxu2(m, q.x & 0x7FFF7FFFu);
    m = __vmaxu2(m, q.y & 0x7FFF7FFFu);
    m = __vmaxu2(m, q.z & 0x7FFF7FFFu);
    return __vmaxu2(m, q.w & 0x7FFF7FFFu);
  }
  static __device__ __forceinline__ uint32_t bits(uint32_t m) { return max(m & 0xFFFF0000u, m << 16); }
};
template <> struct Vec8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = *reinterpret_cast<const float4*>(p); b = *reinterpret_cast<const float4*>(p + 4); }
  __device__ __forceinline__ void part(const float* p, int n) {
    a = make_float4(n > 0 ? p[0] : 0.f, n > 1 ? p[1] : 0.f, n > 2 ? p[2] : 0.f, n > 3 ? p[3] : 0.f);
    b = make_float4(n > 4 ? p[4] : 0.f, n > 5 ? p[5] : 0.f, n > 6 ? p[6] : 0.f, n > 7 ? p[7] : 0.f);
  }
  __device__ __forceinline__ void pairs(f32x2* x) const { x[0] = pair(a.x, a.y); x[1] = pair(a.z, a.w); x[2] = pair(b.x, b.y); x[3] = pair(b.z, b.w); }
  __device__ __forceinline__ uint32_t largest(uint32_t m) const {
    const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(v[j]) & 0x7FFFFFFFu);
    return m;
  }
  static __device__ __forceinline__ uint32_t bits(uint32_t m) { return m; }
};

template <typename T>
__device__ __forceinline__ Vec8<T> fetch(const T* row, int64_t i, int64_t K, bool wide) {
  Vec8<T> v;
  if (wide && i + 8 <= K) v.load(row + i);
  else v.part(row + i, static_cast<int>(min(K - i, static_cast<int64_t>(8))));
  return v;
}

template <typename T>
__device__ __forceinline__ void put(int8_t* row, int64_t i, int64_t K, bool wide, const Vec8<T>& v, float s, float inv, bool tiny) {
  f32x2 x[4];
  v.pairs(x);
  const uint2 w = quotients(x, s, inv, tiny);
  if (wide && i + 8 <= K) { *reinterpret_cast<uint2*>(row + i) = w; return; }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (i + j < K) row[i + j] = static_cast<int8_t>((j < 4 ? w.x : w.y) >> (8 * (j & 3)));
}

// One row per block.  FORM 2: whole aligned vectors, PER of them per thread in registers between the two passes (the usual case:
// nothing but the arithmetic is left per vector); 1: in registers, any alignment and length; 0: a row too long for that is
// read a second time.  (Persistent blocks with the next rows on their way through shared memory were slower, 60 against 52 us on 8192 x 8192:
// the instructions of a row count here, not its latency.)
template <typename T, int FORM>
__global__ void __launch_bounds__(1024)
quantize_rows_kernel(const T* __restrict__ X, int64_t ldx, int64_t K, int8_t* __restrict__ Q, int64_t ldq, float* __restrict__ scale,
                     int wide_in, int wide_out) {
  __shared__ uint32_t warp_max[32];
  const int tid = threadIdx.x, n = blockDim.x;
  pdl_trigger();
  pdl_wait();
  const T* row = X + blockIdx.x * ldx;
  int8_t* out = Q + blockIdx.x * ldq;
  const int vectors = static_cast<int>((K + 7) / 8);
  uint32_t m = 0;
  Vec8<T> v[FORM ? PER : 1];
  if (FORM == 2) {
    const T* at = row + 8 * tid;
#pragma unroll
    for (int j = 0; j < PER; ++j, at += 8 * n)
      if (tid + j * n < vectors) v[j].load(at);
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (tid + j * n < vectors) m = v[j].largest(m);
  } else if (FORM == 1) {
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (tid + j * n < vectors) v[j] = fetch(row, 8 * static_cast<int64_t>(tid + j * n), K, wide_in);
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (tid + j * n < vectors) m = v[j].largest(m);
  } else {
    for (int64_t i = 8 * static_cast<int64_t>(tid); i < K; i += 8 * n) m = fetch(row, i, K, wide_in).largest(m);
  }
  m = __reduce_max_sync(0xffffffffu, Vec8<T>::bits(m));
  if (n > 32) {
    if ((tid & 31) == 0) warp_max[tid >> 5] = m;
    __syncthreads();
    m = __reduce_max_sync(0xffffffffu, (tid & 31) < (n >> 5) ? warp_max[tid & 31] : 0u);
  }
  const Scale c = scale_of(m);
  if (tid == 0) scale[blockIdx.x] = c.s;
  if (FORM == 2) {
    int8_t* at = out + 8 * tid;
#pragma unroll
    for (int j = 0; j < PER; ++j, at += 8 * n)
      if (tid + j * n < vectors) {
        f32x2 x[4];
        v[j].pairs(x);
        *reinterpret_cast<uint2*>(at) = quotients(x, c.s, c.inv, c.tiny);
      }
  } else if (FORM == 1) {
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (tid + j * n < vectors) put(out, 8 * static_cast<int64_t>(tid + j * n), K, wide_out, v[j], c.s, c.inv, c.tiny);
  } else {
    for (int64_t i = 8 * static_cast<int64_t>(tid); i < K; i += 8 * n) put(out, i, K, wide_out, fetch(row, i, K, wide_in), c.s, c.inv, c.tiny);
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
  if (vectors > static_cast<int64_t>(threads) * PER)
    return launch_pdl(quantize_rows_kernel<T, 0>, grid, block, 0, stream, 1, x, ldx, K, Q, ldq, scale, wide_in, wide_out);
  if (wide_in && wide_out && K % 8 == 0)
    return launch_pdl(quantize_rows_kernel<T, 2>, grid, block, 0, stream, 1, x, ldx, K, Q, ldq, scale, wide_in, wide_out);
  return launch_pdl(quantize_rows_kernel<T, 1>, grid, block, 0, stream, 1, x, ldx, K, Q, ldq, scale, wide_in, wide_out);
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
