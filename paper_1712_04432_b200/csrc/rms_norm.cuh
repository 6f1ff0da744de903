// What the norm and its gradients share: sums over a row, rows on their way through shared memory, the shapes they go in.
#pragma once
#include <math_constants.h>

#include <atomic>

#include "../../include/mbd.h"
#include "vec8.cuh"

namespace mbd {
namespace {

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

template <typename TR> __device__ __forceinline__ Raw8<TR> smaller8(const Raw8<TR>& h) {
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = h.at(i) * SMALLER;
  Raw8<TR> r;
  r.set(v);
  return r;
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
