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
// Bound by HBM: 30 bytes per element with float moments, bf16 weights, float masters and gradients, 18 with 8 bits.  A
// warp owns 256 consecutive elements (so a block's maximum is two warp reductions) and issues all of their loads before
// its first use of one; every block of threads takes one contiguous range of the list, so that a tensor's pointers are read
// once per range and not once per 256 elements.
#include <math.h>

#include <algorithm>
#include <new>
#include <vector>

#include <cuda_fp8.h>

#include "../../include/mbd.h"
#include "epi.cuh"

namespace mbd {
namespace {

constexpr int BLOCK = 256;             // elements per warp and pass; also the elements that share a scale
constexpr int THREADS = 256;

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
enum { P_BF16 = 1, G_BF16 = 2, WIDE = 4 };

struct Clock {                         // device: steps taken, and the powers of the two rates
  double b1_t, b2_t;
  long long t;
  unsigned int seen;
};

__device__ __forceinline__ void load4(const float* p, int n, bool wide, float* x) {
  if (wide) {
    const float4 q = *reinterpret_cast<const float4*>(p);
    x[0] = q.x; x[1] = q.y; x[2] = q.z; x[3] = q.w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = i < n ? p[i] : 0.f;
  }
}
__device__ __forceinline__ void load4(const __nv_bfloat16* p, int n, bool wide, float* x) {
  if (wide) {
    const uint2 q = *reinterpret_cast<const uint2*>(p);
    x[0] = bf16_bits_to_f32(q.x & 0xFFFFu); x[1] = bf16_bits_to_f32(q.x >> 16);
    x[2] = bf16_bits_to_f32(q.y & 0xFFFFu); x[3] = bf16_bits_to_f32(q.y >> 16);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = i < n ? __bfloat162float(p[i]) : 0.f;
  }
}
__device__ __forceinline__ void store4(float* p, int n, bool wide, const float* x) {
  if (wide) {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) if (i < n) p[i] = x[i];
  }
}
__device__ __forceinline__ void store4(__nv_bfloat16* p, int n, bool wide, const float* x) {
  if (wide) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) if (i < n) p[i] = __float2bfloat16_rn(x[i]);
  }
}

__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int n, bool wide) {
  if (wide) return *reinterpret_cast<const uint32_t*>(p);
  uint32_t c = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) if (i < n) c |= static_cast<uint32_t>(p[i]) << (8 * i);
  return c;
}
__device__ __forceinline__ void store_codes(uint8_t* p, int n, bool wide, uint32_t c) {
  if (wide) { *reinterpret_cast<uint32_t*>(p) = c; return; }
#pragma unroll
  for (int i = 0; i < 4; ++i) if (i < n) p[i] = static_cast<uint8_t>(c >> (8 * i));
}
__device__ __forceinline__ void from_codes(uint32_t c, float* x) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const __half2_raw r = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(c >> (16 * h)), __NV_E4M3);
    const float2 f = __half22float2(__half2(r));
    x[2 * h] = f.x; x[2 * h + 1] = f.y;
  }
}
__device__ __forceinline__ uint32_t to_codes(const float* x) {         // nearest, halves to even, NaN stays NaN
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(x[0], x[1]), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(x[2], x[3]), __NV_SATFINITE, __NV_E4M3);
  return lo | (hi << 16);
}

// The largest finite |x| of a warp's 8 x 32 values.
__device__ __forceinline__ float block_max(const float* x) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t b = __float_as_uint(x[i]) & 0x7FFFFFFFu;
    m = max(m, b < 0x7F800000u ? b : 0u);
  }
  return __uint_as_float(__reduce_max_sync(0xffffffffu, m));
}

constexpr float E4M3_MAX = 448.f, E4M3_MIN = 0.001953125f;

// Each value over the block's scale; what is not finite becomes NaN and stays that element's own.
template <bool POSITIVE>
__device__ __forceinline__ void scaled(const float* x, float scale, float* q) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float y = scale > 0.f ? __fdiv_rn(x[i], scale) : 0.f;
    if (POSITIVE && x[i] > 0.f) y = fmaxf(y, E4M3_MIN);
    if (!(fabsf(x[i]) < INFINITY)) y = NAN;
    q[i] = y;
  }
}

template <int BITS>
__global__ void __launch_bounds__(THREADS)
adamw_kernel(const Tensor* __restrict__ tensors, const int* __restrict__ first, int count, int total, Clock* clock, double b1, double b2,
             float eps, double lr, float grad_scale) {
  __shared__ float rates[2];           // 1 / sqrt(1 - b2^t), lr / (1 - b1^t)
  if (threadIdx.x == 0) {
    const double p1 = clock->b1_t * b1, p2 = clock->b2_t * b2;
    const long long t = clock->t;
    rates[0] = static_cast<float>(1.0 / sqrt(1.0 - p2));
    rates[1] = static_cast<float>(lr / (1.0 - p1));
    // the block that comes last has read the clock after every other one, and moves it on
    __threadfence();
    if (atomicAdd(&clock->seen, 1u) == gridDim.x - 1) {
      clock->b1_t = p1; clock->b2_t = p2; clock->t = t + 1;
      clock->seen = 0;
    }
  }
  __syncthreads();
  const float root_rate = rates[0], step = rates[1];
  const float fb1 = static_cast<float>(b1), fb2 = static_cast<float>(b2);
  const float c1 = static_cast<float>(1.0 - b1), c2 = static_cast<float>(1.0 - b2);
  const int lane = threadIdx.x & 31;
  const int lo = static_cast<int>(static_cast<long long>(blockIdx.x) * total / gridDim.x);
  const int hi = static_cast<int>(static_cast<long long>(blockIdx.x + 1) * total / gridDim.x);
  int b = lo + (threadIdx.x >> 5);
  if (b >= hi) return;
  int t = 0;                           // the tensor of block b: the last one that starts at or before it
  for (int step2 = 1 << 30; step2; step2 >>= 1)
    if (t + step2 < count && first[t + step2] <= b) t += step2;
  Tensor w = tensors[t];
  int start = first[t], end = first[t + 1];
  for (; b < hi; b += THREADS / 32) {
    if (b >= end) {
      do { ++t; end = first[t + 1]; } while (b >= end);
      w = tensors[t];
      start = first[t];
    }
    const int64_t at0 = static_cast<int64_t>(b - start) * BLOCK + 4 * lane, at1 = at0 + 128;
    const int n0 = static_cast<int>(min(max(w.n - at0, int64_t(0)), int64_t(4))), n1 = static_cast<int>(min(max(w.n - at1, int64_t(0)), int64_t(4)));
    const bool wide0 = (w.flags & WIDE) && n0 == 4, wide1 = (w.flags & WIDE) && n1 == 4;
    float g[8], x[8], m[8], v[8];
    uint32_t cm[2], cv[2];
    float ms = 0.f, vs = 0.f;
    if (w.flags & G_BF16) {
      load4(static_cast<const __nv_bfloat16*>(w.g) + at0, n0, wide0, g);
      load4(static_cast<const __nv_bfloat16*>(w.g) + at1, n1, wide1, g + 4);
    } else {
      load4(static_cast<const float*>(w.g) + at0, n0, wide0, g);
      load4(static_cast<const float*>(w.g) + at1, n1, wide1, g + 4);
    }
    if (w.master || !(w.flags & P_BF16)) {
      const float* src = w.master ? w.master : static_cast<const float*>(w.p);
      load4(src + at0, n0, wide0, x);
      load4(src + at1, n1, wide1, x + 4);
    } else {
      load4(static_cast<const __nv_bfloat16*>(w.p) + at0, n0, wide0, x);
      load4(static_cast<const __nv_bfloat16*>(w.p) + at1, n1, wide1, x + 4);
    }
    if (BITS == 32) {
      load4(static_cast<const float*>(w.m) + at0, n0, wide0, m);
      load4(static_cast<const float*>(w.m) + at1, n1, wide1, m + 4);
      load4(static_cast<const float*>(w.v) + at0, n0, wide0, v);
      load4(static_cast<const float*>(w.v) + at1, n1, wide1, v + 4);
    } else {
      cm[0] = load_codes(static_cast<const uint8_t*>(w.m) + at0, n0, wide0);
      cm[1] = load_codes(static_cast<const uint8_t*>(w.m) + at1, n1, wide1);
      cv[0] = load_codes(static_cast<const uint8_t*>(w.v) + at0, n0, wide0);
      cv[1] = load_codes(static_cast<const uint8_t*>(w.v) + at1, n1, wide1);
      ms = w.ms[b - start];
      vs = w.vs[b - start];
      from_codes(cm[0], m); from_codes(cm[1], m + 4);
      from_codes(cv[0], v); from_codes(cv[1], v + 4);
    }
    const float keep = __fsub_rn(1.f, __fmul_rn(static_cast<float>(lr), w.decay));
    float root[8];
    // every product and sum is rounded by itself (no fused multiply-add), so that the result is the formula's in plain float
    // arithmetic, bit for bit
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float gi = __fmul_rn(g[i], grad_scale);
      if (BITS == 8) {
        m[i] = __fmul_rn(m[i], ms);
        v[i] = __fmul_rn(v[i], vs);
        v[i] = __fmul_rn(v[i], v[i]);
      }
      m[i] = __fadd_rn(__fmul_rn(m[i], fb1), __fmul_rn(gi, c1));
      v[i] = __fadd_rn(__fmul_rn(v[i], fb2), __fmul_rn(__fmul_rn(gi, gi), c2));
      root[i] = __fsqrt_rn(v[i]);
      const float d = __fadd_rn(__fmul_rn(root[i], root_rate), eps);
      x[i] = __fsub_rn(__fmul_rn(x[i], keep), __fmul_rn(__fdiv_rn(m[i], d), step));
    }
    if (w.flags & P_BF16) {
      if (w.master) {
        store4(w.master + at0, n0, wide0, x);
        store4(w.master + at1, n1, wide1, x + 4);
      }
      store4(static_cast<__nv_bfloat16*>(w.p) + at0, n0, wide0, x);
      store4(static_cast<__nv_bfloat16*>(w.p) + at1, n1, wide1, x + 4);
    } else {
      store4(static_cast<float*>(w.p) + at0, n0, wide0, x);
      store4(static_cast<float*>(w.p) + at1, n1, wide1, x + 4);
    }
    if (BITS == 32) {
      store4(static_cast<float*>(w.m) + at0, n0, wide0, m);
      store4(static_cast<float*>(w.m) + at1, n1, wide1, m + 4);
      store4(static_cast<float*>(w.v) + at0, n0, wide0, v);
      store4(static_cast<float*>(w.v) + at1, n1, wide1, v + 4);
    } else {
      ms = __fdiv_rn(block_max(m), E4M3_MAX);
      vs = __fdiv_rn(block_max(root), E4M3_MAX);
      float q[8];
      scaled<false>(m, ms, q);
      store_codes(static_cast<uint8_t*>(w.m) + at0, n0, wide0, to_codes(q));
      store_codes(static_cast<uint8_t*>(w.m) + at1, n1, wide1, to_codes(q + 4));
      scaled<true>(root, vs, q);
      store_codes(static_cast<uint8_t*>(w.v) + at0, n0, wide0, to_codes(q));
      store_codes(static_cast<uint8_t*>(w.v) + at1, n1, wide1, to_codes(q + 4));
      if (lane == 0) { w.ms[b - start] = ms; w.vs[b - start] = vs; }
    }
  }
}

}  // namespace
}  // namespace mbd

using namespace mbd;

struct mbd_adamw {
  int dev = 0, sms = 0, count = 0, total = 0, bits = 32;
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
      !(eps > 0.0 && eps < 1.0)) return MBD_E_INVALID;
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
      if (t.n > (int64_t(1) << 46) || (total += blocks) > INT32_MAX - 1024) return MBD_E_UNSUPPORTED;
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
      const bool wide = at(t.param_dev) % (4 * psize) == 0 && at(t.master_dev) % 16 == 0 && at(t.grad_dev) % (4 * gsize) == 0 &&
                        at(t.m_dev) % (4 * ssize) == 0 && at(t.v_dev) % (4 * ssize) == 0;
      d.flags = (t.param_bf16 ? P_BF16 : 0) | (t.grad_bf16 ? G_BF16 : 0) | (wide ? WIDE : 0);
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
    h->count = count; h->total = static_cast<int>(total); h->bits = state_bits;
    h->b1 = beta1; h->b2 = beta2; h->eps = static_cast<float>(eps);
    const size_t bytes = 64 + sizeof(Tensor) * count + sizeof(int) * (count + 1);
    mbd_status st = MBD_OK;
    if (cudaGetDevice(&h->dev) != cudaSuccess || cudaDeviceGetAttribute(&h->sms, cudaDevAttrMultiProcessorCount, h->dev) != cudaSuccess) st = MBD_E_CUDA;
    else if (cudaMalloc(reinterpret_cast<void**>(&h->block), bytes) != cudaSuccess) { h->block = nullptr; st = MBD_E_ALLOC; }
    if (st == MBD_OK) {
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
  } catch (const std::bad_alloc&) {
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
  if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpy(opt->clock, &c, sizeof(c), cudaMemcpyHostToDevice) != cudaSuccess) { (void)cudaGetLastError(); return MBD_E_CUDA; }
  return MBD_OK;
}

extern "C" mbd_status mbd_adamw_get_steps(mbd_adamw* opt, int64_t* steps_done_host) {
  if (!opt || !steps_done_host) return MBD_E_INVALID;
  Clock c{};
  if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpy(&c, opt->clock, sizeof(c), cudaMemcpyDeviceToHost) != cudaSuccess) { (void)cudaGetLastError(); return MBD_E_CUDA; }
  *steps_done_host = c.t;
  return MBD_OK;
}

extern "C" mbd_status mbd_adamw_step(mbd_adamw* opt, double lr, double grad_scale, void* cuda_stream) {
  if (!opt || !(lr >= 0.0 && lr < 1e30) || !(fabs(grad_scale) < 1e30)) return MBD_E_INVALID;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { (void)cudaGetLastError(); return MBD_E_CUDA; }
  if (dev != opt->dev) return MBD_E_STATE;                     // the list's device has to be the current one
  const int64_t ctas = (static_cast<int64_t>(opt->total) + THREADS / 32 - 1) / (THREADS / 32);
  const int64_t most = static_cast<int64_t>(opt->sms) * 4;
  const dim3 grid(static_cast<unsigned>(ctas < most ? ctas : most)), block(THREADS);
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = opt->bits == 32
      ? launch_pdl(adamw_kernel<32>, grid, block, 0, stream, 0, static_cast<const Tensor*>(opt->tensors), static_cast<const int*>(opt->first), opt->count, opt->total, opt->clock, opt->b1, opt->b2, opt->eps, lr, static_cast<float>(grad_scale))
      : launch_pdl(adamw_kernel<8>, grid, block, 0, stream, 0, static_cast<const Tensor*>(opt->tensors), static_cast<const int*>(opt->first), opt->count, opt->total, opt->clock, opt->b1, opt->b2, opt->eps, lr, static_cast<float>(grad_scale));
  if (e != cudaSuccess) { (void)cudaGetLastError(); return MBD_E_CUDA; }
  return MBD_OK;
}
