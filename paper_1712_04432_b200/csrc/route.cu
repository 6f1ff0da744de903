// Routing of tokens to experts: from a token's scores of E experts the k best ones, their weights, and the places of the (token, slot)
// rows in the order of the experts that the products grouped by expert want; and the gradient of the logits.
//
//   p = softmax(l) or sigmoid(l);  key = p + bias, or the logit itself without a bias (the same order, and exact)
//   an expert whose logit or key is -inf is never chosen;  NaN keys come after all numbers
//   groups: a group's score is its best key, or the sum of its two best (without a bias: of its two best p);  only the best groups stay
//   the k largest keys, equal ones by rising index;  w = c p, or c p / (sum of the chosen p)
//
// One warp per token, its keys in registers as integers in the order of the floats: a maximum is one warp-wide instruction.  Keys
// made of float scores can lie nearer to each other than they are exact; where a choice hangs on such a gap the warp takes the
// token again in double (about one token in a thousand with a bias).
//
// Places: a block marks for each expert which of 64 tokens chose it, one bit a token, so a slot's rank is a count of bits and neither
// it nor anything else depends on the order of atomics.  A second kernel adds up the blocks' counts (up to 64 tokens are one block, and one launch).
#include <math_constants.h>

#include "../../include/mbd.h"
#include "vec8.cuh"

namespace mbd {
namespace {

typedef __nv_bfloat16 bf16;
constexpr int MAX_E = 512, MAX_K = 32, MAX_G = 32;
constexpr int SUB = 64;                        // tokens whose choices are held as bits at a time
constexpr int MOST_BLOCKS = 256, MOST_TOKENS = 65472;   // of the first kernel; of one of its blocks (counts are 16 bits wide)

struct Route {
  const void* logits;
  const float* bias;
  const int32_t* count;
  int32_t *ids, *places, *offsets;
  float* weights;
  uint16_t* counts;             // [blocks][E2]: slots of a block's tokens per expert; null: one block does it all
  int64_t ld;
  int T, E, E2, k, chunk;       // E2: E rounded up to an even number
  int sigmoid, renorm, G, top_groups, best;
  uint32_t by_group;            // e / (E / G) = e * by_group >> 20
  float scale;
};

// ---- numbers as integers of the same order; 0: not there, 1: NaN
template <typename F> struct Code;
template <> struct Code<float> {
  typedef uint32_t type;
  static __device__ __forceinline__ uint32_t of(float f) {
    const uint32_t u = __float_as_uint(f + 0.f);               // (-0 is 0)
    return f != f ? 1u : u & 0x80000000u ? ~u : u | 0x80000000u;
  }
  static __device__ __forceinline__ float value(uint32_t c) { return c <= 1u ? CUDART_NAN_F : __uint_as_float(c & 0x80000000u ? c & 0x7FFFFFFFu : ~c); }
  static __device__ __forceinline__ uint32_t largest(uint32_t c) { return __reduce_max_sync(0xffffffffu, c); }
  static __device__ __forceinline__ float exponential(float x) { return expf(x); }
};
template <> struct Code<double> {
  typedef unsigned long long type;
  static __device__ __forceinline__ type of(double f) {
    const type u = static_cast<type>(__double_as_longlong(f + 0.0));
    return f != f ? 1ull : u >> 63 ? ~u : u | 0x8000000000000000ull;
  }
  static __device__ __forceinline__ double value(type c) {
    return c <= 1ull ? CUDART_NAN : __longlong_as_double(static_cast<long long>(c >> 63 ? c & 0x7FFFFFFFFFFFFFFFull : ~c));
  }
  static __device__ __forceinline__ type largest(type c) {
    const uint32_t hi = static_cast<uint32_t>(c >> 32), top = __reduce_max_sync(0xffffffffu, hi);
    const uint32_t low = __reduce_max_sync(0xffffffffu, hi == top ? static_cast<uint32_t>(c) : 0u);
    return static_cast<type>(top) << 32 | low;
  }
  static __device__ __forceinline__ double exponential(double x) { return exp(x); }
};

template <typename F> __device__ __forceinline__ F warp_sum(F x) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
  return x;
}
__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
  return x;
}

__device__ __forceinline__ float logit(const bf16* row, int e) { return __bfloat162float(row[e]); }
__device__ __forceinline__ float logit(const float* row, int e) { return row[e]; }

// 1 / (1 + exp(-z)), without an exponential that overflows.
template <typename F> __device__ __forceinline__ F sigmoid(F z) {
  const F t = Code<F>::exponential(z < F(0) ? z : -z);
  return (z < F(0) ? t : F(1)) / (F(1) + t);
}

// A token's choice: lane j < chosen has the j-th expert.  l: the logits of experts i * 32 + lane (-inf behind the last).
// top, total: the largest logit and the sum of exp(l - top), where a softmax needs them.
template <typename F> struct Choice { int id, chosen; float top; F total; bool unsure; };

template <typename F, int NPL, typename T>
__device__ __forceinline__ Choice<F> choose(const Route& p, const T* row, const float (&l)[NPL], int lane) {
  typedef typename Code<F>::type code;
  constexpr bool FLOAT = sizeof(F) == 4;
  const bool scored = p.bias || (p.G > 1 && p.best == 2);      // whether the choice needs more than the order of the logits
  Choice<F> c;
  c.unsure = false;
  c.top = -CUDART_INF_F;
  c.total = F(1);
  if (!p.sigmoid && (scored || !p.renorm)) {
#pragma unroll
    for (int i = 0; i < NPL; ++i) c.top = fmaxf(c.top, l[i]);
    c.top = warp_max(c.top);
    F sum = F(0);
#pragma unroll
    for (int i = 0; i < NPL; ++i)
      if (l[i] != -CUDART_INF_F) sum += Code<F>::exponential(F(l[i]) - F(c.top));
    c.total = warp_sum(sum);
  }
  auto score = [&](float z) { return p.sigmoid ? sigmoid(F(z)) : Code<F>::exponential(F(z) - F(c.top)) / c.total; };
  code key[NPL];
#pragma unroll
  for (int i = 0; i < NPL; ++i) {
    const int e = i * 32 + lane;
    key[i] = 0;
    if (l[i] != -CUDART_INF_F) {                               // (so e < E)
      const F v = p.bias ? score(l[i]) + F(p.bias[e]) : F(l[i]);
      if (v != F(-CUDART_INF)) key[i] = Code<F>::of(v);
    }
  }
  // how far float scores, and with them gaps between keys, can be off: the exponentials, the sum of up to 512 of them, the
  // quotient (3e-6 of the largest p; 1e-6 for a sigmoid), and the sum with the bias
  const float slack = p.sigmoid ? 1e-6f : 3e-6f / static_cast<float>(c.total);
  if (p.G > 1) {
    const bool by_score = p.best == 2 && !p.bias;
    code mine = 0;                                             // lane g: the score of group g
    for (int g = 0; g < p.G; ++g) {
      code a = 0, b = 0;                                       // this lane's two best of the group
#pragma unroll
      for (int i = 0; i < NPL; ++i) {
        const int e = i * 32 + lane;
        if (key[i] == 0 || static_cast<int>(e * p.by_group >> 20) != g) continue;
        const code v = by_score ? Code<F>::of(score(l[i])) : key[i];
        if (v > a) { b = a; a = v; }
        else if (v > b) b = v;
      }
      const code first = Code<F>::largest(a);
      code of = first;
      if (p.best == 2 && first) {
        const unsigned owners = __ballot_sync(0xffffffffu, a == first);
        const code second = Code<F>::largest(lane == __ffs(owners) - 1 ? b : a);
        of = Code<F>::of(Code<F>::value(first) + (second ? Code<F>::value(second) : F(0)));
      }
      if (lane == g) mine = of;
    }
    int rank = 0;
    for (int g = 0; g < p.G; ++g) {
      const code other = __shfl_sync(0xffffffffu, mine, g);
      rank += other > mine || (other == mine && g < lane);
    }
    const bool keep = lane < p.G && mine && rank < p.top_groups;
    const unsigned kept = __ballot_sync(0xffffffffu, keep);
    if (FLOAT && scored) {
      const code out = Code<F>::largest(keep ? 0 : mine);      // (lanes behind the last group hold 0)
      const code in = ~Code<F>::largest(keep ? ~mine : 0);
      if (out && kept) {
        const F a = Code<F>::value(in), b = Code<F>::value(out);
        c.unsure = !(a - b > 2.f * slack + 6e-7f * fabsf(static_cast<float>(a)));
      }
    }
#pragma unroll
    for (int i = 0; i < NPL; ++i)
      if (!(kept >> ((i * 32 + lane) * p.by_group >> 20 & 31u) & 1u)) key[i] = 0;       // (experts behind the last are not there anyway)
  }
  c.id = -1;
  c.chosen = 0;
  code mine = 0;
  for (int j = 0; j < p.k; ++j) {
    code best = 0;
#pragma unroll
    for (int i = 0; i < NPL; ++i) best = key[i] > best ? key[i] : best;
    const code top = Code<F>::largest(best);
    if (!top) break;
    int e = MAX_E;
#pragma unroll
    for (int i = NPL - 1; i >= 0; --i)
      if (key[i] == top) e = i * 32 + lane;
    e = __reduce_min_sync(0xffffffffu, e);
#pragma unroll
    for (int i = 0; i < NPL; ++i)
      if (e == i * 32 + lane) key[i] = 0;
    if (lane == j) { c.id = e; mine = top; }
    c.chosen = j + 1;
  }
  if (FLOAT && p.bias && !c.unsure) {
    // neighbours in the order, and the last one against all that are left; equal logits with equal biases are really equal
    const float z = c.id >= 0 ? logit(row, c.id) : 0.f, b = c.id >= 0 ? p.bias[c.id] : 0.f, v = static_cast<float>(Code<F>::value(mine));
    const float z2 = __shfl_down_sync(0xffffffffu, z, 1), b2 = __shfl_down_sync(0xffffffffu, b, 1), v2 = __shfl_down_sync(0xffffffffu, v, 1);
    bool near = lane + 1 < c.chosen && !(v - v2 > slack + 3e-7f * fabsf(v)) && !(z == z2 && b == b2);
    if (c.chosen == p.k) {
      const float zk = __shfl_sync(0xffffffffu, z, p.k - 1), bk = __shfl_sync(0xffffffffu, b, p.k - 1), vk = __shfl_sync(0xffffffffu, v, p.k - 1);
#pragma unroll
      for (int i = 0; i < NPL; ++i)
        if (key[i]) near |= !(vk - static_cast<float>(Code<F>::value(key[i])) > slack + 3e-7f * fabsf(vk)) && !(l[i] == zk && p.bias[i * 32 + lane] == bk);
    }
    c.unsure = __any_sync(0xffffffffu, near);
  }
  return c;
}

template <int NPL, typename T>
__device__ __forceinline__ void logits_of(const Route& p, const T* row, int lane, float (&l)[NPL]) {
#pragma unroll
  for (int i = 0; i < NPL; ++i) l[i] = i * 32 + lane < p.E ? logit(row, i * 32 + lane) : -CUDART_INF_F;
}

// The choice between values that lie too near to each other for floats.
template <int NPL, typename T>
__device__ __noinline__ int2 choose_in_double(const Route& p, const T* row, int lane) {
  float l[NPL];
  logits_of<NPL>(p, row, lane, l);
  const Choice<double> c = choose<double, NPL>(p, row, l, lane);
  return make_int2(c.id, c.chosen);
}

// The weight of lane j's expert, of logit z; total: over all experts.  Renormalised scores are taken relative to the largest
// chosen one, so that scores below float's range keep their ratios: sigmoid(z) is exp(z) far below zero.
__device__ __forceinline__ float share(float z, bool there, bool by_sigmoid, bool renorm, float top, float total) {
  if (!renorm) return there ? (by_sigmoid ? sigmoid(z) : __fdiv_rn(expf(z - top), total)) : 0.f;
  const float most = warp_max(there ? z : -CUDART_INF_F);
  const float r = !there || z == -CUDART_INF_F ? 0.f : by_sigmoid && !(most < -60.f) ? sigmoid(z) : expf(z - most);
  const float sum = warp_sum(r);
  return there && sum != 0.f ? __fdiv_rn(r, sum) : 0.f;
}

// Exclusive sums of E numbers in shared memory, by one warp; all of them go behind the last.
__device__ __forceinline__ void offsets_of(int* n, int E, int lane) {
  const int per = (E + 31) / 32, first = lane * per;
  int sum = 0;
  for (int i = 0; i < per; ++i)
    if (first + i < E) sum += n[first + i];
  int before = sum;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, before, d);
    if (lane >= d) before += v;
  }
  if (lane == 31) n[E] = before;
  before -= sum;
  for (int i = 0; i < per; ++i)
    if (first + i < E) {
      const int v = n[first + i];
      n[first + i] = before;
      before += v;
    }
}

template <typename T, int NPL>
__global__ void __launch_bounds__(1024) route_kernel(const __grid_constant__ Route p) {
  __shared__ uint32_t chose[MAX_E][SUB / 32];
  __shared__ int running[MAX_E + 1];
  __shared__ int16_t ids[SUB * MAX_K];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  pdl_trigger();
  pdl_wait();
  const int live = p.count ? min(max(*p.count, 0), p.T) : p.T;
  for (int e = threadIdx.x; e <= p.E; e += blockDim.x) running[e] = 0;
  const int64_t begin = blockIdx.x * static_cast<int64_t>(p.chunk), end = min(begin + p.chunk, static_cast<int64_t>(p.T));
  for (int64_t sub = begin; sub < end; sub += SUB) {
    for (int e = threadIdx.x; e < p.E * (SUB / 32); e += blockDim.x) chose[0][e] = 0u;
    __syncthreads();
    const int tokens = static_cast<int>(min(end - sub, static_cast<int64_t>(SUB)));
    for (int i = warp; i < tokens; i += warps) {
      const int64_t t = sub + i;
      int id = -1;
      float w = 0.f;
      if (t < live) {
        const T* row = static_cast<const T*>(p.logits) + t * p.ld;
        float l[NPL];
        logits_of<NPL>(p, row, lane, l);
        const Choice<float> c = choose<float, NPL>(p, row, l, lane);
        id = c.unsure ? choose_in_double<NPL>(p, row, lane).x : c.id;
        w = share(id >= 0 ? logit(row, id) : 0.f, id >= 0, p.sigmoid, p.renorm, c.top, c.total) * p.scale;
      }
      if (lane < p.k) {
        p.ids[t * p.k + lane] = id;
        p.weights[t * p.k + lane] = id >= 0 ? w : 0.f;
        ids[i * p.k + lane] = static_cast<int16_t>(id);
        if (id >= 0) atomicOr(&chose[id][i >> 5], 1u << (i & 31));
      }
    }
    __syncthreads();
    if (!p.counts) {                                           // the only block: the experts' first rows are known here
      for (int e = threadIdx.x; e < p.E; e += blockDim.x) running[e] = __popc(chose[e][0]) + __popc(chose[e][1]);
      __syncthreads();
      if (warp == 0) offsets_of(running, p.E, lane);
      __syncthreads();
      for (int e = threadIdx.x; e <= p.E; e += blockDim.x) p.offsets[e] = running[e];
    }
    for (int s = threadIdx.x; s < tokens * p.k; s += blockDim.x) {
      const int i = s / p.k, e = ids[s];
      int at = -1;
      if (e >= 0) {
        const uint32_t below = (1u << (i & 31)) - 1u;
        at = running[e] + (i < 32 ? __popc(chose[e][0] & below) : __popc(chose[e][0]) + __popc(chose[e][1] & below));
      }
      p.places[sub * p.k + s] = at;
    }
    if (!p.counts) return;
    __syncthreads();
    for (int e = threadIdx.x; e < p.E; e += blockDim.x) running[e] += __popc(chose[e][0]) + __popc(chose[e][1]);
    __syncthreads();
  }
  for (int e = threadIdx.x; e < p.E2; e += blockDim.x) p.counts[blockIdx.x * static_cast<int64_t>(p.E2) + e] = e < p.E ? static_cast<uint16_t>(running[e]) : 0;
}

// Each block adds up the blocks' counts: its experts' first rows, and what the blocks before it have.
__global__ void __launch_bounds__(512) places_kernel(const __grid_constant__ Route p) {
  __shared__ int total[MAX_E + 1], before[MAX_E];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  pdl_trigger();
  pdl_wait();
  for (int e = threadIdx.x; e <= p.E; e += blockDim.x) {
    total[e] = 0;
    if (e < p.E) before[e] = 0;
  }
  __syncthreads();
  const int pairs = p.E2 / 2, strands = blockDim.x / pairs, strand = threadIdx.x / pairs, at = threadIdx.x - strand * pairs;
  if (strand < strands) {
    const uint32_t* counts = reinterpret_cast<const uint32_t*>(p.counts) + at;
    int all0 = 0, all1 = 0, own0 = 0, own1 = 0;
#pragma unroll 8
    for (int b = strand; b < static_cast<int>(gridDim.x); b += strands) {
      const uint32_t v = counts[b * static_cast<int64_t>(pairs)];
      const int lo = static_cast<int>(v & 0xFFFFu), hi = static_cast<int>(v >> 16);
      all0 += lo; all1 += hi;
      if (b < static_cast<int>(blockIdx.x)) { own0 += lo; own1 += hi; }
    }
    atomicAdd(&total[2 * at], all0);
    atomicAdd(&before[2 * at], own0);
    if (2 * at + 1 < p.E) {
      atomicAdd(&total[2 * at + 1], all1);
      atomicAdd(&before[2 * at + 1], own1);
    }
  }
  __syncthreads();
  if (warp == 0) offsets_of(total, p.E, lane);
  __syncthreads();
  if (blockIdx.x == 0)
    for (int e = threadIdx.x; e <= p.E; e += blockDim.x) p.offsets[e] = total[e];
  const int64_t begin = blockIdx.x * static_cast<int64_t>(p.chunk), end = min(begin + p.chunk, static_cast<int64_t>(p.T));
  for (int64_t s = begin * p.k + threadIdx.x; s < end * p.k; s += blockDim.x) {
    const int e = p.ids[s];
    if (e >= 0) p.places[s] += total[e] + before[e];
  }
}

// ---- backward ---------------------------------------------------------------------------------------------------------
struct RouteGrad {
  const void* logits;
  const int32_t* ids;
  const float* d_weights;
  void* d_logits;
  int64_t ld, ldd;
  int T, E, k, sigmoid, renorm, out_bf16;
  float scale;
};

template <typename T>
__global__ void __launch_bounds__(256) route_backward_kernel(const __grid_constant__ RouteGrad p) {
  const int lane = threadIdx.x & 31;
  const int64_t t = blockIdx.x * static_cast<int64_t>(blockDim.x >> 5) + (threadIdx.x >> 5);
  pdl_trigger();
  pdl_wait();
  if (t >= p.T) return;
  const T* row = static_cast<const T*>(p.logits) + t * p.ld;
  int id = lane < p.k ? p.ids[t * p.k + lane] : -1;
  if (id >= p.E) id = -1;
  const bool there = id >= 0;
  const float z = there ? logit(row, id) : 0.f, dw = there ? p.d_weights[t * p.k + lane] * p.scale : 0.f;
  float top = -CUDART_INF_F, total = 1.f, common = 0.f, own = 0.f;       // dl_e = -p_e common (softmax over all) + own of the slots with e
  const bool all = !p.sigmoid && !p.renorm;
  if (all) {
    for (int e = lane; e < p.E; e += 32) top = fmaxf(top, logit(row, e));
    top = warp_max(top);
    float sum = 0.f;
    for (int e = lane; e < p.E; e += 32) {
      const float v = logit(row, e);
      if (v != -CUDART_INF_F) sum += expf(v - top);
    }
    total = warp_sum(sum);
  }
  const float s = share(z, there, p.sigmoid, p.renorm, top, total);
  if (all) {
    const bool chosen = there && z != -CUDART_INF_F;
    own = chosen ? s * dw : 0.f;
    common = warp_sum(own);
  } else {
    const float mean = p.renorm ? warp_sum(there ? s * dw : 0.f) : 0.f;
    const float slope = p.sigmoid ? sigmoid(-z) : 1.f;  // (sigmoid(-z) = 1 - sigmoid(z))
    own = there ? s * slope * (dw - mean) : 0.f;
  }
  for (int first = 0; first < p.E; first += 32) {
    const int e = first + lane;
    float v = 0.f;
    if (all && e < p.E) {
      const float ze = logit(row, e);
      v = ze == -CUDART_INF_F ? 0.f : -common * __fdiv_rn(expf(ze - top), total);
    }
    for (int j = 0; j < p.k; ++j) {                            // (the same expert named twice gets both)
      const int ej = __shfl_sync(0xffffffffu, id, j);
      const float x = __shfl_sync(0xffffffffu, own, j);
      if (ej == e) v += x;
    }
    if (e < p.E) {
      if (p.out_bf16) static_cast<bf16*>(p.d_logits)[t * p.ldd + e] = __float2bfloat16_rn(v);
      else static_cast<float*>(p.d_logits)[t * p.ldd + e] = v;
    }
  }
}

// ---- launches ---------------------------------------------------------------------------------------------------------
int chunk_of(int64_t T) {
  int64_t chunk = ((T + MOST_BLOCKS - 1) / MOST_BLOCKS + SUB - 1) / SUB * SUB;
  return static_cast<int>(chunk < MOST_TOKENS ? chunk : MOST_TOKENS);
}
int64_t blocks_of(int64_t T) { return T <= SUB ? 1 : (T + chunk_of(T) - 1) / chunk_of(T); }

template <typename T> cudaError_t launch(const Route& p, dim3 grid, dim3 block, cudaStream_t stream) {
  if (p.E <= 32) return launch_pdl(route_kernel<T, 1>, grid, block, 0, stream, 1, p);
  if (p.E <= 64) return launch_pdl(route_kernel<T, 2>, grid, block, 0, stream, 1, p);
  if (p.E <= 128) return launch_pdl(route_kernel<T, 4>, grid, block, 0, stream, 1, p);
  if (p.E <= 256) return launch_pdl(route_kernel<T, 8>, grid, block, 0, stream, 1, p);
  return launch_pdl(route_kernel<T, 16>, grid, block, 0, stream, 1, p);
}

mbd_status done(cudaError_t e) {
  if (e == cudaSuccess) return MBD_OK;
  (void)cudaGetLastError();
  return MBD_E_CUDA;
}

mbd_status check(const mbd_router* r, int64_t T) {
  if (!r || T < 0 || r->experts < 1 || r->top_k < 1 || r->groups < 1 || r->top_groups < 1 || (r->group_best != 1 && r->group_best != 2) ||
      (r->score != MBD_ROUTE_SOFTMAX && r->score != MBD_ROUTE_SIGMOID) || !(r->scale - r->scale == 0.f)) return MBD_E_INVALID;
  if (r->experts % r->groups || r->top_groups > r->groups || r->top_k > r->experts / r->groups * r->top_groups) return MBD_E_INVALID;
  if (r->experts > MAX_E || r->top_k > MAX_K || r->groups > MAX_G || T > INT32_MAX / MAX_K) return MBD_E_UNSUPPORTED;
  return MBD_OK;
}

}  // namespace
}  // namespace mbd

using namespace mbd;

extern "C" int64_t mbd_expert_route_scratch(int64_t T, int E) {
  if (T <= SUB || E < 1) return 0;
  return blocks_of(T) * ((E + 1) / 2);
}

extern "C" mbd_status mbd_expert_route(const mbd_router* router, int64_t T, const void* logits_dev, int logits_bf16, int64_t ld, const float* bias_dev,
                                       const int32_t* count_dev, int32_t* ids_dev, float* weights_dev, int32_t* places_dev, int32_t* offsets_dev,
                                       int32_t* scratch_dev, void* cuda_stream) {
  const mbd_status st = check(router, T);
  if (st != MBD_OK) return st;
  const int E = router->experts, k = router->top_k;
  const int64_t words = mbd_expert_route_scratch(T, E);
  if (!offsets_dev || (T > 0 && (!logits_dev || !ids_dev || !weights_dev || !places_dev)) || (words && !scratch_dev)) return MBD_E_INVALID;
  if (T > 1 && ld < E) return MBD_E_INVALID;
  const Rows logits{T > 0 ? logits_dev : nullptr, T, E, ld, logits_bf16 ? 2 : 4}, bias{bias_dev, 1, E, E, 4}, count{count_dev, 1, 1, 1, 4};
  const Rows ids{T > 0 ? ids_dev : nullptr, 1, T * k, T * k, 4}, weights{T > 0 ? weights_dev : nullptr, 1, T * k, T * k, 4},
      places{T > 0 ? places_dev : nullptr, 1, T * k, T * k, 4}, offsets{offsets_dev, 1, E + 1, E + 1, 4}, scratch{words ? scratch_dev : nullptr, 1, words, words, 4};
  const Rows *in[] = {&logits, &bias, &count}, *out[] = {&ids, &weights, &places, &offsets, &scratch};
  for (const Rows* t : in)
    if (t->misplaced()) return MBD_E_UNSUPPORTED;
  for (const Rows* t : out)
    if (t->misplaced()) return MBD_E_UNSUPPORTED;
  for (const Rows* a : out) {
    for (const Rows* b : in)
      if (!apart(*a, *b)) return MBD_E_INVALID;
    for (const Rows* b : out)
      if (a != b && !apart(*a, *b)) return MBD_E_INVALID;
  }
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  if (T == 0) return done(cudaMemsetAsync(offsets_dev, 0, (static_cast<size_t>(E) + 1) * 4, stream));
  const uint32_t S = static_cast<uint32_t>(E / router->groups);
  const bool one = T <= SUB;
  const Route p{logits_dev, bias_dev, count_dev, ids_dev, places_dev, offsets_dev, weights_dev, one ? nullptr : reinterpret_cast<uint16_t*>(scratch_dev), ld,
                static_cast<int>(T), E, (E + 1) / 2 * 2, k, one ? SUB : chunk_of(T), router->score == MBD_ROUTE_SIGMOID, router->renormalise != 0,
                router->groups, router->top_groups, router->group_best, ((1u << 20) + S - 1) / S, router->scale};
  int warps = one ? 1 : 16;
  while (one && warps < T && warps < 32) warps *= 2;
  const dim3 grid(static_cast<unsigned>(blocks_of(T))), block(32 * warps);
  const cudaError_t e = logits_bf16 ? launch<bf16>(p, grid, block, stream) : launch<float>(p, grid, block, stream);
  if (e != cudaSuccess || one) return done(e);
  return done(launch_pdl(places_kernel, grid, dim3(512), 0, stream, 1, p));
}

extern "C" mbd_status mbd_expert_route_backward(const mbd_router* router, int64_t T, const void* logits_dev, int logits_bf16, int64_t ld,
                                                const int32_t* ids_dev, const float* d_weights_dev, void* d_logits_dev, int d_logits_bf16,
                                                int64_t ldd, void* cuda_stream) {
  const mbd_status st = check(router, T);
  if (st != MBD_OK) return st;
  if (T == 0) return MBD_OK;
  const int E = router->experts, k = router->top_k;
  if (!logits_dev || !ids_dev || !d_weights_dev || !d_logits_dev || (T > 1 && (ld < E || ldd < E))) return MBD_E_INVALID;
  const Rows logits{logits_dev, T, E, ld, logits_bf16 ? 2 : 4}, ids{ids_dev, 1, T * k, T * k, 4}, dw{d_weights_dev, 1, T * k, T * k, 4},
      out{d_logits_dev, T, E, ldd, d_logits_bf16 ? 2 : 4};
  for (const Rows* t : {&logits, &ids, &dw, &out})
    if (t->misplaced()) return MBD_E_UNSUPPORTED;
  if (!apart(out, logits) || !apart(out, ids) || !apart(out, dw)) return MBD_E_INVALID;
  const RouteGrad p{logits_dev, ids_dev, d_weights_dev, d_logits_dev, ld, ldd, static_cast<int>(T), E, k, router->score == MBD_ROUTE_SIGMOID,
                    router->renormalise != 0, d_logits_bf16 != 0, router->scale};
  const dim3 grid(static_cast<unsigned>((T + 7) / 8)), block(256);
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  return done(logits_bf16 ? launch_pdl(route_backward_kernel<bf16>, grid, block, 0, stream, 1, p)
                          : launch_pdl(route_backward_kernel<float>, grid, block, 0, stream, 1, p));
}
