// Routing of tokens to experts: from a token's scores of E experts the k best ones, their weights, and the places of the (token, slot)
// rows in the order of the experts that the products grouped by expert want; and the gradient of the logits.
//
//   p = softmax(l) or sigmoid(l);  key = p + bias, or the logit itself without a bias (the same order)
//   an expert whose logit or key is -inf is never chosen;  NaN keys come after all numbers
//   groups: a group's score is its best key, or the sum of its two best (without a bias: of its two best p);  only the best groups stay
//   the k largest keys, equal ones by rising index;  w = c p, or c p / (sum of the chosen p)
//
// One warp per token, a lane having NPL experts in a row.  Keys are integers, their lowest bits (one to four) giving way to the expert's
// place in the lane: a lane sorts its keys once by minima and maxima, and each choice is one warp-wide maximum, the first lane that has
// it, and that lane's list moving up.  Logits become integers of the same order.  Scores plus biases are counted in steps of 2^-30: a score next
// to one is known by what it lacks, which a float has to 4e-7 of itself, so that keys of the best experts are good to some 1e-8, where their
// sum as a float would be good to 1e-7.  What that cannot tell apart (unless logits and biases are the same) is settled in
// double, about one token in ten thousand: it costs a token's warp, and so the whole call, microseconds.  8150 tokens of 256 experts in groups, biases of
// 0.05: 17.5 us in nine of ten sets of inputs, 30 in the one with a token whose groups were settled so.  Keys are floats where a bias is beyond 0.99: one
// token in 300 is settled, 31 us.  Groups that tie are always settled: 66 us with logits and biases of zero, 75 without biases.  Without groups 14 us,
// 45 with equal logits (the list of what ties with the last choice is gone through).  Instructions bound large calls, about 1050 a token with groups; 16
// tokens take 3.3 us, the latency of one token and the sums over the experts.
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
constexpr int MOST_BLOCKS = 148, MOST_TOKENS = 65472;   // of the first kernel; of one of its blocks (counts are 16 bits wide)

struct Route {
  const void* logits;
  const float* bias;
  const int32_t* count;
  int32_t *ids, *places, *offsets;
  float* weights;
  uint16_t* counts;             // [blocks][E8]: slots of a block's tokens per expert; null: one block does it all
  int64_t ld;
  int T, E, E8, k, chunk;       // E8: E rounded up to a multiple of 8
  int whole;                    // rows of logits can be read in whole runs of a lane's experts
  int sigmoid, renorm, G, top_groups, best;
  uint32_t by_group;            // e / (E / G) = e * by_group >> 20
  int S, group_lanes, per;      // S: E / G; groups dealt out to lanes: 1 + log2 of the lanes of a group, and the experts of a lane; else 0
  float scale;
};

// ---- numbers as integers of the same order; 0: not there, NAN_CODE: NaN (below all numbers, with room for the low bits)
constexpr uint32_t NAN_CODE = 16;
__device__ __forceinline__ uint32_t code_of(float f) {
  const uint32_t u = __float_as_uint(f + 0.f);                 // (-0 is 0)
  return f != f ? NAN_CODE : u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t c) { return c <= 2 * NAN_CODE ? CUDART_NAN_F : __uint_as_float(c & 0x80000000u ? c ^ 0x80000000u : ~c); }
typedef unsigned long long code64;
__device__ __forceinline__ code64 code_of(double f) {
  const code64 u = static_cast<code64>(__double_as_longlong(f + 0.0));
  return f != f ? NAN_CODE : u >> 63 ? ~u : u | 0x8000000000000000ull;
}
__device__ __forceinline__ double value_of(code64 c) {
  return c <= NAN_CODE ? CUDART_NAN : __longlong_as_double(static_cast<long long>(c >> 63 ? c & 0x7FFFFFFFFFFFFFFFull : ~c));
}
__device__ __forceinline__ uint32_t largest(uint32_t c) { return __reduce_max_sync(0xffffffffu, c); }
__device__ __forceinline__ code64 largest(code64 c) {
  const uint32_t hi = static_cast<uint32_t>(c >> 32), top = largest(hi), low = largest(hi == top ? static_cast<uint32_t>(c) : 0u);
  return static_cast<code64>(top) << 32 | low;
}

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
__device__ __forceinline__ float sigmoid(float z) {
  const float t = expf(-fabsf(z));
  return __fdividef(z < 0.f ? t : 1.f, 1.f + t);
}
// Scores in steps of 2^-30, and how far they can be off.  small: what the score, or one minus the score, has, to 4e-7 of itself (the exponential
// an ulp, 1 + t half of one, its reciprocal one, the product half of one; a softmax has the error of its sum besides, 1.3e-6 common to all).
constexpr float STEPS = 1073741824.f;
__device__ __forceinline__ uint32_t steps_of(float small, bool lacks) {
  const uint32_t n = __float2uint_rn(small * STEPS);
  return lacks ? (1u << 30) - n : n;
}
__device__ __forceinline__ float sigmoid_small(float z) {      // min(sigmoid(z), sigmoid(-z))
  float r;
  const float t = expf(-fabsf(z));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + t));
  return t * r;
}

// Whether a group is among the best: lane l has the score of group l >> shift; equal ones by rising index.
template <typename C> __device__ __forceinline__ bool among_best(C mine, int shift, int groups, int top_groups, int lane) {
  int rank = 0;
  for (int g = 0; g < groups; ++g) {
    const C other = __shfl_sync(0xffffffffu, mine, g << shift);
    rank += other > mine || (other == mine && g < lane >> shift);
  }
  return mine && rank < top_groups;                            // (lanes behind the last group have 0)
}

// Scores in double, for what lies too near to each other for floats.  One exponential and one quotient for both kinds: this code is met
// seldom and then cold.
struct Exact { float top; double total; };
template <typename T> __device__ __noinline__ double exact_score(const Exact x, bool by_sigmoid, float z) {
  const double t = exp(by_sigmoid ? -fabs(static_cast<double>(z)) : static_cast<double>(z) - x.top);
  return (by_sigmoid && z >= 0.f ? 1.0 : t) / (by_sigmoid ? 1.0 + t : x.total);
}
template <typename T> __device__ __noinline__ Exact exact_sum(const Route& p, const T* row, int lane) {
  Exact x{-CUDART_INF_F, 1.0};
  if (p.sigmoid) return x;
  for (int e = lane; e < p.E; e += 32) x.top = fmaxf(x.top, logit(row, e));
  x.top = warp_max(x.top);
  double sum = 0.0;
#pragma unroll 1
  for (int e = lane; e < p.E; e += 32)
    if (logit(row, e) != -CUDART_INF_F) sum += exact_score<T>(x, false, logit(row, e));
  x.total = warp_sum(sum);
  return x;
}

// The whole choice in double: lane j gets the j-th expert, or -1.
template <typename T>
__device__ __noinline__ int choose_exactly(const Route& p, const T* row, const float* bias, int lane) {
  const bool by_two = p.G > 1 && p.best == 2, by_score = by_two && !p.bias;
  const int per = (p.E + 31) / 32, first_e = lane * per;
  code64 key[MAX_E / 32], count[MAX_E / 32];                   // what is chosen by, what a group counts: in local memory
  const Exact x = p.bias || by_score ? exact_sum(p, row, lane) : Exact{};
#pragma unroll 1
  for (int i = 0; i < per; ++i) {
    const int e = first_e + i;
    key[i] = count[i] = 0;
    if (e >= p.E) continue;
    const float z = logit(row, e);
    if (z == -CUDART_INF_F) continue;
    const double s = p.bias || by_score ? exact_score<T>(x, p.sigmoid, z) : 0.0;
    const double v = p.bias ? s + static_cast<double>(bias[e]) : z;
    if (v == -CUDART_INF) continue;
    key[i] = code_of(v);
    count[i] = by_score ? code_of(s) : key[i];
  }
  if (p.G > 1) {
    const int S = p.S;
    code64 mine = 0;                                           // lane g: the score of group g
#pragma unroll 1
    for (int g = 0; g < p.G; ++g) {
      code64 a = 0, b = 0;                                     // this lane's two best of the group
      const int from = max(g * S - first_e, 0), to = min(g * S + S - first_e, per);
#pragma unroll 1
      for (int i = from; i < to; ++i) {
        const code64 v = count[i];
        if (v > a) { b = a; a = v; }
        else if (v > b) b = v;
      }
      const code64 first = largest(a);
      code64 of = first;
      if (p.best == 2 && first) {
        const unsigned owners = __ballot_sync(0xffffffffu, a == first);
        const code64 second = largest(lane == __ffs(owners) - 1 ? b : a);
        of = code_of(value_of(first) + (second ? value_of(second) : 0.0));
      }
      if (lane == g) mine = of;
    }
    const unsigned kept = __ballot_sync(0xffffffffu, among_best(mine, 0, p.G, p.top_groups, lane));
#pragma unroll 1
    for (int i = 0; i < per; ++i)
      if (first_e + i < p.E && !(kept >> (first_e + i) / S & 1u)) key[i] = 0;
  }
  int id = -1;
#pragma unroll 1
  for (int j = 0; j < p.k; ++j) {
    code64 best = 0;
    int at = 0;
#pragma unroll 1
    for (int i = 0; i < per; ++i)
      if (key[i] > best) { best = key[i]; at = i; }
    const code64 first = largest(best);
    if (!first) break;
    const int src = __ffs(__ballot_sync(0xffffffffu, best == first)) - 1;
    if (lane == src) key[at] = 0;
    const int e = __shfl_sync(0xffffffffu, first_e + at, src);
    if (lane == j) id = e;
  }
  return id;
}

// The order of n experts (lane j < n has one, `id`) whose keys lie near to each other, in double: lane j gets the j-th.
template <typename T>
__device__ __noinline__ int settle(const Route& p, const T* row, const float* bias, int id, int n, int lane) {
  const float z = lane < n ? logit(row, id) : 0.f;
  double v = z;
  if (p.bias) v = exact_score<T>(exact_sum(p, row, lane), p.sigmoid, z) + (lane < n ? static_cast<double>(bias[id]) : 0.0);
  const code64 mine = code_of(v);
  int rank = 0;
  for (int j = 0; j < n; ++j) {
    const code64 other = __shfl_sync(0xffffffffu, mine, j);
    const int e = __shfl_sync(0xffffffffu, id, j);
    rank += other > mine || (other == mine && e < id);
  }
  int got = -1;
  for (int j = 0; j < n; ++j) {
    const int src = __ffs(__ballot_sync(0xffffffffu, lane < n && rank == j)) - 1;
    const int e = __shfl_sync(0xffffffffu, id, src);
    if (lane == j) got = e;
  }
  return got;
}

// NPL logits of a lane, experts `first` on; -inf behind its `count`.
template <int NPL, typename T>
__device__ __forceinline__ void logits_of(const T* row, int first, int count, bool whole, float (&l)[NPL]) {
  if (NPL * sizeof(T) >= 4 && whole) {                         // whole runs of NPL, aligned
    if (count == 0) {
#pragma unroll
      for (int i = 0; i < NPL; ++i) l[i] = -CUDART_INF_F;
      return;
    }
    constexpr int WORDS = NPL * static_cast<int>(sizeof(T)) / 4 > 0 ? NPL * static_cast<int>(sizeof(T)) / 4 : 1;
    uint32_t w[WORDS];
    const uint32_t* at = reinterpret_cast<const uint32_t*>(row + first);
    if constexpr (WORDS >= 4) {
#pragma unroll
      for (int i = 0; i < WORDS; i += 4) {
        const uint4 v = *reinterpret_cast<const uint4*>(at + i);
        w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
      }
    } else if constexpr (WORDS == 2) {
      const uint2 v = *reinterpret_cast<const uint2*>(at);
      w[0] = v.x; w[1] = v.y;
    } else {
      w[0] = *at;
    }
#pragma unroll
    for (int i = 0; i < NPL; ++i)
      l[i] = __uint_as_float(sizeof(T) == 4 ? w[i] : i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
  } else {
#pragma unroll
    for (int i = 0; i < NPL; ++i) l[i] = i < count ? logit(row, first + i) : -CUDART_INF_F;
  }
}

__device__ __forceinline__ void order(uint32_t& a, uint32_t& b) {
  const uint32_t hi = max(a, b);
  b = min(a, b);
  a = hi;
}
// Falling order, by Batcher's odd-even merges.
template <int N> __device__ __forceinline__ void sort_falling(uint32_t (&s)[N]) {
#pragma unroll
  for (int p = 1; p < N; p *= 2)
#pragma unroll
    for (int k = p; k >= 1; k /= 2)
#pragma unroll
      for (int j = k % p; j + k < N; j += 2 * k)
#pragma unroll
        for (int i = 0; i < k; ++i)
          if (i + j + k < N && (i + j) / (2 * p) == (i + j + k) / (2 * p)) order(s[i + j], s[i + j + k]);
}

// A token's choice: lane j < chosen has the j-th expert.  top, total: the largest logit and the sum of exp(l - top), where a
// softmax needs them.
struct Choice { int id; float z, top, total; bool unsure; };          // z: the logit of expert id

// first_e: the lane's first expert.  list: k words of the warp's in shared memory.  Keys with a bias: fixed if all biases are within 0.99,
// (score + bias + 1) 2^30, the biases' share in shared memory; else the float sum's code.
template <int NPL, typename T>
__device__ __forceinline__ Choice choose(const Route& p, const T* row, const float (&l)[NPL], const float* bias, const uint32_t* bias_steps, bool fixed, uint2* list,
                                        int first_e, int lane) {
  constexpr uint32_t LOW = NPL - 1;
  const bool by_two = p.G > 1 && p.best == 2, scored = p.bias || by_two;      // whether the choice needs more than the order of the logits
  Choice c{-1, 0.f, -CUDART_INF_F, 1.f, false};
  if (!p.sigmoid && (scored || !p.renorm)) {
#pragma unroll
    for (int i = 0; i < NPL; ++i) c.top = fmaxf(c.top, l[i]);
    c.top = warp_max(c.top);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NPL; ++i)
      if (l[i] != -CUDART_INF_F) sum += expf(l[i] - c.top);
    c.total = warp_sum(sum);
  }
  const float inv_total = p.sigmoid ? 1.f : __fdividef(1.f, c.total);
  auto small = [&](float z) { return p.sigmoid ? sigmoid_small(z) : expf(z - c.top) * inv_total; };
  auto steps = [&](float z, bool by_sigmoid) {                 // one in front
    const float s = by_sigmoid ? sigmoid_small(z) : expf(z - c.top) * inv_total;
    return s != s ? NAN_CODE : (1u << 30) + steps_of(s, by_sigmoid && z >= 0.f);
  };
  auto in_steps = [&](float z, uint32_t bias, bool by_sigmoid) {
    const uint32_t s = steps(z, by_sigmoid);
    return z == -CUDART_INF_F ? 0u : s == NAN_CODE ? s : s + bias;
  };
  uint32_t key[NPL];
  if (p.bias && fixed) {
    if (p.sigmoid) {
#pragma unroll
      for (int i = 0; i < NPL; ++i) key[i] = in_steps(l[i], bias_steps[first_e + i], true);
    } else {
#pragma unroll
      for (int i = 0; i < NPL; ++i) key[i] = in_steps(l[i], bias_steps[first_e + i], false);
    }
#pragma unroll
    for (int i = 0; i < NPL; ++i) key[i] = key[i] ? (key[i] & ~LOW) | (LOW - i) : 0u;
  } else if (p.bias) {
#pragma unroll
    for (int i = 0; i < NPL; ++i) {
      key[i] = 0;
      if (l[i] != -CUDART_INF_F) {
        const float s = small(l[i]), v = (p.sigmoid && l[i] >= 0.f ? 1.f - s : s) + bias[first_e + i];
        if (v != -CUDART_INF_F) key[i] = (code_of(v) & ~LOW) | (LOW - i);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < NPL; ++i) key[i] = l[i] != -CUDART_INF_F ? (code_of(l[i]) & ~LOW) | (LOW - i) : 0u;
  }
  // A lane's two best by all of their bits, where a group counts by their scores: the keys cannot tell logits up to NPL - 1 units apart, which
  // are 1e-4 of a score at logits of 100.
  const bool by_score = by_two && !p.bias;
  uint32_t best_a = 0, best_b = 0;
  if (by_score && p.group_lanes) {
#pragma unroll
    for (int i = 0; i < NPL; ++i) {
      const uint32_t v = l[i] != -CUDART_INF_F ? code_of(l[i]) : 0u;
      best_b = max(best_b, min(best_a, v));
      best_a = max(best_a, v);
    }
  }
  sort_falling(key);
  // How far the gap between two keys can be off, in steps or (keys that are sums of floats) by value.  Of a score: 4e-7 of the largest small
  // part there is, a half or the largest p, whose sum's error counts with it; the steps' rounding and the bits given away.
  const float part = p.sigmoid ? 0.5f : inv_total;
  const float relative = p.sigmoid ? 4e-7f : 2e-6f, coarse = 2.f * relative * part;
  const float coarse_float = coarse + (p.sigmoid ? 2e-7f : 0.f);              // (one minus the small part is rounded there, too)
  if (p.G > 1) {
    const bool sums = by_two && (fixed || by_score);
    // a key as a group counts it
    auto counted = [&](uint32_t k) { return by_score && k ? steps(logit(row, first_e + static_cast<int>(LOW - (k & LOW))), p.sigmoid) : k & ~LOW; };
    auto group_score = [&](uint32_t first, uint32_t second) {
      if (p.best == 1 || !first) return first;
      if (first <= 2 * NAN_CODE || (second && second <= 2 * NAN_CODE)) return NAN_CODE;
      if (sums) return first / 2 + (second ? second / 2 : 1u << 29);             // (both have one in front)
      return code_of(0.5f * value_of(first) + (second ? 0.5f * value_of(second) : 0.f));   // (halves: no sum is beyond a float)
    };
    uint32_t mine, one = 0, two = 0;                           // the score of this lane's group, or of group `lane`, and the keys it is made of
    bool keep;
    if (p.group_lanes) {                                       // a lane has experts of one group, a group 1, 2, 4 .. lanes
      uint32_t a = key[0] & ~LOW, b = NPL > 1 ? key[NPL > 1 ? 1 : 0] & ~LOW : 0u;
      if (by_score) {
        a = best_a ? steps(value_of(best_a), p.sigmoid) : 0u;
        b = best_b ? steps(value_of(best_b), p.sigmoid) : 0u;
        order(a, b);                                           // (two scores next to each other may be off by a step)
      }
      for (int d = 1; d < 1 << (p.group_lanes - 1); d *= 2) {
        const uint32_t a2 = __shfl_xor_sync(0xffffffffu, a, d), b2 = __shfl_xor_sync(0xffffffffu, b, d);
        b = max(min(a, a2), max(b, b2));
        a = max(a, a2);
      }
      one = a;
      two = b;
      mine = group_score(a, b);
      keep = among_best(mine, p.group_lanes - 1, p.G, p.top_groups, lane);
      if (!keep) {
#pragma unroll
        for (int i = 0; i < NPL; ++i) key[i] = 0;
      }
    } else {
      mine = 0;
      for (int g = 0; g < p.G; ++g) {
        uint32_t a = 0, b = 0;
#pragma unroll
        for (int i = 0; i < NPL; ++i) {
          const int e = first_e + static_cast<int>(LOW - (key[i] & LOW));
          if (key[i] == 0 || static_cast<int>(e * p.by_group >> 20) != g) continue;
          const uint32_t v = counted(key[i]);
          if (v > a) { b = a; a = v; }
          else if (v > b) b = v;
        }
        const uint32_t first = largest(a), owners = __ballot_sync(0xffffffffu, a == first);
        const uint32_t second = largest(lane == __ffs(owners) - 1 ? b : a);
        if (lane == g) {
          one = first;
          two = second;
          mine = group_score(first, second);
        }
      }
      keep = among_best(mine, 0, p.G, p.top_groups, lane);
      const unsigned kept = __ballot_sync(0xffffffffu, keep);
#pragma unroll
      for (int i = 0; i < NPL; ++i) {
        const int e = first_e + static_cast<int>(LOW - (key[i] & LOW));
        if (!(kept >> (e * p.by_group >> 20 & 31u) & 1u)) key[i] = 0;
      }
      sort_falling(key);
    }
    const uint32_t in = ~largest(keep ? ~mine : 0u), out = largest(keep ? 0u : mine);
    if (out && in != ~0u) {
      // (two groups of equal logits, by their best: the lower one, as it should be, if the bits given away are zeros anyway)
      if (!scored) c.unsure = sizeof(T) == 4 && in == out;
      else if (fixed || by_score)                              // (of two: twice as far off, in steps twice as long)
        c.unsure = out <= 2 * NAN_CODE || in - out <= static_cast<uint32_t>(coarse * STEPS) + 2 * NPL + 4;
      else {                                                   // each key is off by its own size, which a sum of two may be far below
        const float a = value_of(one), b = p.best == 2 && two ? value_of(two) : 0.f, score = value_of(mine);
        float off = 0.5f * coarse_float + (NPL + 2) * 1.2e-7f * (p.best == 2 ? 0.5f * fabsf(a) + 0.5f * fabsf(b) : fabsf(a));
        if (a == CUDART_INF_F) off = 0.f;                      // (as it is in exact arithmetic)
        c.unsure = ~largest(keep ? ~code_of(score - off) : 0u) <= largest(keep || !mine ? 0u : code_of(score + off));
      }
    }
  }
  for (int j = 0; j < p.k; ++j) {
    const uint32_t own = key[0] & ~LOW, first = largest(own);
    if (lane == __ffs(__ballot_sync(0xffffffffu, own == first)) - 1) {
      list[j] = make_uint2(first, first ? first_e + (LOW - (key[0] & LOW)) : ~0u);
#pragma unroll
      for (int i = 0; i + 1 < NPL; ++i) key[i] = key[i + 1];
      key[NPL - 1] = 0;
    }
  }
  __syncwarp();
  const uint2 got = lane < p.k ? list[lane] : make_uint2(0u, ~0u);
  const uint32_t mine = got.x;
  const int chosen = __popc(__ballot_sync(0xffffffffu, mine != 0));
  c.id = static_cast<int>(got.y);
  if (c.id >= 0) c.z = logit(row, c.id);
  if (!p.bias && sizeof(T) == 2) return c;                     // (logits of bf16 end in zeros: nothing was given away)
  if (c.unsure) return c;
  // Neighbours in the order, and the last one against those that are left; equal logits with equal biases are really equal.  A first look by
  // the largest error there can be, a second one by the two experts' own small parts.
  const uint32_t reach = p.bias && fixed ? static_cast<uint32_t>(coarse * STEPS) + NPL + 4 : 0u;
  auto close = [&](uint32_t hi, uint32_t lo) {
    if (!p.bias || fixed) return hi - lo <= reach || lo <= 2 * NAN_CODE;
    const float v = value_of(hi);
    return !(v - value_of(lo) > coarse_float + (NPL + 2) * 1.2e-7f * fabsf(v));
  };
  const uint32_t next = __shfl_down_sync(0xffffffffu, mine, 1), last = __shfl_sync(0xffffffffu, mine, p.k - 1), left = key[0] & ~LOW;
  const bool near_next = lane + 1 < chosen && close(mine, next), near_left = chosen == p.k && left && close(last, left);
  if (__any_sync(0xffffffffu, near_next || near_left)) {
    const float z = c.z, b = c.id >= 0 && p.bias ? bias[c.id] : 0.f, s = p.bias && fixed && c.id >= 0 ? small(z) : 0.f;
    auto differ = [&](uint32_t hi, uint32_t lo, float z1, float b1, float s1, float z2, float b2, float s2) {
      if (z1 == z2 && b1 == b2) return false;
      if (!(p.bias && fixed) || hi <= 2 * NAN_CODE || lo <= 2 * NAN_CODE) return true;
      return hi - lo <= static_cast<uint32_t>(relative * (s1 + s2) * STEPS) + NPL + 4;
    };
    const float z2 = __shfl_down_sync(0xffffffffu, z, 1), b2 = __shfl_down_sync(0xffffffffu, b, 1), s2 = __shfl_down_sync(0xffffffffu, s, 1);
    bool near = near_next && differ(mine, next, z, b, s, z2, b2, s2);
    int n = chosen, id = c.id;                                 // with the keys that are left and near to the last one
    if (__any_sync(0xffffffffu, near_left)) {
      const float zk = __shfl_sync(0xffffffffu, z, p.k - 1), bk = __shfl_sync(0xffffffffu, b, p.k - 1), sk = __shfl_sync(0xffffffffu, s, p.k - 1);
#pragma unroll
      for (int i = 0; i < NPL; ++i) {
        const int e = first_e + static_cast<int>(LOW - (key[i] & LOW));
        const bool may = key[i] && close(last, key[i] & ~LOW);
        if (may) {
          const float ze = logit(row, e);
          near |= differ(last, key[i] & ~LOW, zk, bk, sk, ze, p.bias ? bias[e] : 0.f, p.bias && fixed ? small(ze) : 0.f);
        }
        for (unsigned who = __ballot_sync(0xffffffffu, may); who; who &= who - 1) {
          const int other = __shfl_sync(0xffffffffu, e, __ffs(who) - 1);
          if (lane == n) id = other;
          ++n;
        }
      }
    }
    if (__any_sync(0xffffffffu, near)) {
      c.unsure = n > 32;
      if (!c.unsure) {
        id = settle(p, row, bias, id, n, lane);
        c.id = lane < chosen ? id : -1;
        c.z = c.id >= 0 ? logit(row, c.id) : 0.f;
      }
    }
  }
  return c;
}

// The weight of lane j's expert, of logit z; total: over all experts.  Renormalised scores are taken relative to the largest
// chosen one, so that scores below float's range keep their ratios: a softmax always, sigmoids where one of them is next to the end of the range
// (exp(-87)) and none is a half or more (the quotients are as small as the scores then); sigmoid(z) exp(-most) = exp(z - most) / (1 + exp(z)).
__device__ __forceinline__ float share(float z, bool there, bool by_sigmoid, bool renorm, float top, float total) {
  if (!renorm) return there ? (by_sigmoid ? sigmoid(z) : __fdividef(expf(z - top), total)) : 0.f;
  const bool tiny = by_sigmoid && __any_sync(0xffffffffu, there && z < -80.f) && !__any_sync(0xffffffffu, there && z >= 0.f);
  const float most = !by_sigmoid || tiny ? warp_max(there ? z : -CUDART_INF_F) : 0.f;
  float r = !there || z == -CUDART_INF_F ? 0.f : by_sigmoid && !tiny ? sigmoid(z) : expf(z - most);
  if (tiny) r = __fdividef(r, 1.f + expf(z));
  const float sum = warp_sum(r);
  return there && sum != 0.f ? __fdiv_rn(r, sum) : 0.f;       // (the only one chosen: exactly 1, and its gradient exactly 0)
}

// Exclusive sums of E numbers in shared memory, by a block of at least as many threads; all of them go behind the last.
__device__ __forceinline__ void offsets_of(int* n, int E) {
  __shared__ int totals[32];
  const int e = threadIdx.x, lane = e & 31, warp = e >> 5, own = e < E ? n[e] : 0;
  int sum = own;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, sum, d);
    if (lane >= d) sum += v;
  }
  if (lane == 31) totals[warp] = sum;
  __syncthreads();
  if (e < E) {
#pragma unroll
    for (int w = 0; w < MAX_E / 32 - 1; ++w)
      if (w < warp) sum += totals[w];
    n[e] = sum - own;
    if (e == E - 1) n[E] = sum;
  }
  __syncthreads();
}

template <typename T, int NPL>
__global__ void __launch_bounds__(1024) route_kernel(const __grid_constant__ Route p) {
  __shared__ uint32_t chose[MAX_E][SUB / 32];
  __shared__ int running[MAX_E + 1];
  __shared__ int16_t ids[SUB * MAX_K];
  __shared__ uint2 lists[32][MAX_K];
  __shared__ __align__(16) float bias[MAX_E + 16];               // (a lane with fewer experts than places looks behind its last)
  __shared__ __align__(16) uint32_t bias_steps[MAX_E + 16];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  pdl_trigger();
  pdl_wait();
  // this lane's experts, those of one group where groups are dealt out to lanes
  int first_e = lane * NPL, count = min(max(p.E - first_e, 0), NPL);
  if (p.group_lanes) {
    const int g = lane >> (p.group_lanes - 1), q = (lane & ((1 << (p.group_lanes - 1)) - 1)) * p.per;
    first_e = g < p.G ? g * p.S + min(q, p.S) : 0;
    count = g < p.G ? min(max(p.S - q, 0), p.per) : 0;
  }
  const int live = p.count ? min(max(*p.count, 0), p.T) : p.T;
  int fits = 1;
  for (int e = threadIdx.x; e <= p.E; e += blockDim.x) {
    running[e] = 0;
    if (p.bias && e < p.E) {
      const float b = p.bias[e];
      bias[e] = b;
      fits &= fabsf(b) <= 0.99f;
      bias_steps[e] = static_cast<uint32_t>(__float2int_rn(b * STEPS));        // (exact but for the rounding to a step; negative ones wrap around)
    }
  }
  const bool fixed = __syncthreads_and(fits);
  const int64_t begin = blockIdx.x * static_cast<int64_t>(p.chunk), end = min(begin + p.chunk, static_cast<int64_t>(p.T));
  for (int64_t sub = begin; sub < end; sub += SUB) {
    for (int e = threadIdx.x; e < p.E * (SUB / 32); e += blockDim.x) chose[0][e] = 0u;
    __syncthreads();
    const int tokens = static_cast<int>(min(end - sub, static_cast<int64_t>(SUB)));
    constexpr bool AHEAD = NPL < 16;                           // (with 16 more registers a thread 512 threads fit, not 1024: 16384 tokens of 512 experts took 107 instead of 99 us)
    float next[NPL];                                           // the warp's next token is on its way
    if (AHEAD && warp < tokens) logits_of<NPL>(static_cast<const T*>(p.logits) + (sub + warp) * p.ld, first_e, count, p.whole, next);
    for (int i = warp; i < tokens; i += warps) {
      const int64_t t = sub + i;
      int id = -1;
      float w = 0.f, l[NPL];
#pragma unroll
      for (int m = 0; m < NPL; ++m) l[m] = AHEAD ? next[m] : 0.f;
      if (!AHEAD) logits_of<NPL>(static_cast<const T*>(p.logits) + t * p.ld, first_e, count, p.whole, l);
      else if (i + warps < tokens) logits_of<NPL>(static_cast<const T*>(p.logits) + (t + warps) * p.ld, first_e, count, p.whole, next);
      if (t < live) {
        const T* row = static_cast<const T*>(p.logits) + t * p.ld;
        const Choice c = choose<NPL>(p, row, l, bias, bias_steps, fixed, lists[warp], first_e, lane);
        float z = c.z;
        id = c.id;
        if (c.unsure) {
          id = choose_exactly(p, row, bias, lane);
          z = id >= 0 ? logit(row, id) : 0.f;
        }
        w = share(z, id >= 0, p.sigmoid, p.renorm, c.top, c.total) * p.scale;
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
      offsets_of(running, p.E);
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
  for (int e = threadIdx.x; e < p.E8; e += blockDim.x) p.counts[blockIdx.x * static_cast<int64_t>(p.E8) + e] = e < p.E ? static_cast<uint16_t>(running[e]) : 0;
}

// Each block takes the slots of one block of the kernel above: it adds up all blocks' counts, which gives the experts' first rows, and those
// of the blocks before its own; eight experts a thread, the blocks dealt out to STRANDS threads, all of whose loads are under way at once.  About 5 us
// with its launch: four dependent round trips and barriers.
constexpr int STRANDS = 8;
__global__ void __launch_bounds__(512) places_kernel(const __grid_constant__ Route p) {
  __shared__ int total[MAX_E + 1], before[MAX_E];
  __shared__ __align__(16) int all[STRANDS][MAX_E], earlier[STRANDS][MAX_E];
  const int blocks = gridDim.x, own = blockIdx.x;
  const int64_t begin = own * static_cast<int64_t>(p.chunk) * p.k, end = min((own + 1) * static_cast<int64_t>(p.chunk), static_cast<int64_t>(p.T)) * p.k;
  pdl_trigger();
  pdl_wait();
  const int64_t slot = begin + threadIdx.x;                    // the first of this thread's slots is on its way meanwhile
  const int first_id = slot < end ? p.ids[slot] : -1, first_place = slot < end ? p.places[slot] : -1;
  const int eights = p.E8 / 8, strand = threadIdx.x / eights, at = threadIdx.x - strand * eights;
  if (strand < STRANDS) {
    const uint4* counts = reinterpret_cast<const uint4*>(p.counts) + at;
    int n[8] = {}, m[8] = {};
#pragma unroll 10
    for (int b = strand; b < blocks; b += STRANDS) {
      const uint4 v = counts[b * static_cast<int64_t>(eights)];
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
      const int before_own = b < own ? -1 : 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int c = static_cast<int>(i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xFFFFu);
        n[i] += c;
        m[i] += c & before_own;
      }
    }
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      *reinterpret_cast<int4*>(&all[strand][8 * at + i]) = make_int4(n[i], n[i + 1], n[i + 2], n[i + 3]);
      *reinterpret_cast<int4*>(&earlier[strand][8 * at + i]) = make_int4(m[i], m[i + 1], m[i + 2], m[i + 3]);
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < p.E; e += blockDim.x) {
    int n = 0, m = 0;
#pragma unroll
    for (int s = 0; s < STRANDS; ++s) {
      n += all[s][e];
      m += earlier[s][e];
    }
    total[e] = n;
    before[e] = m;
  }
  __syncthreads();
  offsets_of(total, p.E);
  if (own == 0)
    for (int e = threadIdx.x; e <= p.E; e += blockDim.x) p.offsets[e] = total[e];
  if (first_id >= 0) p.places[slot] = first_place + total[first_id] + before[first_id];
  for (int64_t s = slot + blockDim.x; s < end; s += blockDim.x) {
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
  int T, E, k, sigmoid, renorm, out_bf16, pairs;      // pairs: two elements of the result at a time
  float scale;
};

// One warp per token; its row of the result is put together in shared memory, the slots' shares one after the other (the same expert
// named twice gets both).  16384 x 512 floats of 12 slots: 20 us (3.4 TB/s); 8192 x 64 bf16 5 us, latency.
constexpr int GRAD_WARPS = 8;
template <typename T>
__global__ void __launch_bounds__(32 * GRAD_WARPS) route_backward_kernel(const __grid_constant__ RouteGrad p) {
  __shared__ __align__(16) float rows[GRAD_WARPS][MAX_E];
  const int lane = threadIdx.x & 31;
  const int64_t t = blockIdx.x * static_cast<int64_t>(GRAD_WARPS) + (threadIdx.x >> 5);
  float* out = rows[threadIdx.x >> 5];
  pdl_trigger();
  pdl_wait();
  if (t >= p.T) return;
  const T* row = static_cast<const T*>(p.logits) + t * p.ld;
  int id = lane < p.k ? p.ids[t * p.k + lane] : -1;
  if (id >= p.E) id = -1;
  const bool there = id >= 0;
  const float z = there ? logit(row, id) : 0.f, dw = there ? p.d_weights[t * p.k + lane] * p.scale : 0.f;
  float top = -CUDART_INF_F, total = 1.f, own;
  const bool all = !p.sigmoid && !p.renorm;              // every logit has a part: dl_e = own of the slots with e - p_e * (sum of own)
  if (all) {
    for (int e = lane; e < p.E; e += 32) {
      const float l = logit(row, e);
      out[e] = l;
      top = fmaxf(top, l);
    }
    top = warp_max(top);
    float sum = 0.f;
    for (int e = lane; e < p.E; e += 32) {
      const float l = out[e], v = l == -CUDART_INF_F ? 0.f : expf(l - top);
      out[e] = v;
      sum += v;
    }
    total = warp_sum(sum);
  }
  const float s = share(z, there, p.sigmoid, p.renorm, top, total);
  if (all) {
    own = there && z != -CUDART_INF_F ? s * dw : 0.f;
    const float common = -__fdividef(warp_sum(own), total);
    for (int e = lane; e < p.E; e += 32) out[e] = out[e] == 0.f ? 0.f : common * out[e];      // (a masked expert has none, whatever the total)
  } else {
    const float mean = p.renorm ? warp_sum(there ? s * dw : 0.f) : 0.f;
    const float slope = p.sigmoid ? sigmoid(-z) : 1.f;   // (sigmoid(-z) = 1 - sigmoid(z))
    own = there ? s * slope * (dw - mean) : 0.f;
    for (int e = lane; e < p.E; e += 32) out[e] = 0.f;
  }
  __syncwarp();
  for (int j = 0; j < p.k; ++j) {
    if (lane == j && there) out[id] += own;
    __syncwarp();
  }
  if (p.out_bf16) {
    bf16* to = static_cast<bf16*>(p.d_logits) + t * p.ldd;
    if (p.pairs)
      for (int e = lane; e < p.E / 2; e += 32) {
        const float2 v = *reinterpret_cast<const float2*>(out + 2 * e);
        *reinterpret_cast<uint32_t*>(to + 2 * e) = pack_bf16x2(v.x, v.y);
      }
    else
      for (int e = lane; e < p.E; e += 32) to[e] = __float2bfloat16_rn(out[e]);
  } else {
    float* to = static_cast<float*>(p.d_logits) + t * p.ldd;
    if (p.pairs)
      for (int e = lane; e < p.E / 2; e += 32) *reinterpret_cast<float2*>(to + 2 * e) = *reinterpret_cast<const float2*>(out + 2 * e);
    else
      for (int e = lane; e < p.E; e += 32) to[e] = out[e];
  }
}

// ---- launches ---------------------------------------------------------------------------------------------------------
// Tokens of a block: 16 or more, but at most MOST_BLOCKS blocks, one per SM.
int chunk_of(int64_t T) {
  int64_t chunk = ((T + MOST_BLOCKS - 1) / MOST_BLOCKS + 7) / 8 * 8;
  if (chunk < 16) chunk = 16;
  return static_cast<int>(chunk < MOST_TOKENS ? chunk : MOST_TOKENS);
}
int64_t blocks_of(int64_t T) { return T <= SUB ? 1 : (T + chunk_of(T) - 1) / chunk_of(T); }

template <typename T, int NPL> cudaError_t launch_npl(Route p, dim3 grid, dim3 block, cudaStream_t stream) {
  constexpr uint64_t BYTES = NPL * sizeof(T) < 16 ? NPL * sizeof(T) : 16;
  p.whole = p.E % NPL == 0 && (!p.group_lanes || (p.per == NPL && p.S % NPL == 0)) && reinterpret_cast<uintptr_t>(p.logits) % BYTES == 0 && (p.T <= 1 || static_cast<uint64_t>(p.ld) * sizeof(T) % BYTES == 0);
  return launch_pdl(route_kernel<T, NPL>, grid, block, 0, stream, 1, p);
}
template <typename T> cudaError_t launch(Route p, dim3 grid, dim3 block, cudaStream_t stream) {
  int per = (p.E + 31) / 32;
  if (p.G > 1) {                                               // 1, 2, 4 .. lanes a group, if its experts find room in them
    int log_lanes = 0;
    while (p.G << (log_lanes + 1) <= 32) ++log_lanes;
    const int of_lane = (p.S + (1 << log_lanes) - 1) >> log_lanes;
    if (of_lane <= 16) {
      p.group_lanes = 1 + log_lanes;
      p.per = per = of_lane;
    }
  }
  if (per <= 1) return launch_npl<T, 1>(p, grid, block, stream);
  if (per <= 2) return launch_npl<T, 2>(p, grid, block, stream);
  if (per <= 4) return launch_npl<T, 4>(p, grid, block, stream);
  if (per <= 8) return launch_npl<T, 8>(p, grid, block, stream);
  return launch_npl<T, 16>(p, grid, block, stream);
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
  return blocks_of(T) * ((E + 7) / 8 * 4);
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
  if (words && reinterpret_cast<uintptr_t>(scratch_dev) % 16) return MBD_E_UNSUPPORTED;
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
                static_cast<int>(T), E, (E + 7) / 8 * 8, k, one ? SUB : chunk_of(T), 0, router->score == MBD_ROUTE_SIGMOID, router->renormalise != 0,
                router->groups, router->top_groups, router->group_best, ((1u << 20) + S - 1) / S, static_cast<int>(S), 0, 0, router->scale};
  int warps = (E + 31) / 32;                                  // (a thread per expert at least)
  while (warps < (one ? T : chunk_of(T)) && warps < 32) ++warps;
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
                    router->renormalise != 0, d_logits_bf16 != 0,
                    E % 2 == 0 && (T == 1 || ldd % 2 == 0) && reinterpret_cast<uintptr_t>(d_logits_dev) % (2 * out.size) == 0, router->scale};
  const dim3 grid(static_cast<unsigned>((T + GRAD_WARPS - 1) / GRAD_WARPS)), block(32 * GRAD_WARPS);
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  return done(logits_bf16 ? launch_pdl(route_backward_kernel<bf16>, grid, block, 0, stream, 1, p)
                          : launch_pdl(route_backward_kernel<float>, grid, block, 0, stream, 1, p));
}
