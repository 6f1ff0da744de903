// Products grouped by expert on the 5th-generation tensor cores (tcgen05): the three contractions of a layer
// (Section 1 of the paper) where every row of the batch belongs to one of E experts with a weight matrix of its own,
// and the product of 8-bit integers with a scale per row and per channel, dense or grouped.
//
//   variant 0  Y[r, :]  = X[r, :]  W_e^T          rows o[e] <= r < o[e+1]
//   variant 1  dX[r, :] = dY[r, :] W_e
//   variant 2  dW_e     = sum_{r in e} dY[r, :]^T X[r, :]
//
// The group sizes are known on the device only.  The output's CONTIGUOUS dimension (channels) takes the M side of the
// instruction (128 rows per CTA, always full tiles of a weight matrix) and the output's rows the N side, which an
// instruction takes in steps of 32: a group of a few rows fills few columns and loads few rows, and a weight matrix that is all the
// traffic streams through full tiles.  The accumulator has a channel per TMEM lane and an output row per column, so that bias and
// channel scale are one register per lane, and rows behind a group's last one are just not stored.
//
// One persistent CTA (or CTA pair, cta_group::2: 256 channels x up to 256 rows, each CTA loads its 128 channels and half
// of the rows) per SM; warp roles as in the dense kernel: 0 TMA producer, 1 MMA issuer, 2..9 epilogue, and for
// variant 2 a warp 10 that clears what the last k-block of a group holds of the next group (see `fixer`).
// Measured (one B200, in a graph): 8 experts, 8192 rows, 4096 -> 4096 forward 0.209 - 0.214 ms (1.28 - 1.31 PFLOP/s; the dense kernel 1.5 on
// one matrix), their weight gradients in float 0.245 - 0.262 ms (1.05 - 1.12 PFLOP/s: with both operands MN-major a k-block takes 0.43 us
// instead of 0.33, in the dense kernel as well); 16 tokens over 64 experts of 1024 -> 4096 41 us (5.2 TB/s); int8 8192^3 0.315 - 0.320 ms
// (3.4 - 3.5 Pop/s).
// The split form cuts K over the CTAs of a cluster and joins the pieces through distributed shared memory, for calls
// with too few tiles to keep the SMs busy.
// Every wait is bounded; on time-out the kernel records a code and leaves.
#include <math.h>

#include <atomic>

#include "../../include/mbd.h"
#include "epi.cuh"
#include "tc_common.cuh"

namespace mbd {
namespace {

using namespace tc;

constexpr int MAX_EXPERTS = 512;              // bounds and tile counts of all groups are held in shared memory
constexpr int RING_BYTES = 160 * 1024;
constexpr int BOX_BYTES = 2048, BOXES = 3;    // epilogue staging: three boxes per warp
constexpr int SMEM_BYTES = RING_BYTES + 8 * BOXES * BOX_BYTES;
constexpr int CH = 128;                       // channels (M side) per CTA
constexpr int A_BYTES = CH * 128;             // one k-block is 128 bytes of every row: 64 bf16 or 128 int8
constexpr int SEG_BLOCKS = 64;                // k-blocks per accumulation segment of a float result, see Params::seg

enum { KIND_BF16 = 0, KIND_I8 = 1 };

// Division of 0 <= n < 2^31 by a number fixed on the host: n * ceil(2^(31 + l) / d) >> (31 + l), 2^(l - 1) < d <= 2^l, which is
// exact.  (A tile's place took six integer divisions, in every warp's chain from one tile to the next.)
struct Divisor {
  uint32_t m = 0;
  int s = 0;
  Divisor() = default;
  explicit Divisor(uint32_t d) {
    int l = 0;
    while ((1ull << l) < d) ++l;
    s = 31 + l;
    m = static_cast<uint32_t>(((1ull << s) + d - 1) / d);
  }
  __device__ __forceinline__ int of(int n) const { return static_cast<int>((static_cast<uint64_t>(static_cast<uint32_t>(n)) * m) >> s); }
};

constexpr int DIRECT_BELOW = 8;               // k-blocks, see `epilogue`
constexpr int GROUP_N = 8;                    // row tiles per raster group

struct Params {
  int E, T;                  // experts; rows of the row tensors (offsets are clamped to [0, T])
  const int32_t* offsets;    // [E + 1] on the device, or null: one group of all T rows
  int M, N;                  // output channels; variant 2: output rows per expert (d_out)
  int kb_total;              // variants 0, 1: k-blocks
  int m_tiles, n_tiles;      // n_tiles: variant 2 only
  int n_step;                // variant 2: rows of a tile
  Divisor per_expert, per_group, by[GROUP_N];       // variant 2: tiles of an expert; tiles of a raster group; 1 .. GROUP_N
  int chunked_a, chunked_b;  // MN-major operands: the map has chunks of 64 columns as a dimension, one box holds all of a tile's
  int seg;                   // k-blocks per segment: the tensor core truncates when it adds to the accumulator (relative error
                             // ~1.1e-9 per element of K, measured), so a float result is summed from segments of 4096 in
                             // full float arithmetic; a bf16 result's rounding hides it
  int op, out_bf16, relu;
  void* out;
  int64_t ldo, out_stride;   // out_stride: variant 2, elements between experts
  const float* bias;         // [E][M] or null
  const void* mask;
  int64_t ldmask;
  float scale;
  const float* row_scale;    // i8: [T]
  const float* ch_scale;     // i8: [E][M]
  int* status;
};

// ------------------------------------------------------------------------------------------------ PTX forms
__device__ __forceinline__ uint32_t cta_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t in_cta(uint32_t saddr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(saddr), "r"(rank));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void arrive_cluster(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// Bounded wait for a barrier that another CTA of the pair arrives on after writing shared memory.
__device__ __noinline__ bool wait_cluster(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* status, int code) {
  const unsigned long long t0 = globaltimer_ns();
  for (;;) {
    for (int i = 0; i < 256; ++i) {
      uint32_t ok;
      asm volatile(
          "{\n\t.reg .pred p;\n\t"
          "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
          "selp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
      if (ok) return true;
    }
    if (*abort_flag) return false;
    if (globaltimer_ns() - t0 > WAIT_LIMIT_NS) {
      *abort_flag = 1;
      atomicCAS(status, 0, code);
      return false;
    }
  }
}
__device__ __forceinline__ void load_3d(uint32_t dst, const CUtensorMap* tm, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void load_3d_pair(uint32_t dst, const CUtensorMap* tm, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void load_4d(uint32_t dst, const CUtensorMap* tm, int y, int c, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(0), "r"(y), "r"(c), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void load_4d_pair(uint32_t dst, const CUtensorMap* tm, int y, int c, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(0), "r"(y), "r"(c), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void store_3d(const CUtensorMap* tm, int x, int y, int z, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];"
               ::"l"(reinterpret_cast<uint64_t>(tm)), "r"(x), "r"(y), "r"(z), "r"(src) : "memory");
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
__device__ __forceinline__ void ld16(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(taddr) : "memory");
}
template <int KIND, int PAIR>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
#define MBD_MMA(GROUP, TYPE)                                                                            \
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"                                        \
               "tcgen05.mma.cta_group::" GROUP ".kind::" TYPE " [%0], %1, %2, %3, p;\n\t}"              \
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory")
  if (KIND == KIND_BF16 && !PAIR) MBD_MMA("1", "f16");
  if (KIND == KIND_BF16 && PAIR) MBD_MMA("2", "f16");
  if (KIND == KIND_I8 && !PAIR) MBD_MMA("1", "i8");
  if (KIND == KIND_I8 && PAIR) MBD_MMA("2", "i8");
#undef MBD_MMA
}
template <int PAIR>
__device__ __forceinline__ void commit(uint32_t bar) {
  if (PAIR)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"(static_cast<uint16_t>(3)) : "memory");
  else
    tc_commit(bar);
}

// ------------------------------------------------------------------------------------------------ work
template <int N> struct Int { static constexpr int value = N; };
struct Yes { static constexpr bool value = true; };
struct No { static constexpr bool value = false; };

struct Unit {
  int e, m0;                 // expert, first channel of the (pair's) tile
  int row0, rows;            // first output row (variant 2: within dW_e) and how many exist
  int nt;                    // columns of the instruction
  int k0, kb, tail;          // variant 2: first row of the group, its k-blocks, rows in the last one
};

// Groups in shared memory: bound[e] .. bound[e+1] are the rows of expert e (the running maximum of the clamped offsets, so
// that groups never overlap whatever the offsets hold), first[e] the row tiles of the experts before e.
struct Groups {
  int bound[MAX_EXPERTS + 1];
  int first[MAX_EXPERTS + 1];
  int step[MAX_EXPERTS];     // rows of a tile of expert e
};

template <int B_MN, int BN>
__device__ __forceinline__ void find_groups(const Params& p, Groups* g, int lane) {
  int top = 0, tiles = 0;
  for (int base = 0; base <= p.E; base += 32) {
    const int i = base + lane;
    int v = 0;
    if (i <= p.E) v = p.offsets ? min(max(p.offsets[i], 0), p.T) : (i == 0 ? 0 : p.T);
    for (int d = 1; d < 32; d <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, v, d);
      if (lane >= d) v = max(v, o);
    }
    v = max(v, top);
    int before = __shfl_up_sync(0xffffffffu, v, 1);
    if (lane == 0) before = base == 0 ? v : top;
    const int own = i <= p.E ? (v - before + BN - 1) / BN : 0;  // tiles of expert i - 1
    int t = own;
    for (int d = 1; d < 32; d <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, t, d);
      if (lane >= d) t += o;
    }
    t += tiles;
    if (i <= p.E) { g->bound[i] = v; g->first[i] = t; }
    // the rows of a group are dealt out evenly over its tiles, in steps of 32
    if (!B_MN && i >= 1 && i <= p.E && own > 0) g->step[i - 1] = ((v - before + own - 1) / own + 31) / 32 * 32;
    top = __shfl_sync(0xffffffffu, v, 31);
    tiles = __shfl_sync(0xffffffffu, t, 31);
  }
}

template <int B_MN, int BN, int PAIR>
__device__ __forceinline__ int total_units(const Params& p, const Groups* g) {
  return B_MN ? p.E * p.m_tiles * p.n_tiles : g->first[p.E] * p.m_tiles;
}

// Unit w of the launch; `e` is the expert of the unit before it (units come in rising order).
template <int B_MN, int BN, int PAIR>
__device__ __forceinline__ Unit unit_at(const Params& p, const Groups* g, int w, int& e) {
  constexpr int STEP = B_MN ? (PAIR ? 128 : 64) : 32;
  Unit u;
  int local, tiles, count, step;
  if (B_MN) {
    tiles = p.n_tiles;
    e = p.per_expert.of(w);
    local = w - e * (p.m_tiles * tiles);
    count = p.N;
    step = p.n_step;
  } else {
    while (w >= g->first[e + 1] * p.m_tiles) ++e;
    local = w - g->first[e] * p.m_tiles;
    tiles = g->first[e + 1] - g->first[e];
    count = g->bound[e + 1] - g->bound[e];
    step = g->step[e];
  }
  // raster groups of GROUP_N row tiles, row tiles first: the operands of neighbouring units are shared in L2
  const int gi = p.per_group.of(local);
  const int size = min(tiles - gi * GROUP_N, GROUP_N);
  const int r = local - gi * (GROUP_N * p.m_tiles);
  const int mt = p.by[size - 1].of(r);
  const int tn = gi * GROUP_N + r - mt * size;
  u.e = e;
  u.m0 = mt * (PAIR ? 2 * CH : CH);
  u.row0 = tn * step;
  u.rows = min(step, count - u.row0);
  u.nt = (u.rows + STEP - 1) / STEP * STEP;
  u.k0 = 0;
  u.kb = p.kb_total;
  u.tail = 64;
  if (B_MN) {
    u.k0 = g->bound[e];
    const int len = g->bound[e + 1] - u.k0;
    u.kb = (len + 63) / 64;
    u.tail = len - (u.kb - 1) * 64;
  } else {
    u.row0 += g->bound[e];
  }
  return u;
}

// ------------------------------------------------------------------------------------------------ epilogue
__device__ __forceinline__ float relu(float x) { return x < 0.f ? 0.f : x; }        // (NaN stays NaN)

// CNT output rows row0 .. of one channel per lane: r holds the accumulators of rows row0 + j.  `again`: the result so far
// (the earlier segments of K) is in `out`; `last`: the tail operation is due.
template <int KIND, int CNT>
__device__ __forceinline__ void finish(const Params& p, const Unit& u, const uint32_t* r, int row0, int rows, int m, int lane,
                                       float bias, float ch_scale, bool again, bool last) {
  float v[CNT];
  const int64_t base = u.row0 + row0;
  if (KIND == KIND_I8) {
#pragma unroll
    for (int j = 0; j < CNT; ++j) {
      const float s = j < rows ? p.row_scale[base + j] : 0.f;
      v[j] = static_cast<float>(static_cast<int>(r[j])) * s * ch_scale;
    }
  } else {
#pragma unroll
    for (int j = 0; j < CNT; ++j) v[j] = __uint_as_float(r[j]);
  }
  if (p.out_bf16) {
    // pairs of channels: the even lane of a pair takes row 2j, the odd lane row 2j + 1
    __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(p.out) + u.e * p.out_stride;
    const __nv_bfloat16* mask = reinterpret_cast<const __nv_bfloat16*>(p.mask);
    const int odd = lane & 1, mp = m & ~1;
    const bool two = mp + 1 < p.M, any = mp < p.M;
    uint32_t x[CNT / 2];
    const bool read = p.op == EPI_SGD || (p.op == EPI_MASK && mask != nullptr);
    if (read) {
      const __nv_bfloat16* src = p.op == EPI_SGD ? out : mask;
      const int64_t ld = p.op == EPI_SGD ? p.ldo : p.ldmask;
#pragma unroll
      for (int j = 0; j < CNT / 2; ++j) {
        const __nv_bfloat16* a = src + (base + 2 * j + odd) * ld + mp;
        x[j] = 0;
        if (2 * j + odd < rows) {
          if (two) x[j] = *reinterpret_cast<const uint32_t*>(a);
          else if (any) x[j] = *reinterpret_cast<const unsigned short*>(a);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < CNT / 2; ++j) {
      float a = v[2 * j] + bias, b = v[2 * j + 1] + bias;
      if (p.relu) { a = relu(a); b = relu(b); }
      const float got = __shfl_xor_sync(0xffffffffu, odd ? a : b, 1);
      float lo = odd ? got : a, hi = odd ? b : got;
      if (read) {
        const float xl = bf16_bits_to_f32(x[j] & 0xFFFFu), xh = bf16_bits_to_f32(x[j] >> 16);
        if (p.op == EPI_SGD) { lo = fmaf(p.scale, lo, xl); hi = fmaf(p.scale, hi, xh); }
        else { if (!(xl > 0.f)) lo = 0.f; if (!(xh > 0.f)) hi = 0.f; }
      }
      if (2 * j + odd < rows) {
        __nv_bfloat16* d = out + (base + 2 * j + odd) * p.ldo + mp;
        if (two) *reinterpret_cast<uint32_t*>(d) = pack_bf16x2(lo, hi);
        else if (any) *d = __float2bfloat16_rn(lo);
      }
    }
    return;
  }
  float* out = reinterpret_cast<float*>(p.out) + u.e * p.out_stride + base * p.ldo + m;
  const bool here = m < p.M;
  const bool masked = p.op == EPI_MASK && p.mask != nullptr;
  if (p.op == EPI_SGD || again || masked) {
    // A mask over several segments is met by the first one, which may find it in the memory that it writes.  What the mask closes
    // is left as -0 for the segments to come: an open sum is never -0, it starts as a sum with +0 (and x + v is -0 for x = v = -0 only).
    constexpr uint32_t CLOSED = 0x80000000u;
    const float closed = last ? 0.f : __uint_as_float(CLOSED);
    const bool meets = masked && !again;
    const float* src = meets ? reinterpret_cast<const float*>(p.mask) + base * p.ldmask + m : out;
    const int64_t ld = meets ? p.ldmask : p.ldo;
    float x[CNT];
#pragma unroll
    for (int j = 0; j < CNT; ++j) x[j] = here && j < rows ? src[j * ld] : 0.f;
#pragma unroll
    for (int j = 0; j < CNT; ++j) {
      if (p.op == EPI_SGD) v[j] = fmaf(p.scale, v[j], x[j]);
      else if (meets) v[j] = x[j] > 0.f ? v[j] + 0.f : closed;
      else v[j] = masked && __float_as_uint(x[j]) == CLOSED ? closed : x[j] + v[j];
    }
  }
  if (!here) return;
#pragma unroll
  for (int j = 0; j < CNT; ++j) {
    if (last) {
      v[j] += bias;
      if (p.relu) v[j] = relu(v[j]);
    }
    if (j < rows) out[j * p.ldo] = v[j];
  }
}

// The accumulators of CNT output rows of a channel, scaled, with bias and ReLU.
template <int KIND, int CNT>
__device__ __forceinline__ void values(const Params& p, const uint32_t* r, float* v, int64_t row, int rows, int lane, float bias, float ch_scale) {
  if (KIND == KIND_I8) {
    const float mine = lane < rows ? p.row_scale[row + lane] : 0.f;
#pragma unroll
    for (int j = 0; j < CNT; ++j) v[j] = static_cast<float>(static_cast<int>(r[j])) * __shfl_sync(0xffffffffu, mine, j) * ch_scale;
  } else {
#pragma unroll
    for (int j = 0; j < CNT; ++j) v[j] = __uint_as_float(r[j]);
  }
  if (p.bias) {
#pragma unroll
    for (int j = 0; j < CNT; ++j) v[j] += bias;
  }
  if (p.relu) {
#pragma unroll
    for (int j = 0; j < CNT; ++j) v[j] = relu(v[j]);
  }
}

// 16 float rows straight from the accumulator's layout: a warp stores 32 channels of a row, with nothing to wait for.  `out`: row
// `row`, channel 0.
template <int KIND>
__device__ __forceinline__ void put_rows(const Params& p, const uint32_t* r, float* out, int64_t row, int left, int m, int lane, float bias, float ch_scale) {
  float v[16];
  values<KIND, 16>(p, r, v, row, left, lane, bias, ch_scale);
  if (m >= p.M) return;
  float* at = out + m;
  if (left >= 16) {
#pragma unroll
    for (int j = 0; j < 16; ++j, at += p.ldo) *at = v[j];
  } else {
#pragma unroll
    for (int j = 0; j < 16; ++j, at += p.ldo)
      if (j < left) *at = v[j];
  }
}

// A box of CNT output rows of this warp's 32 channels (float: 16 rows of 128 bytes, bf16: 32 rows of 64 bytes) in staging memory: turned
// from a channel per lane to rows, so that 16 bytes of a row can leave (and 16 bytes of a mask be met) per lane.  Going to global memory
// straight from the accumulator's layout cost 24 instructions per element of address and predicate (skewed weight gradients 127
// against 85 us).  met: the box holds the old weights of Eq. 1 or a mask and is combined in place.
enum Met { NOTHING, OLD_WEIGHTS, MASK };
template <int KIND, int CNT>
__device__ __forceinline__ void fill_box(const Params& p, uint8_t* box, const uint32_t* r, int64_t row, int rows, int lane, float bias, float ch_scale, Met met) {
  float v[CNT];
  values<KIND, CNT>(p, r, v, row, rows, lane, bias, ch_scale);
  if (CNT == 16) {
    float* at = reinterpret_cast<float*>(box) + lane;
    if (met == OLD_WEIGHTS) {
#pragma unroll
      for (int j = 0; j < CNT; ++j) v[j] = fmaf(p.scale, v[j], at[j * 32]);
    } else if (met == MASK) {
#pragma unroll
      for (int j = 0; j < CNT; ++j) v[j] = at[j * 32] > 0.f ? v[j] : 0.f;
    }
#pragma unroll
    for (int j = 0; j < CNT; ++j) at[j * 32] = v[j];
  } else {
    // pairs of channels: the even lane of a pair takes row 2j, the odd lane row 2j + 1
    const int odd = lane & 1;
    uint32_t* at = reinterpret_cast<uint32_t*>(box) + odd * 16 + (lane >> 1);
    uint32_t w[CNT / 2];
    if (met != NOTHING) {
#pragma unroll
      for (int j = 0; j < CNT / 2; ++j) w[j] = at[j * 32];
    }
#pragma unroll
    for (int j = 0; j < CNT / 2; ++j) {
      const float got = __shfl_xor_sync(0xffffffffu, odd ? v[2 * j] : v[2 * j + 1], 1);
      float lo = odd ? got : v[2 * j], hi = odd ? v[2 * j + 1] : got;
      if (met == OLD_WEIGHTS) {
        const float xl = bf16_bits_to_f32(w[j] & 0xFFFFu), xh = bf16_bits_to_f32(w[j] >> 16);
        lo = fmaf(p.scale, lo, xl);
        hi = fmaf(p.scale, hi, xh);
      }
      uint32_t both = pack_bf16x2(lo, hi);
      if (met == MASK) both &= __hgt2_mask(*reinterpret_cast<const __nv_bfloat162*>(&w[j]), __float2bfloat162_rn(0.f));
      at[j * 32] = both;
    }
  }
}

// The epilogue of one warp: 32 channels (a quarter of the CTA's lanes) of every second box of CNT output rows.
template <int KIND, int B_MN, int BN, int PAIR, int CNT>
__device__ __forceinline__ void epilogue(const Params& p, const Groups* groups, const CUtensorMap* tmOut, uint8_t* boxes, uint64_t* box_bars,
                                         uint64_t* tmem_full, uint64_t* tmem_empty, uint32_t tmem_base, int w_first, int w_step, int total,
                                         int q, int half, int lane, uint32_t rank, volatile int* abortp) {
  constexpr int SIZE = CNT == 32 ? 2 : 4, LANES = 32 * SIZE / 16, ROWS = 32 / LANES;      // lanes per row, rows per access
  const bool sgd = p.op == EPI_SGD, mask = p.op == EPI_MASK && p.mask != nullptr;
  int it = 0, expert = 0;
  uint32_t n = 0, phases = 0;              // boxes so far modulo BOXES; SGD: the parity of each box's barrier
  bool ok = true;
  for (int w = w_first; w < total && ok; w += w_step) {
    const Unit u = unit_at<B_MN, BN, PAIR>(p, groups, w, expert);
    const int m0 = u.m0 + (PAIR ? static_cast<int>(rank) * CH : 0) + q * 32, m = m0 + lane;
    const float bias = p.bias && m < p.M ? p.bias[static_cast<int64_t>(u.e) * p.M + m] : 0.f;
    const float cs = KIND == KIND_I8 && m < p.M ? p.ch_scale[static_cast<int64_t>(u.e) * p.M + m] : 0.f;
    const int count = (u.rows + CNT - 1) / CNT;
    // element by element: a sum over segments (it adds to `out`), and an edge that cuts 16 bytes in two
    const bool staged = u.kb <= p.seg && (m0 + 32 <= p.M || p.M % (16 / SIZE) == 0);
    const int plane = B_MN ? u.e : 0;
    // Float rows of a tile with no main loop to speak of: stores that wait for nothing (skewed weight gradients, a k-block or two a tile:
    // 82 against 97 us; from 16 k-blocks on the bulk stores, which leave the LSU and the issue slots to the others, are as good or better:
    // weight gradients of 8 experts 253 against 263 us)
    const bool direct = CNT == 16 && !sgd && !mask && u.kb < DIRECT_BELOW;
    if (u.kb == 0 && sgd) continue;                          // an expert without rows: nothing to add to its weights
    // this lane's 16 bytes of a box's first rows
    const int ch = m0 + lane % LANES * (16 / SIZE), lr = lane / LANES;
    const bool column = ch < p.M;
    char* const out = reinterpret_cast<char*>(p.out) + (u.e * p.out_stride + (u.row0 + lr) * p.ldo + ch) * SIZE;
    const char* const mask_at = reinterpret_cast<const char*>(p.mask) + ((u.row0 + lr) * p.ldmask + ch) * SIZE;
    // A mask arrives by 16 bytes a lane straight into the boxes, zeros beyond the group, two boxes early.  5003 rows of 16 groups, 4096
    // channels, K = 64 and 1000, side by side on one set of groups: 33 and 53 us (27 and 49 without a mask); by loads into registers a box
    // early 44 and 59 us, a latency under load of 1.8 us per box; two boxes early in twice the registers 52 and 66; by bulk copies it
    // queues behind the operands'.  Over equal and skewed groups of those sizes 35 - 37 and 57 - 60 us (27 - 29 and 52 - 58 without a mask).
    auto fetch = [&](int b, uint32_t at) {
      if (b < count) {
        const uint32_t to = smem_u32(boxes) + at * BOX_BYTES + lane * 16;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = b * CNT + i * ROWS;
          const bool there = column && row + lr < u.rows;
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + i * 512),
                       "l"(there ? mask_at + row * p.ldmask * SIZE : static_cast<const char*>(p.mask)), "r"(there ? 16 : 0) : "memory");
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // the old weights arrive by bulk copies
    auto request = [&](int b, uint32_t at) {                 // lane 0
      const uint32_t bar = smem_u32(&box_bars[at]);
      mbar_expect_tx(bar, BOX_BYTES);
      load_3d(smem_u32(boxes) + at * BOX_BYTES, tmOut, m0, u.row0 + b * CNT, u.e, bar);
    };
    if (sgd && staged && lane == 0) {
      asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");             // the last store is that of the third box
      if (half < count) request(half, n);
      if (half + 2 < count) request(half + 2, n + 1 == BOXES ? 0 : n + 1);
    }
    if (mask && staged) {                                    // (the latency of the first two passes under the tile's products)
      if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
      __syncwarp();
      fetch(half, n);
      fetch(half + 2, n + 1 == BOXES ? 0 : n + 1);
    }
    for (int kb = 0; (kb < u.kb || kb == 0) && ok; kb += p.seg) {
      const bool last = kb + p.seg >= u.kb, some = u.kb > 0; // an expert without rows has a gradient of zeros and no accumulator
      const int acc = it & 1;
      if (some) {
        ok = mbar_wait(smem_u32(&tmem_full[acc]), (it >> 1) & 1u, abortp, p.status, DEV_TIMEOUT_EPILOGUE);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        ++it;
        tc_fence_after();
      }
      const uint32_t taddr = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + acc * BN;
      for (int b = half; b < count; b += 2) {
        uint32_t r[CNT];
        if (some) {
          if (CNT == 32) tc_ld32(taddr + b * CNT, r);
          else ld16(taddr + b * CNT, r);
          tc_wait_ld();
          if (b + 2 >= count) {                              // all of this warp's part is read: hand it back
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_cluster(in_cta(smem_u32(&tmem_empty[acc]), 0));
          }
        } else {
#pragma unroll
          for (int j = 0; j < CNT; ++j) r[j] = 0;
        }
        const int left = u.rows - b * CNT;
        if (CNT == 16 && direct) {
          put_rows<KIND>(p, r, static_cast<float*>(p.out) + u.e * p.out_stride + (u.row0 + b * CNT) * p.ldo, u.row0 + b * CNT, left, m, lane, bias, cs);
          continue;
        }
        if (!staged) {
          finish<KIND, CNT>(p, u, r, b * CNT, left, m, lane, bias, cs, kb > 0, last);
          continue;
        }
        uint8_t* box = boxes + n * BOX_BYTES;
        if (sgd) {                                           // (only for an expert's weights: rows beyond them are cut off by the map)
          ok = mbar_wait(smem_u32(&box_bars[n]), (phases >> n) & 1u, abortp, p.status, DEV_TIMEOUT_EPILOGUE);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          phases ^= 1u << n;
          fill_box<KIND, CNT>(p, box, r, u.row0 + b * CNT, left, lane, bias, cs, OLD_WEIGHTS);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            store_3d(tmOut, m0, u.row0 + b * CNT, u.e, smem_u32(box));
            if (b + 4 < count) {                             // two boxes on: into the box before this one, once its store has read it
              asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
              request(b + 4, n == 0 ? BOXES - 1 : n - 1);
            }
          }
        } else {
          // by one bulk store where the whole box is this group's; at a group's last rows (those behind them are another group's) by
          // 16 bytes a lane.  (All boxes that way: weight gradients 282 against 251 us, the stores share the issue slots of the warps.)
          const bool bulk = B_MN || left >= CNT;
          if (mask) asm volatile("cp.async.wait_group 1;" ::: "memory");                                     // all but the next box's
          else if (lane == 0) asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(BOXES - 1) : "memory"); // the store that used this box has read it
          __syncwarp();
          // (two calls, each of them straight code: one with a run-time choice cost results without a mask 2 us in 28)
          if (mask) fill_box<KIND, CNT>(p, box, r, u.row0 + b * CNT, left, lane, bias, cs, MASK);
          else fill_box<KIND, CNT>(p, box, r, u.row0 + b * CNT, left, lane, bias, cs, NOTHING);
          if (bulk) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) store_3d(tmOut, m0, u.row0 + b * CNT, plane, smem_u32(box));
          } else {
            if (lane == 0) asm volatile("cp.async.bulk.commit_group;" ::: "memory");      // (a group of its own, so that the count above holds)
            __syncwarp();
            uint4 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const uint4*>(box + i * 512 + lane * 16);
            char* at = out + b * CNT * p.ldo * SIZE;
#pragma unroll
            for (int i = 0; i < 4; ++i, at += ROWS * p.ldo * SIZE)
              if (column && lr + i * ROWS < left) *reinterpret_cast<uint4*>(at) = v[i];
          }
          if (mask) {                                        // two boxes on: into the box before this one, once its store has read it
            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
            __syncwarp();
            fetch(b + 4, n == 0 ? BOXES - 1 : n - 1);
          }
        }
        if (++n == BOXES) n = 0;
      }
      if (some && half >= count) {                           // nothing to read for this warp
        __syncwarp();
        if (lane == 0) arrive_cluster(in_cta(smem_u32(&tmem_empty[acc]), 0));
      }
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");                               // copies and stores done before the CTA exits
  if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  __syncwarp();
}

// ------------------------------------------------------------------------------------------------ the kernel
// KIND: bf16 or int8.  A (the M side) and B (the N side) are K-major (0) or MN-major (1, bf16 only).  B_MN is variant 2:
// K is the rows of a group.  BN: most output rows of a tile.  PAIR: two CTAs share a tile of 256 channels.  SPLIT: one unit
// per cluster, its K range cut over the CTAs.
template <int KIND, int A_MN, int B_MN, int BN, int PAIR, int SPLIT>
__global__ void __launch_bounds__(B_MN ? 352 : 320, 1)
expert_gemm_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                   const __grid_constant__ CUtensorMap tmB32, const __grid_constant__ CUtensorMap tmOut,
                   const Params p) {
  constexpr int BNL = PAIR ? BN / 2 : BN;
  constexpr int STAGE_BYTES = A_BYTES + BNL * 128;
  constexpr int STAGES = RING_BYTES / STAGE_BYTES;
  constexpr int ACC_BUFS = SPLIT ? 1 : 2;
  constexpr int TMEM_COLS = ACC_BUFS * BN;
  constexpr int ELEMS = KIND == KIND_I8 ? 128 : 64;          // elements of a k-block
  static_assert(TMEM_COLS >= 32 && TMEM_COLS <= 512 && STAGES <= 16 && (BNL == 64 || BNL == 128 || BNL == 256) &&
                !(SPLIT && BN * CH * 4 > RING_BYTES), "");

  extern __shared__ __align__(1024) uint8_t smem_raw[];
  __shared__ Groups groups;
  __shared__ __align__(8) uint64_t full_bar[STAGES], empty_bar[STAGES];
  __shared__ __align__(8) uint64_t landed_bar[B_MN ? STAGES : 1], fixed_bar[B_MN ? STAGES : 1];
  __shared__ __align__(8) uint64_t tmem_full_bar[2], tmem_empty_bar[2], box_bar[8 * BOXES];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;

  const uint32_t ring = smem_u32(smem_raw);
  if (ring & 1023u) {                     // same answer in every CTA
    if (threadIdx.x == 0) atomicCAS(p.status, 0, DEV_SMEM_MISALIGNED);
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = PAIR || SPLIT ? cta_rank() : 0u;
  const int pieces = SPLIT ? static_cast<int>(cluster_size()) : 1;
  const int w_first = PAIR ? blockIdx.x >> 1 : SPLIT ? blockIdx.x / pieces : blockIdx.x;
  const int w_step = PAIR ? gridDim.x >> 1 : SPLIT ? 1 << 30 : gridDim.x;

  if (threadIdx.x == 0) {
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(smem_u32(&full_bar[i]), 1);
      mbar_init(smem_u32(&empty_bar[i]), 1);
      if (B_MN) {
        mbar_init(smem_u32(&landed_bar[i]), 1);
        mbar_init(smem_u32(&fixed_bar[i]), PAIR ? 2 : 1);
      }
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&tmem_full_bar[i]), 1);
      mbar_init(smem_u32(&tmem_empty_bar[i]), PAIR ? 16 : 8);
    }
    for (int i = 0; i < 8 * BOXES; ++i) mbar_init(smem_u32(&box_bar[i]), 1);
    abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    if (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(TMEM_COLS) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      tmem_alloc<TMEM_COLS>(smem_u32(&tmem_slot));
    }
  }
  if (warp == 2 && lane < 3) {             // the maps are the launch's own: they may be fetched before the kernel before this one is done
    const CUtensorMap* tm = lane == 0 ? &tmA : lane == 1 ? &tmB : &tmB32;
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(tm)) : "memory");
  }
  pdl_trigger();
  pdl_wait();                              // the offsets may come from the kernel before this one
  if (warp == 0) find_groups<B_MN, BN>(p, &groups, lane);
  tc_fence_before();
  __syncthreads();
  if (PAIR) cluster_sync();                // the other CTA's barriers exist before anything remote touches them (SPLIT meets below)
  tc_fence_after();
  const uint32_t tmem_base = tmem_slot;
  const int total = total_units<B_MN, BN, PAIR>(p, &groups);
  volatile int* abortp = &abort_flag;
  int expert = 0;

  // k-blocks of this CTA's share of a unit
  auto first_kb = [&](const Unit& u) { return SPLIT ? static_cast<int>(static_cast<long long>(rank) * u.kb / pieces) : 0; };
  auto last_kb = [&](const Unit& u) { return SPLIT ? static_cast<int>(static_cast<long long>(rank + 1) * u.kb / pieces) : u.kb; };
  // the last k-block of a group of rows holds rows of the next group, and an instruction takes 16
  auto ragged = [&](const Unit& u, int kb) { return B_MN && kb == u.kb - 1 && (u.tail & 15) != 0; };
  // That k-block is consumed last, but takes its place in the ring (and is asked for) up to TAIL_AHEAD blocks earlier, so that
  // clearing it is over by then: consumed where it stands it cost 1.3 us per unit.  kb1 if there is none.
  constexpr int TAIL_AHEAD = STAGES - 2;
  auto tail_place = [&](const Unit& u, int kb0, int kb1) { return kb1 > kb0 && ragged(u, kb1 - 1) ? max(kb0, kb1 - 1 - TAIL_AHEAD) : kb1; };

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int w = w_first; w < total && ok; w += w_step) {
        const Unit u = unit_at<B_MN, BN, PAIR>(p, &groups, w, expert);
        const int m = u.m0 + (PAIR ? static_cast<int>(rank) * CH : 0);
        const int half = PAIR ? u.nt / 2 : u.nt;                      // output rows this CTA loads
        const int n = u.row0 + (PAIR ? static_cast<int>(rank) * half : 0);
        const int kb0 = first_kb(u), kb1 = last_kb(u);
        const int ez = B_MN ? 0 : u.e;
        // One k-block's copies, as straight code: the issuing thread paces a tile of short boxes (with a loop over the boxes and a
        // choice of barrier at each, the weight gradients ran at 0.97 instead of 1.1 PFLOP/s).
        auto k_block = [&](int kb, auto clear_later, auto boxes_c, auto chunked_c) {
          constexpr bool LATER = decltype(clear_later)::value;          // both operands' last rows will be cleared, see `fixer`
          constexpr bool ONE_A = decltype(chunked_c)::value & 1, ONE_B = decltype(chunked_c)::value & 2;
          constexpr int NB = decltype(boxes_c)::value;                  // boxes of the N side; K-major: 0 one box of BNL rows, else of 32
          constexpr uint32_t BYTES = A_BYTES + (B_MN ? NB * 8192u : NB == 0 ? BNL * 128u : NB * 4096u);
          const uint32_t sa = ring + stage * STAGE_BYTES, sb = sa + A_BYTES;
          uint32_t bar = smem_u32(&full_bar[stage]);
          if (LATER) {                     // each CTA of a pair waits for its own bytes; nobody waits for the stage's own barrier then
            if (!PAIR || rank == 0) mbar_arrive(bar);
            bar = smem_u32(&landed_bar[stage]);
            mbar_expect_tx(bar, BYTES);
          } else if (!PAIR) {
            mbar_expect_tx(bar, BYTES);
          } else {
            if (rank == 0) mbar_expect_tx(bar, 2 * BYTES);
            bar = in_cta(bar, 0);
          }
          auto load = [&](uint32_t dst, const CUtensorMap* tm, int x, int y, int z) {
            if (PAIR && !LATER) load_3d_pair(dst, tm, x, y, z, bar);
            else load_3d(dst, tm, x, y, z, bar);
          };
          const int k = B_MN ? u.k0 + kb * 64 : kb * ELEMS;
          auto load_chunks = [&](uint32_t dst, const CUtensorMap* tm, int column, int row, int z) {
            if (PAIR && !LATER) load_4d_pair(dst, tm, row, column >> 6, z, bar);
            else load_4d(dst, tm, row, column >> 6, z, bar);
          };
          if (A_MN == 0) {
            load(sa, &tmA, k, m, ez);
          } else if (ONE_A) {
            load_chunks(sa, &tmA, m, k, ez);
          } else {
#pragma unroll
            for (int c = 0; c < CH / 64; ++c) load(sa + c * 8192, &tmA, m + c * 64, k, ez);
          }
          if (B_MN && ONE_B) {
            load_chunks(sb, &tmB, n, k, 0);
          } else if (B_MN) {
#pragma unroll
            for (int c = 0; c < NB; ++c) load(sb + c * 8192, &tmB, n + c * 64, k, 0);
          } else if (NB == 0) {
            load(sb, &tmB, k, n, 0);
          } else {
#pragma unroll
            for (int c = 0; c < NB; ++c) load(sb + c * 4096, &tmB32, k, n + c * 32, 0);
          }
          if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        };
        auto k_blocks = [&](auto boxes_c, auto chunked_c) {
          const int tail_at = tail_place(u, kb0, kb1);
          for (int i = kb0; i < kb1; ++i) {
            ok = mbar_wait(smem_u32(&empty_bar[stage]), phase ^ 1u, abortp, p.status, DEV_TIMEOUT_PRODUCER);
            if (!ok) break;
            if (!B_MN || i < tail_at) k_block(i, No{}, boxes_c, chunked_c);
            else if (i == tail_at) k_block(kb1 - 1, Yes{}, boxes_c, chunked_c);
            else k_block(i - 1, No{}, boxes_c, chunked_c);
          }
        };
        auto by_rows = [&](auto chunked_c) {
          if (half > (BNL == 256 ? 128 : BNL - 32)) k_blocks(Int<0>{}, chunked_c);
          else if (BNL <= 64 || half <= 32) k_blocks(Int<1>{}, chunked_c);
          else if (half <= 64) k_blocks(Int<2>{}, chunked_c);
          else if (BNL <= 128 || half <= 96) k_blocks(Int<3>{}, chunked_c);
          else k_blocks(Int<4>{}, chunked_c);
        };
        if (B_MN) {
          if (p.chunked_a && p.chunked_b) k_blocks(Int<BNL / 64>{}, Int<3>{});
          else k_blocks(Int<BNL / 64>{}, Int<0>{});
        } else if (A_MN && p.chunked_a) {
          by_rows(Int<1>{});
        } else {
          by_rows(Int<0>{});
        }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer
    if (lane == 0 && (!PAIR || rank == 0)) {
      int stage = 0, it = 0;
      uint32_t phase = 0, fixed_phase = 0;                 // fixed_phase: one bit per stage
      bool ok = true;
      for (int w = w_first; w < total && ok; w += w_step) {
        const Unit u = unit_at<B_MN, BN, PAIR>(p, &groups, w, expert);
        const uint32_t idesc = (KIND == KIND_I8 ? (2u << 4) | (1u << 7) | (1u << 10)
                                                : (1u << 4) | (1u << 7) | (1u << 10) | (uint32_t(A_MN) << 15) | (uint32_t(B_MN) << 16)) |
                               (static_cast<uint32_t>(u.nt >> 3) << 17) | (uint32_t((PAIR ? 2 * CH : CH) >> 4) << 24);
        const int kb1 = last_kb(u);
        int kb = first_kb(u), tail_stage = 0;
        const int tail_at = tail_place(u, kb, kb1);
        while (kb < kb1 && ok) {                           // a segment
          const int seg_end = min(kb1, kb + p.seg);
          const int acc = it % ACC_BUFS;
          ok = mbar_wait(smem_u32(&tmem_empty_bar[acc]), ((it / ACC_BUFS) & 1u) ^ 1u, abortp, p.status, DEV_TIMEOUT_MMA_TMEM);
          if (!ok) break;
          ++it;
          tc_fence_after();
          const uint32_t d = tmem_base + acc * BN;
          bool add = false;
          for (; kb < seg_end; ++kb) {
            const bool rag = B_MN && tail_at < kb1 && kb == kb1 - 1;
            if (B_MN && kb == tail_at) {                   // the ring's next place holds the ragged block: step over it
              tail_stage = stage;
              if (++stage == STAGES) { stage = 0; phase ^= 1u; }
            }
            const int at = rag ? tail_stage : stage;
            if (rag) {
              ok = wait_cluster(smem_u32(&fixed_bar[at]), (fixed_phase >> at) & 1u, abortp, p.status, DEV_TIMEOUT_MMA_FULL);
              fixed_phase ^= 1u << at;
            } else {
              ok = mbar_wait(smem_u32(&full_bar[stage]), phase, abortp, p.status, DEV_TIMEOUT_MMA_FULL);
            }
            if (!ok) break;
            tc_fence_after();
            const uint32_t sa = ring + at * STAGE_BYTES, sb = sa + A_BYTES;
            const uint64_t ad = A_MN ? make_desc(sa, 8192, 1024) : make_desc(sa, 16, 1024);
            const uint64_t bd = B_MN ? make_desc(sb, 8192, 1024) : make_desc(sb, 16, 1024);
            constexpr uint64_t A_STEP = (A_MN ? 2048 : 32) >> 4, B_STEP = (B_MN ? 2048 : 32) >> 4;
            const int steps = B_MN && kb == u.kb - 1 ? (u.tail + 15) >> 4 : 4;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              if (!B_MN || k < steps) {
                mma<KIND, PAIR>(d, ad + k * A_STEP, bd + k * B_STEP, idesc, add ? 1u : 0u);
                add = true;
              }
            }
            commit<PAIR>(smem_u32(&empty_bar[at]));
            if (!rag && ++stage == STAGES) { stage = 0; phase ^= 1u; }
          }
          if (ok) commit<PAIR>(smem_u32(&tmem_full_bar[acc]));
        }
      }
    }
  } else if (warp < 10) {
    // ------------------------------------------------------------------ epilogue
    const int q = warp & 3, half = (warp - 2) >> 2;
    if (SPLIT) {
      if (w_first < total) {
        const Unit u = unit_at<B_MN, BN, PAIR>(p, &groups, w_first, expert);
        if (first_kb(u) < last_kb(u)) (void)mbar_wait(smem_u32(&tmem_full_bar[0]), 0, abortp, p.status, DEV_TIMEOUT_EPILOGUE);
        __syncwarp();
      }
    } else {
      uint8_t* boxes = smem_raw + RING_BYTES + (warp - 2) * BOXES * BOX_BYTES;
      uint64_t* bars = box_bar + (warp - 2) * BOXES;
      if (p.out_bf16) epilogue<KIND, B_MN, BN, PAIR, 32>(p, &groups, &tmOut, boxes, bars, tmem_full_bar, tmem_empty_bar, tmem_base, w_first, w_step, total, q, half, lane, rank, abortp);
      else epilogue<KIND, B_MN, BN, PAIR, 16>(p, &groups, &tmOut, boxes, bars, tmem_full_bar, tmem_empty_bar, tmem_base, w_first, w_step, total, q, half, lane, rank, abortp);
    }
  } else if (B_MN) {
    // ------------------------------------------------------------------ fixer
    // A group's last k-block ends with rows of the next group (or behind the last group).  They are no zeros, and may be
    // infinities or NaN, so multiplying them by zeros would not do: both operands' rows up to the next multiple of 16 are
    // cleared in shared memory before the instruction reads them.  A row of a swizzled chunk is 128 bytes whatever the swizzle.
    int stage = 0;
    uint32_t landed_phase = 0;             // one bit per stage
    bool ok = true;
    for (int w = w_first; w < total && ok; w += w_step) {
      const Unit u = unit_at<B_MN, BN, PAIR>(p, &groups, w, expert);
      const int kb0 = first_kb(u), kb1 = last_kb(u), tail_at = tail_place(u, kb0, kb1);
      const int at = (stage + tail_at - kb0) % STAGES;
      stage = (stage + kb1 - kb0) % STAGES;
      if (tail_at == kb1) continue;
      ok = mbar_wait(smem_u32(&landed_bar[at]), (landed_phase >> at) & 1u, abortp, p.status, DEV_TIMEOUT_PRODUCER);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      landed_phase ^= 1u << at;
      const int rows = ((u.tail + 15) & ~15) - u.tail;
      uint8_t* base = smem_raw + at * STAGE_BYTES + u.tail * 128;
      for (int c = 0; c < CH / 64 + BNL / 64; ++c)
        for (int v = lane; v < rows * 8; v += 32) *reinterpret_cast<uint4*>(base + c * 8192 + v * 16) = make_uint4(0, 0, 0, 0);
      asm volatile("fence.proxy.async;" ::: "memory");
      __syncwarp();
      if (lane == 0) arrive_cluster(in_cta(smem_u32(&fixed_bar[at]), PAIR ? 0 : rank));
    }
  }

  if (SPLIT) {
    // The pieces of K meet in the cluster's shared memory: the CTA with rank g % pieces adds the pieces of output rows
    // 8 g .. 8 g + 7 in ascending order and finishes them.  The ring is idle in every CTA once its accumulator is complete.
    __syncwarp();
    cluster_sync();
    const bool work = w_first < total;
    Unit u{};
    if (work && warp >= 2 && warp < 10) {
      expert = 0;
      u = unit_at<B_MN, BN, PAIR>(p, &groups, w_first, expert);
    }
    const int q = warp & 3, half = (warp - 2) >> 2;
    const int eights = work ? (u.rows + 7) / 8 : 0;
    const int own_max = (BN / 8 + pieces - 1) / pieces;
    if (work && warp >= 2 && warp < 10) {
      const bool some = first_kb(u) < last_kb(u);
      tc_fence_after();
      for (int g = half; g < eights; g += 2) {
        uint32_t r[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (some) {
          tc_ld8(tmem_base + (static_cast<uint32_t>(q * 32) << 16) + g * 8, r);
          tc_wait_ld();
        }
        const uint32_t at = in_cta(ring + (((rank * own_max + g / pieces) * 8) * CH + q * 32 + lane) * 4, g % pieces);
#pragma unroll
        for (int j = 0; j < 8; ++j) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at + j * CH * 4), "r"(r[j]) : "memory");
      }
    }
    __syncwarp();
    cluster_sync();
    if (work && warp >= 2 && warp < 10) {
      const int m = u.m0 + q * 32 + lane;
      const float bias = p.bias && m < p.M ? p.bias[static_cast<int64_t>(u.e) * p.M + m] : 0.f;
      const float cs = KIND == KIND_I8 && m < p.M ? p.ch_scale[static_cast<int64_t>(u.e) * p.M + m] : 0.f;
      for (int o = half; o * pieces + static_cast<int>(rank) < eights; o += 2) {
        const int g = o * pieces + rank;
        uint32_t r[8];
        for (int s = 0; s < pieces; ++s) {
          const uint32_t* src = reinterpret_cast<const uint32_t*>(smem_raw) + ((s * own_max + o) * 8) * CH + q * 32 + lane;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const uint32_t x = src[j * CH];
            if (s == 0) r[j] = x;
            else if (KIND == KIND_I8) r[j] += x;
            else r[j] = __float_as_uint(__uint_as_float(r[j]) + __uint_as_float(x));
          }
        }
        finish<KIND, 8>(p, u, r, g * 8, u.rows - g * 8, m, lane, bias, cs, false, true);
      }
    }
  }

  if (abort_flag && threadIdx.x == 0) {    // a wait ran out: let the copies in flight land before shared memory is given back
    const unsigned long long t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 1000000ull) {}
  }
  tc_fence_before();
  __syncthreads();
  if (PAIR) cluster_sync();                // the other CTA may still signal barriers in this one's shared memory
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS) : "memory");
    else tmem_dealloc<TMEM_COLS>(tmem_base);
  }
}

// ------------------------------------------------------------------------------------------------ host side
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
  static const EncodeTiledFn fn = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) f = nullptr;
    return reinterpret_cast<EncodeTiledFn>(f);
  }();
  return fn;
}

// [depth][rows][inner] with row stride `ld` and plane stride `plane` in elements of `esize` bytes; 128 bytes per box row.
bool make_map(CUtensorMap* tm, const void* base, int esize, uint64_t inner, uint64_t rows, uint64_t depth, uint64_t ld, uint64_t plane,
              uint32_t box_rows, uint32_t box_bytes = 128, bool swizzle = true) {
  const cuuint64_t dims[3] = {inner, rows, depth};
  const cuuint64_t strides[2] = {ld * esize, (depth > 1 ? plane : ld) * esize};         // (one plane: its stride means nothing, but has a limit)
  const cuuint32_t box[3] = {box_bytes / esize, box_rows, 1};
  const cuuint32_t estr[3] = {1, 1, 1};
  return encode_fn()(tm, esize == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : esize == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, const_cast<void*>(base), dims,
                     strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE,
                     CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The same with its columns as [chunks of 64][64]: a box holds `chunks` of them, box_rows rows each.  The width is a multiple of 64.
bool make_chunk_map(CUtensorMap* tm, const void* base, uint64_t inner, uint64_t rows, uint64_t depth, uint64_t ld, uint64_t plane,
                    uint32_t box_rows, uint32_t chunks) {
  const cuuint64_t dims[4] = {64, rows, inner / 64, depth};
  const cuuint64_t strides[3] = {ld * 2, 128, (depth > 1 ? plane : ld) * 2};
  const cuuint32_t box[4] = {64, box_rows, chunks, 1};
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  return encode_fn()(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                     CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr int MAX_DEVICES = 64;

struct Launch {
  int BN, pair, split;       // split: CTAs that share a unit's K range; 0: the persistent forms
  int grid;
};

template <int KIND, int A_MN, int B_MN>
cudaError_t set_attributes() {
  constexpr cudaFuncAttribute SIZE = cudaFuncAttributeMaxDynamicSharedMemorySize;
  cudaError_t e;
  if ((e = cudaFuncSetAttribute(expert_gemm_kernel<KIND, A_MN, B_MN, 256, 1, 0>, SIZE, SMEM_BYTES)) != cudaSuccess) return e;
  if ((e = cudaFuncSetAttribute(expert_gemm_kernel<KIND, A_MN, B_MN, 64, 0, 0>, SIZE, SMEM_BYTES)) != cudaSuccess) return e;
  if ((e = cudaFuncSetAttribute(expert_gemm_kernel<KIND, A_MN, B_MN, 64, 0, 1>, SIZE, SMEM_BYTES)) != cudaSuccess) return e;
  if ((e = cudaFuncSetAttribute(expert_gemm_kernel<KIND, A_MN, B_MN, 128, 0, 1>, SIZE, SMEM_BYTES)) != cudaSuccess) return e;
  return cudaFuncSetAttribute(expert_gemm_kernel<KIND, A_MN, B_MN, 256, 0, 1>, SIZE, SMEM_BYTES);
}

// What a device needs before its first launch, and how many SMs it has.  (The opt-in to large shared memory is per device; two threads
// that come here at once set the same values.)
mbd_status ready(int dev, int* sms) {
  static std::atomic<int> known[MAX_DEVICES];
  if (dev < 0 || dev >= MAX_DEVICES) return MBD_E_UNSUPPORTED;
  if ((*sms = known[dev].load(std::memory_order_acquire)) > 0) return MBD_OK;
  int major = 0;
  if (cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess) return MBD_E_CUDA;
  if (major != 10) return MBD_E_UNSUPPORTED;
  if (!encode_fn() || set_attributes<KIND_BF16, 0, 0>() != cudaSuccess || set_attributes<KIND_BF16, 1, 0>() != cudaSuccess ||
      set_attributes<KIND_BF16, 1, 1>() != cudaSuccess || set_attributes<KIND_I8, 0, 0>() != cudaSuccess) return MBD_E_CUDA;
  known[dev].store(*sms, std::memory_order_release);
  return MBD_OK;
}

template <int KIND, int A_MN, int B_MN>
cudaError_t launch(const Launch& l, const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& b32,
                   const CUtensorMap& out, const Params& p, cudaStream_t stream) {
  const dim3 grid(l.grid), block(B_MN ? 352 : 320);
  if (l.pair) return launch_pdl(expert_gemm_kernel<KIND, A_MN, B_MN, 256, 1, 0>, grid, block, SMEM_BYTES, stream, 2, a, b, b32, out, p);
  if (!l.split) return launch_pdl(expert_gemm_kernel<KIND, A_MN, B_MN, 64, 0, 0>, grid, block, SMEM_BYTES, stream, 1, a, b, b32, out, p);
  if (l.BN == 64) return launch_pdl(expert_gemm_kernel<KIND, A_MN, B_MN, 64, 0, 1>, grid, block, SMEM_BYTES, stream, l.split, a, b, b32, out, p);
  if (l.BN == 128) return launch_pdl(expert_gemm_kernel<KIND, A_MN, B_MN, 128, 0, 1>, grid, block, SMEM_BYTES, stream, l.split, a, b, b32, out, p);
  return launch_pdl(expert_gemm_kernel<KIND, A_MN, B_MN, 256, 0, 1>, grid, block, SMEM_BYTES, stream, l.split, a, b, b32, out, p);
}

// Most units a call can have: a group of c rows is cut into ceil(c / BN) row tiles.
int64_t most_units(int variant, int E, int64_t T, int64_t M, int64_t N, int BN, int ch) {
  const int64_t mt = (M + ch - 1) / ch;
  if (variant == 2) return E * mt * ((N + BN - 1) / BN);
  const int64_t groups = E < T ? E : T;
  return mt * (E == 1 ? (T + BN - 1) / BN : T / BN + groups);
}

// The form of a call, by a model in SM clocks: waves of tiles over the SMs (or pairs of them), a tile's k-blocks, what a tile costs
// beside them and, for the split forms, joining the pieces.  A k-block of these kernels takes at least 400 clocks however few its rows
// (540 for a pair: halving a pair's rows took 8 % off a tile's time; the ring has as many stages then as for the widest tile), or filling
// shared memory at about 70 bytes a clock.  The group sizes are not known here: the T rows of the row tensors, padding included, spread evenly
// over the experts they can touch, a tile and a half each beyond one.
// Measured with 16 rows of K = 9216 int8 on 4096 channels: 28 us by the pair form, 12.9 us split in 4; 8192 rows: 0.31 ms by the pair
// form, and 128-row tiles twice that.
Launch plan(int kind, int variant, int E, int64_t T, int64_t M, int64_t N, int64_t K, bool out_f32, int sms) {
  const int64_t per_kb = kind == KIND_I8 ? 128 : 64;
  const double groups = variant == 2 ? E : static_cast<double>(E < T ? E : T);
  const double rows = variant == 2 ? static_cast<double>(N) : static_cast<double>(T) / groups;      // output rows of a group
  const double k = variant == 2 ? static_cast<double>(T) / E : static_cast<double>(K);
  const double kbs = k / per_kb > 1.0 ? k / per_kb : 1.0;
  const double longest = static_cast<double>(variant == 2 ? T : K);                                // of a sum
  Launch best{256, 1, 0, 0};
  double least = 1e30;
  const auto consider = [&](int BN, int pair, int split) {
    const double tiles = rows <= BN ? groups : variant == 2 ? groups * ((N + BN - 1) / BN) : groups * (rows / BN + (E > 1 ? 0.5 : 0.0));
    const double units = ceil(tiles) * static_cast<double>((M + (pair ? 2 : 1) * CH - 1) / ((pair ? 2 : 1) * CH));
    const double nt = rows < BN ? rows : BN;
    const double mma = pair ? 540.0 : 4.0 * (nt / 2 > 100.0 ? nt / 2 : 100.0), fill = (CH + (pair ? nt / 2 : nt)) * 128.0 / 70.0;
    const int pieces = split > 1 ? split : 1;
    const double waves = ceil(units * pieces / (pair ? sms / 2 : sms));
    const double t = waves * (kbs / pieces * (mma > fill ? mma : fill) + 3000.0) + (pieces > 1 ? 4000.0 : 0.0);
    if (t < least) { least = t; best = Launch{BN, pair, split, 0}; }
  };
  consider(256, 1, 0);
  consider(64, 0, 0);
  for (int BN = 64; BN <= 256; BN *= 2)
    for (int s = 2; s <= 8; s *= 2) {
      if (kbs / s < 4.0) continue;
      if (out_f32 && kind == KIND_BF16 && longest / s > 64.0 * SEG_BLOCKS) continue;               // (a piece is one segment)
      if (most_units(variant, E, T, M, N, BN, CH) * s > (1 << 30)) continue;
      consider(BN, 0, s);
    }
  const int64_t units = most_units(variant, E, T, M, N, best.BN, best.pair ? 2 * CH : CH);
  if (best.split) best.grid = static_cast<int>(units * best.split);
  else if (best.pair) best.grid = static_cast<int>(2 * (units < sms / 2 ? units : sms / 2));
  else best.grid = static_cast<int>(units < sms ? units : sms);
  return best;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// A mask is the result's own memory, element on element, or shares none with it: anything else would be met half written.
bool mask_apart(const mbd_tail& t, int64_t T, int64_t M) {
  const int64_t size = t.out_bf16 ? 2 : 4, ldo = T > 1 ? t.ldo : M, ldmask = T > 1 ? t.ldmask : M;
  const intptr_t out = reinterpret_cast<intptr_t>(t.out_dev), mask = reinterpret_cast<intptr_t>(t.mask_dev);
  const __int128 between = (static_cast<__int128>(mask) - out) / size;
  if (between >= static_cast<__int128>(T - 1) * ldo + M || -between >= static_cast<__int128>(T - 1) * ldmask + M) return true;
  if (ldo != ldmask) return false;
  if (between == 0) return true;
  const int64_t column = static_cast<int64_t>((between % ldo + ldo) % ldo);       // of the mask in the result's rows
  return column >= M && column + M <= ldo;
}

struct Call {
  int kind, variant, E;
  const int32_t* offsets;
  int64_t T, d_out, d_in;
  const void* A; int64_t lda;           // rows: X or dY
  const void* B; int64_t ldb;           // W, or (variant 2) X
  int64_t stride;                       // elements between experts of W, or of dW
  const float* row_scale; const float* ch_scale;
  const mbd_tail* tail;
  int32_t* status;
  void* stream;
};

mbd_status run(Call c) {
  const mbd_tail* t = c.tail;
  mbd_tail tail;
  if (t && c.T == 0) {                                          // no rows: the row tensors may be null, and are not read
    tail = *t;
    t = &tail;
    if (c.variant != 2 && !tail.out_dev) tail.out_dev = const_cast<void*>(c.B);
    if (!c.A) c.A = t->out_dev;
    if (!c.B && c.variant == 2) c.B = t->out_dev;
  }
  if (!c.A || !c.B || !t || !t->out_dev || c.variant < 0 || c.variant > 2 || c.E < 1 || c.T < 0 || c.d_out < 1 || c.d_in < 1) return MBD_E_INVALID;
  if (t->op != MBD_TAIL_STORE && t->op != MBD_TAIL_MASK && t->op != MBD_TAIL_SGD) return MBD_E_INVALID;
  if (!c.offsets && c.E != 1) return MBD_E_INVALID;
  if (c.kind == KIND_I8 && ((!c.row_scale && c.T > 0) || !c.ch_scale)) return MBD_E_INVALID;
  const int unit = c.kind == KIND_I8 ? 16 : 8;                  // elements of 16 bytes
  const int64_t cols_a = c.variant == 0 ? c.d_in : c.d_out, cols_b = c.d_in;
  const int64_t M = c.variant == 0 ? c.d_out : c.d_in;          // channels of the result
  const int64_t N = c.variant == 2 ? c.d_out : 0;
  if (c.lda < cols_a || c.ldb < cols_b || t->ldo < M || (t->mask_dev && t->ldmask < M)) return MBD_E_INVALID;
  const int64_t plane_rows = c.d_out;
  if (c.E > 1 && c.stride < (plane_rows - 1) * (c.variant == 2 ? t->ldo : c.ldb) + c.d_in) return MBD_E_INVALID;   // experts would overlap
  if (c.E > MAX_EXPERTS || c.T > INT32_MAX - 1024 || c.d_out > INT32_MAX - 1024 || c.d_in > INT32_MAX - 1024) return MBD_E_UNSUPPORTED;
  if (c.kind == KIND_I8 && c.d_in > 131071) return MBD_E_UNSUPPORTED;        // 128 * 128 * d_in stays below 2^31
  if (c.lda % unit || c.ldb % unit || t->ldo % 8 || (t->mask_dev && t->ldmask % 8) || (c.E > 1 && c.stride % unit)) return MBD_E_UNSUPPORTED;
  if (!aligned16(c.A) || !aligned16(c.B) || !aligned16(t->out_dev) || !aligned16(t->mask_dev)) return MBD_E_UNSUPPORTED;
  if ((reinterpret_cast<uintptr_t>(t->bias_dev) | reinterpret_cast<uintptr_t>(c.offsets) | reinterpret_cast<uintptr_t>(c.row_scale) |
       reinterpret_cast<uintptr_t>(c.ch_scale)) & 3u) return MBD_E_UNSUPPORTED;
  if (t->op == MBD_TAIL_MASK && t->mask_dev && c.T > 0 && !mask_apart(*t, c.T, M)) return MBD_E_INVALID;
  // each tail operation belongs to one product: bias and ReLU to the forward one, the mask to backward-data, Eq. 1 to
  // backward-weight
  if ((t->bias_dev || t->relu) && c.variant != 0) return MBD_E_UNSUPPORTED;
  if (t->op == MBD_TAIL_MASK && c.variant != 1) return MBD_E_UNSUPPORTED;
  if (t->op == MBD_TAIL_SGD && c.variant != 2) return MBD_E_UNSUPPORTED;
  const int64_t groups = c.E < c.T ? c.E : c.T;
  const int64_t mt = (M + CH - 1) / CH;
  if (c.variant == 2 ? static_cast<double>(c.E) * mt * ((N + 63) / 64) > 1e9 : static_cast<double>(mt) * (c.T / 64 + groups + 1) > 1e9) return MBD_E_UNSUPPORTED;
  if (c.T == 0 && c.variant != 2) return MBD_OK;                // no rows, nothing to write

  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { (void)cudaGetLastError(); return MBD_E_CUDA; }
  {
    const mbd_status st = ready(dev, &sms);
    if (st != MBD_OK) { (void)cudaGetLastError(); return st; }
  }
  cudaStream_t stream = static_cast<cudaStream_t>(c.stream);

  const Launch l = plan(c.kind, c.variant, c.E, c.T, M, N, c.variant == 1 ? c.d_out : c.d_in, !t->out_bf16, sms);
  const int bnl = l.pair ? l.BN / 2 : l.BN;
  const int esize = c.kind == KIND_I8 ? 1 : 2;
  const uint64_t plane = c.E > 1 ? static_cast<uint64_t>(c.stride) : static_cast<uint64_t>(c.d_out) * c.ldb;
  const uint64_t rows = c.T > 0 ? c.T : 1;                      // (a map of no rows cannot be described; nothing is loaded then)
  CUtensorMap a, b, b32;
  bool ok;
  int chunked_a = 0, chunked_b = 0;
  if (c.variant == 0) {
    ok = make_map(&a, c.B, esize, c.d_in, c.d_out, c.E, c.ldb, plane, CH) &&
         make_map(&b, c.A, esize, c.d_in, rows, 1, c.lda, rows * c.lda, bnl) && make_map(&b32, c.A, esize, c.d_in, rows, 1, c.lda, rows * c.lda, 32);
  } else if (c.variant == 1) {
    chunked_a = c.d_in % 64 == 0;
    ok = (chunked_a ? make_chunk_map(&a, c.B, c.d_in, c.d_out, c.E, c.ldb, plane, 64, CH / 64) : make_map(&a, c.B, esize, c.d_in, c.d_out, c.E, c.ldb, plane, 64)) &&
         make_map(&b, c.A, esize, c.d_out, rows, 1, c.lda, rows * c.lda, bnl) && make_map(&b32, c.A, esize, c.d_out, rows, 1, c.lda, rows * c.lda, 32);
  } else {
    chunked_a = chunked_b = c.d_in % 64 == 0 && c.d_out % 64 == 0;
    ok = chunked_a ? make_chunk_map(&a, c.B, c.d_in, rows, 1, c.ldb, rows * c.ldb, 64, CH / 64) && make_chunk_map(&b, c.A, c.d_out, rows, 1, c.lda, rows * c.lda, 64, bnl / 64)
                   : make_map(&a, c.B, esize, c.d_in, rows, 1, c.ldb, rows * c.ldb, 64) && make_map(&b, c.A, esize, c.d_out, rows, 1, c.lda, rows * c.lda, 64);
    b32 = b;
  }
  // results (and old weights) in boxes of 32 channels, see `epilogue`
  const int osize = t->out_bf16 ? 2 : 4;
  const uint64_t orows = c.variant == 2 ? c.d_out : rows;
  CUtensorMap out;
  ok = ok && make_map(&out, t->out_dev, osize, M, orows, c.variant == 2 ? c.E : 1, t->ldo, c.variant == 2 && c.E > 1 ? c.stride : orows * t->ldo,
                      t->out_bf16 ? 32 : 16, 32 * osize, false);
  if (!ok) return MBD_E_CUDA;

  Params p{};
  p.E = c.E; p.T = static_cast<int>(c.T);
  p.offsets = c.offsets;
  p.M = static_cast<int>(M); p.N = static_cast<int>(N);
  const int64_t K = c.variant == 0 ? c.d_in : c.d_out;
  const int per_kb = c.kind == KIND_I8 ? 128 : 64;
  p.kb_total = static_cast<int>((K + per_kb - 1) / per_kb);
  p.m_tiles = static_cast<int>((M + (l.pair ? 2 * CH : CH) - 1) / (l.pair ? 2 * CH : CH));
  p.n_tiles = static_cast<int>((N + l.BN - 1) / l.BN);
  if (c.variant == 2) {                   // the rows of dW_e are dealt out evenly over its tiles
    const int unit_rows = l.pair ? 128 : 64;
    p.n_step = (p.N + p.n_tiles - 1) / p.n_tiles;
    p.n_step = (p.n_step + unit_rows - 1) / unit_rows * unit_rows;
    p.per_expert = Divisor(static_cast<uint32_t>(p.m_tiles) * p.n_tiles);
  }
  p.per_group = Divisor(static_cast<uint32_t>(GROUP_N) * p.m_tiles);
  for (int k = 0; k < GROUP_N; ++k) p.by[k] = Divisor(k + 1);
  p.chunked_a = chunked_a; p.chunked_b = chunked_b;
  p.seg = c.kind == KIND_BF16 && !t->out_bf16 && !l.split ? SEG_BLOCKS : 1 << 30;
  p.op = t->op == MBD_TAIL_STORE ? EPI_ACT : t->op == MBD_TAIL_MASK ? EPI_MASK : EPI_SGD;
  p.out_bf16 = t->out_bf16 != 0;
  p.relu = t->relu != 0;
  p.out = t->out_dev;
  p.ldo = t->ldo;
  p.out_stride = c.variant == 2 ? (c.E > 1 ? c.stride : 0) : 0;
  p.bias = t->bias_dev;
  p.mask = t->op == MBD_TAIL_MASK ? t->mask_dev : nullptr;
  p.ldmask = t->ldmask;
  p.scale = t->scale;
  p.row_scale = c.row_scale;
  p.ch_scale = c.ch_scale;

  int* word = c.status;
  if (!word) {
    if (cudaMalloc(reinterpret_cast<void**>(&word), sizeof(int)) != cudaSuccess) { (void)cudaGetLastError(); return MBD_E_ALLOC; }
    if (cudaMemsetAsync(word, 0, sizeof(int), stream) != cudaSuccess) { (void)cudaGetLastError(); cudaFree(word); return MBD_E_CUDA; }
  }
  p.status = word;
  cudaError_t e;
  if (c.kind == KIND_I8) e = launch<KIND_I8, 0, 0>(l, a, b, b32, out, p, stream);
  else if (c.variant == 0) e = launch<KIND_BF16, 0, 0>(l, a, b, b32, out, p, stream);
  else if (c.variant == 1) e = launch<KIND_BF16, 1, 0>(l, a, b, b32, out, p, stream);
  else e = launch<KIND_BF16, 1, 1>(l, a, b, b32, out, p, stream);
  mbd_status ret = e == cudaSuccess ? MBD_OK : MBD_E_CUDA;
  if (c.status) {                          // enqueue-only: the caller owns and reads the status word
    if (ret != MBD_OK) (void)cudaGetLastError();
    return ret;
  }
  int h = 0;
  if (ret == MBD_OK) {
    if (cudaStreamSynchronize(stream) != cudaSuccess || cudaMemcpy(&h, word, sizeof(int), cudaMemcpyDeviceToHost) != cudaSuccess) ret = MBD_E_CUDA;
    else if (h != 0) ret = h == DEV_SMEM_MISALIGNED ? MBD_E_CUDA : MBD_E_TIMEOUT;
  }
  (void)cudaGetLastError();
  cudaFree(word);
  return ret;
}

}  // namespace
}  // namespace mbd

using namespace mbd;

extern "C" mbd_status mbd_expert_gemm_bf16(int variant, int E, const int32_t* offsets_dev, int64_t T, int64_t d_out, int64_t d_in,
                                           const void* A_dev, int64_t lda, const void* B_dev, int64_t ldb, int64_t expert_stride,
                                           const mbd_tail* tail, int32_t* status_dev, void* cuda_stream) {
  if (!offsets_dev) return MBD_E_INVALID;
  return run(Call{KIND_BF16, variant, E, offsets_dev, T, d_out, d_in, A_dev, lda, B_dev, ldb, expert_stride, nullptr, nullptr, tail,
                  status_dev, cuda_stream});
}

extern "C" mbd_status mbd_expert_gemm_i8(int E, const int32_t* offsets_dev, int64_t T, int64_t d_out, int64_t d_in, const int8_t* A_dev,
                                         int64_t lda, const float* a_scale_dev, const int8_t* B_dev, int64_t ldb, int64_t expert_stride,
                                         const float* b_scale_dev, const mbd_tail* tail, int32_t* status_dev, void* cuda_stream) {
  if (!offsets_dev) return MBD_E_INVALID;
  return run(Call{KIND_I8, 0, E, offsets_dev, T, d_out, d_in, A_dev, lda, B_dev, ldb, expert_stride, a_scale_dev, b_scale_dev, tail,
                  status_dev, cuda_stream});
}

extern "C" mbd_status mbd_gemm_i8(int64_t M, int64_t N, int64_t K, const int8_t* A_dev, int64_t lda, const float* a_scale_dev,
                                  const int8_t* B_dev, int64_t ldb, const float* b_scale_dev, const mbd_tail* tail, int32_t* status_dev,
                                  void* cuda_stream) {
  if (M < 1) return MBD_E_INVALID;
  return run(Call{KIND_I8, 0, 1, nullptr, M, N, K, A_dev, lda, B_dev, ldb, 0, a_scale_dev, b_scale_dev, tail, status_dev, cuda_stream});
}
