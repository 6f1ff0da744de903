// Eight values of a row as one thread holds them (bf16 pairs packed as they lie in memory, or floats), shared by the norm and by the
// rows' way to the experts and back.
//
// n threads share a row; vector j of thread t is
//   WIDE:  the eight columns from 8 (t + j n) on, one access of 16 bytes (bf16) or 32 bytes (float).  The row's length is a multiple of 8,
//          its address a multiple of the access.
//   else:  the columns t + (8 j + i) n, i < 8: any length and alignment, neighbouring threads at neighbouring columns.
// A column belongs to the same thread whatever the tensor's type, so that a result may take the place of what it was made from.
#pragma once
#include "epi.cuh"
#include "pairs.cuh"

namespace mbd {

template <typename T> struct Raw8;
template <> struct Raw8<__nv_bfloat16> {
  uint32_t w[4];
  // unpacked anew from here on (the compiler would keep the floats beside the packed values: twice the registers)
  __device__ __forceinline__ void repack() { asm volatile("" : "+r"(w[0]), "+r"(w[1]), "+r"(w[2]), "+r"(w[3])); }
  __device__ __forceinline__ void clear() { w[0] = w[1] = w[2] = w[3] = 0u; }
  __device__ __forceinline__ float at(int i) const { return __uint_as_float(i & 1 ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16); }
  __device__ __forceinline__ f32x2 two(int i) const { return pair(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u)); }
  __device__ __forceinline__ void set(const float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
  }
};
template <> struct Raw8<float> {
  float f[8];
  __device__ __forceinline__ void repack() {}
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = 0.f;
  }
  __device__ __forceinline__ float at(int i) const { return f[i]; }
  __device__ __forceinline__ f32x2 two(int i) const { return pair(f[2 * i], f[2 * i + 1]); }
  __device__ __forceinline__ void set(const float* v) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = v[i];
  }
};

__device__ __forceinline__ void read8(const __nv_bfloat16* p, Raw8<__nv_bfloat16>& r) {
  asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]) : "l"(p) : "memory");
}
__device__ __forceinline__ void read8(const float* p, Raw8<float>& r) {
  asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=f"(r.f[0]), "=f"(r.f[1]), "=f"(r.f[2]), "=f"(r.f[3]), "=f"(r.f[4]), "=f"(r.f[5]), "=f"(r.f[6]), "=f"(r.f[7]) : "l"(p) : "memory");
}
__device__ __forceinline__ void write8(__nv_bfloat16* p, const Raw8<__nv_bfloat16>& r) {
  asm volatile("st.global.v4.b32 [%0], {%1, %2, %3, %4};" :: "l"(p), "r"(r.w[0]), "r"(r.w[1]), "r"(r.w[2]), "r"(r.w[3]) : "memory");
}
__device__ __forceinline__ void write8(float* p, const Raw8<float>& r) {
  asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               :: "l"(p), "f"(r.f[0]), "f"(r.f[1]), "f"(r.f[2]), "f"(r.f[3]), "f"(r.f[4]), "f"(r.f[5]), "f"(r.f[6]), "f"(r.f[7]) : "memory");
}

// Column of value i of vector j of thread t (rows are a little shorter than 2^31).
template <bool WIDE> __device__ __forceinline__ int column(int t, int j, int n, int i) {
  return WIDE ? 8 * (t + j * n) + i : t + (8 * j + i) * n;
}

// Columns from K on read as zero.
template <bool WIDE>
__device__ __forceinline__ void load8(const __nv_bfloat16* row, int t, int j, int n, int K, Raw8<__nv_bfloat16>& r) {
  r.clear();
  if (WIDE) {
    if (column<true>(t, j, n, 0) < K) read8(row + column<true>(t, j, n, 0), r);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = column<false>(t, j, n, i);
      if (c < K) r.w[i >> 1] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(row)[c]) << (i & 1 ? 16 : 0);
    }
  }
}
template <bool WIDE>
__device__ __forceinline__ void load8(const float* row, int t, int j, int n, int K, Raw8<float>& r) {
  r.clear();
  if (WIDE) {
    if (column<true>(t, j, n, 0) < K) read8(row + column<true>(t, j, n, 0), r);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = column<false>(t, j, n, i);
      if (c < K) r.f[i] = row[c];
    }
  }
}
template <bool WIDE>
__device__ __forceinline__ void store8(__nv_bfloat16* row, int t, int j, int n, int K, const Raw8<__nv_bfloat16>& r) {
  if (WIDE) {
    if (column<true>(t, j, n, 0) < K) write8(row + column<true>(t, j, n, 0), r);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = column<false>(t, j, n, i);
      if (c < K) reinterpret_cast<uint16_t*>(row)[c] = static_cast<uint16_t>(r.w[i >> 1] >> (i & 1 ? 16 : 0));
    }
  }
}
template <bool WIDE>
__device__ __forceinline__ void store8(float* row, int t, int j, int n, int K, const Raw8<float>& r) {
  if (WIDE) {
    if (column<true>(t, j, n, 0) < K) write8(row + column<true>(t, j, n, 0), r);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = column<false>(t, j, n, i);
      if (c < K) row[c] = r.f[i];
    }
  }
}

// ---- host: where a tensor of rows lies ------------------------------------------------------------------------------
struct Rows {
  const void* base;
  int64_t rows, width, ld;     // elements
  int size;                    // bytes of an element
  bool wide() const {          // whether all of its rows can be read eight values at a time
    const int unit = size == 1 ? 8 : 8 * size;
    return !base || (reinterpret_cast<uintptr_t>(base) % unit == 0 && (rows <= 1 || ld % 8 == 0));
  }
  bool misplaced() const { return reinterpret_cast<uintptr_t>(base) % size != 0; }
};
// Whether two tensors share no byte (columns of one wider buffer among them).
inline bool apart(const Rows& a, const Rows& b) {
  if (!a.base || !b.base || a.rows < 1 || b.rows < 1) return true;
  const __int128 pa = reinterpret_cast<intptr_t>(a.base), pb = reinterpret_cast<intptr_t>(b.base);
  const __int128 wa = static_cast<__int128>(a.width) * a.size, wb = static_cast<__int128>(b.width) * b.size;
  const __int128 la = static_cast<__int128>(a.rows > 1 ? a.ld : a.width) * a.size, lb = static_cast<__int128>(b.rows > 1 ? b.ld : b.width) * b.size;
  if (pa + la * (a.rows - 1) + wa <= pb || pb + lb * (b.rows - 1) + wb <= pa) return true;
  if (la != lb) return false;
  const __int128 at = ((pb - pa) % la + la) % la;            // of b's first column in a's rows
  return at >= wa && at + wb <= la;
}
// A result may also lie exactly where an input of its type lies: each element is read before the thread that owns it writes it.
inline bool same_place(const Rows& a, const Rows& b) {
  return a.base == b.base && a.size == b.size && a.rows == b.rows && a.width == b.width && (a.rows <= 1 || a.ld == b.ld);
}
inline bool apart_or_same(const Rows& out, const Rows& in) { return apart(out, in) || same_place(out, in); }

}  // namespace mbd
