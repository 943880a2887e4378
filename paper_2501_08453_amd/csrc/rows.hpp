// What the row kernels around a block's attention share (residual.hip, checkpoint.hip, embedding.hip): N = 8 or 4
// consecutive columns of a row as a thread's vector, sums over a row, and the 8-bit form of a checkpoint.
//
// Vectors are of eight columns where a tensor is bf16 (16 bytes a lane), of four where all are fp32, so that a wave reads and writes
// whole lines in one instruction. (Of a fp32 tensor beside a bf16 one, two instructions take half of every line each. Vectors of
// four there, with 8 bytes a lane of the bf16 one, were slower in the first kernels; in the present ones they take 13.4 us against
// 15.2 in the residual's forward of 3,712 x 1,024, 20.6 against 20.2 in its backward, and 64 against 71 in the sums of 65,536 rows of
// 1,536 to a fp32 gradient.)
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace vcja {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kBlockOf8 = 128;  // columns of a row that share a checkpoint's scale
constexpr float kTopScale = 0x1.020406p+121f;

// A vector as it lies in memory, at any multiple of its elements' size: rows of odd length, or of odd stride, start anywhere (the
// hardware takes such addresses in its wide loads and stores of global memory).
template <class X, int N>
struct Raw;
template <>
struct Raw<__bf16, 8> {
  typedef bf16x8 type;
  typedef bf16x8 any __attribute__((aligned(2)));
};
template <>
struct Raw<__bf16, 4> {
  typedef bf16x4 type;
  typedef bf16x4 any __attribute__((aligned(2)));
};
template <>
struct Raw<float, 4> {
  typedef f32x4 type;
  typedef f32x4 any __attribute__((aligned(4)));
};
template <>
struct Raw<int8_t, 8> {
  typedef u32x2 type;
  typedef u32x2 any __attribute__((aligned(1)));
};
template <>
struct Raw<int8_t, 4> {
  typedef uint32_t type;
  typedef uint32_t any __attribute__((aligned(1)));
};

__device__ __forceinline__ uint32_t word(u32x2 v, int i) { return v[i]; }
__device__ __forceinline__ uint32_t word(uint32_t v, int) { return v; }

template <class X, int N>
struct Cols;
template <>
struct Cols<float, 8> {
  f32x4 v, w;
  __device__ __forceinline__ float operator[](int e) const { return e < 4 ? v[e] : w[e - 4]; }
};
template <class X, int N>
struct Cols {
  typename Raw<X, N>::type v;
  __device__ __forceinline__ float operator[](int e) const {
    if constexpr (sizeof(X) == 1)
      return (float)(int8_t)(word(v, e >> 2) >> (8 * (e & 3)));
    else
      return (float)v[e];
  }
};

// The columns of a thread that begins at column c of a row of C: N from `col` on, of which [lo, hi) are its own. Where the row
// ends within them they are the row's last N, the first of which are the neighbour's too, and a thread
// behind the row's end (lo = N) has those as well: every thread loads the same way, without a branch around its loads (an
// alternative that writes the same registers waits for the load first). Rows of less than N columns: [0, hi) of the first thread.
template <int N>
struct Span {
  int col, lo, hi;
  __device__ __forceinline__ bool has(int e) const { return e >= lo && e < hi; }
  __device__ __forceinline__ bool any() const { return lo < N; }
};
template <int N>
__device__ __forceinline__ Span<N> span_at(int c, int C) {
  if (C < N) return Span<N>{0, c ? N : 0, C};
  const int col = min(c, C - N);
  return Span<N>{col, min(c - col, N), N};
}
// Whether element e is the thread's own. ODD: rows may end within a thread's columns, or be of less than N; else it has all or none.
template <bool ODD, int N>
__device__ __forceinline__ bool own(const Span<N>& s, int e) {
  return ODD ? s.has(e) : s.lo == 0;
}
// A vector at p, whole. ONCE: it is not used again soon, and goes past the caches.
template <bool ONCE, class X, int N>
__device__ __forceinline__ void get(Cols<X, N>& r, const X* p) {
  if constexpr (sizeof(X) * N > 16) {
    Cols<X, 4> u;
    get<ONCE>(u, p);
    r.v = u.v;
    get<ONCE>(u, p + 4);
    r.w = u.v;
  } else if constexpr (ONCE) {
    r.v = __builtin_nontemporal_load((const typename Raw<X, N>::any*)p);
  } else {
    r.v = *(const typename Raw<X, N>::any*)p;
  }
}
template <bool ONCE, int N, class X>
__device__ __forceinline__ void put(X* p, const float* x) {
  if constexpr (sizeof(X) * N > 16) {
    put<ONCE, 4>(p, x);
    put<ONCE, 4>(p + 4, x + 4);
  } else {
    typename Raw<X, N>::type v;
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = (X)x[e];
    if constexpr (ONCE)
      __builtin_nontemporal_store(v, (typename Raw<X, N>::any*)p);
    else
      *(typename Raw<X, N>::any*)p = v;
  }
}
// The columns at p + s.col.
template <bool ODD = true, bool ONCE = false, class X, int N>
__device__ __forceinline__ void load_cols(Cols<X, N>& r, const X* p, const Span<N>& s) {
  p += s.col;
  if (!ODD || s.hi == N) {
    get<ONCE>(r, p);
  } else {
    r = Cols<X, N>{};
#pragma unroll
    for (int e = 0; e < N - 1; ++e)
      if (e < s.hi) {
        if constexpr (sizeof(X) == 1) {
          const uint32_t b = (uint32_t)(uint8_t)p[e] << (8 * (e & 3));
          if constexpr (N == 8)
            r.v[e >> 2] |= b;
          else
            r.v |= b;
        } else if constexpr (sizeof(X) * N > 16) {
          if (e < 4)
            r.v[e] = p[e];
          else
            r.w[e - 4] = p[e];
        } else {
          r.v[e] = p[e];
        }
      }
  }
}
// The thread's own columns of x to p + s.col, each rounded once to the type.
template <bool ODD = true, bool ONCE = false, class X, int N>
__device__ __forceinline__ void store_cols(X* p, const float* x, const Span<N>& s) {
  p += s.col;
  if (s.lo == 0 && (!ODD || s.hi == N)) {
    put<ONCE, N>(p, x);
  } else if constexpr (ODD) {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (s.has(e)) p[e] = (X)x[e];
  }
}
// Columns of a parameter vector whose type only the call knows; `other` without one.
template <bool ODD = true, int N>
__device__ __forceinline__ void load_param(float* out, const void* p, bool f32, const Span<N>& s, float other) {
  if (!p) {
#pragma unroll
    for (int e = 0; e < N; ++e) out[e] = other;
  } else if (f32) {
    Cols<float, N> r;
    load_cols<ODD>(r, (const float*)p, s);
#pragma unroll
    for (int e = 0; e < N; ++e) out[e] = r[e];
  } else {
    Cols<__bf16, N> r;
    load_cols<ODD>(r, (const __bf16*)p, s);
#pragma unroll
    for (int e = 0; e < N; ++e) out[e] = r[e];
  }
}

// A value of another lane of the same 16, by the DPP control C.
template <int C>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, C, 0xf, 0xf, true);
}
template <int C>
__device__ __forceinline__ float dppf(float x) {
  return __uint_as_float(dpp<C>(__float_as_uint(x)));
}
constexpr int kSwap1 = 0xb1, kSwap2 = 0x4e, kHalfMirror = 0x141, kMirror = 0x140;  // quad_perm 1,0,3,2 / 2,3,0,1, row mirrors

// Sum over a wave, the same in every lane: within rows of 16 lanes by DPP, the four rows' sums as scalars.
__device__ __forceinline__ float wave_sum(float x) {
  x += dppf<kSwap1>(x);
  x += dppf<kSwap2>(x);
  x += dppf<kHalfMirror>(x);
  x += dppf<kMirror>(x);
  const int b = __float_as_int(x);
  return (__int_as_float(__builtin_amdgcn_readlane(b, 0)) + __int_as_float(__builtin_amdgcn_readlane(b, 16))) +
         (__int_as_float(__builtin_amdgcn_readlane(b, 32)) + __int_as_float(__builtin_amdgcn_readlane(b, 48)));
}

// The 8-bit form of a block of 128 columns, N in each of 128 / N lanes (zeros where they are not a lane's own): whole steps of
// a 127th of the largest magnitude, at least 2^-100. The largest is found over the bits of |x|, where a NaN is larger than an
// infinity and that than any number: such a block's scale is NaN, and so is all that is unpacked from it.
// Scales are at most the largest number whose 127 fold is finite: that of the largest fp32 numbers is a step of 2^-24 below theirs.
// |x (127 / top)| is at most 127 (1 + 2^-23), which rounds to 127.
template <int N>
struct Kept {
  typename Raw<int8_t, N>::type q;
  float scale;
};
template <int N>
__device__ __forceinline__ Kept<N> keep(const float* x) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < N; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
  top = max(top, dpp<kSwap1>(top));
  top = max(top, dpp<kSwap2>(top));
  top = max(top, dpp<kHalfMirror>(top));
  top = max(top, dpp<kMirror>(top));
  if constexpr (N == 4) top = max(top, (uint32_t)__shfl_xor((int)top, 16, 64));
  const bool finite = top < 0x7f800000u;
  const float m = finite ? fmaxf(__uint_as_float(top), 0x1p-100f) : 1.0f;
  const float inv = 127.0f / m;
  Kept<N> k;
  k.scale = finite ? fminf(m / 127.0f, kTopScale) : __uint_as_float(0x7fc00000u);
  uint32_t w[N / 4];
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    uint32_t q[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) q[e] = (uint32_t)(int)rintf(finite ? x[4 * i + e] * inv : 0.0f) & 0xffu;
    w[i] = q[0] | q[1] << 8 | q[2] << 16 | q[3] << 24;
  }
  if constexpr (N == 8)
    k.q = u32x2{w[0], w[1]};
  else
    k.q = w[0];
  return k;
}
template <bool ODD = true, int N>
__device__ __forceinline__ void store_kept(int8_t* p, const Kept<N>& k, const Span<N>& s) {
  p += s.col;
  if (s.lo == 0 && (!ODD || s.hi == N)) {
    *(typename Raw<int8_t, N>::any*)p = k.q;
  } else if constexpr (ODD) {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (s.has(e)) p[e] = (int8_t)(word(k.q, e >> 2) >> (8 * (e & 3)));
  }
}

}  // namespace vcja
