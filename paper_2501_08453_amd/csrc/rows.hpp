// What the row kernels around a block's attention share (residual.hip, checkpoint.hip, embedding.hip): eight
// consecutive columns of a row per thread, sums over a row, and the 8-bit form of a checkpoint.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace vcja {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
// The same at any multiple of their elements' size: rows of odd length, or of odd stride, start anywhere. The hardware
// takes such addresses in its wide loads and stores of global memory.
typedef bf16x8 bf16x8_any __attribute__((aligned(2)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef u32x2 u32x2_any __attribute__((aligned(1)));

constexpr int kBlockOf8 = 128;  // columns of a row that share a checkpoint's scale: 16 threads, a row of DPP lanes

// Eight columns as they lie in memory.
template <class X>
struct Eight;
template <>
struct Eight<__bf16> {
  bf16x8 v;
  __device__ __forceinline__ float operator[](int e) const { return (float)v[e]; }
};
template <>
struct Eight<float> {
  f32x4 lo, hi;
  __device__ __forceinline__ float operator[](int e) const { return e < 4 ? lo[e] : hi[e - 4]; }
};
template <>
struct Eight<int8_t> {
  u32x2 v;
  __device__ __forceinline__ float operator[](int e) const { return (float)(int8_t)(v[e >> 2] >> (8 * (e & 3))); }
};

__device__ __forceinline__ void get(Eight<__bf16>& r, const __bf16* p) { r.v = *(const bf16x8_any*)p; }
__device__ __forceinline__ void get(Eight<float>& r, const float* p) {
  r.lo = *(const f32x4_any*)p;
  r.hi = *(const f32x4_any*)(p + 4);
}
__device__ __forceinline__ void get(Eight<int8_t>& r, const int8_t* p) { r.v = *(const u32x2_any*)p; }
__device__ __forceinline__ void set(Eight<__bf16>& r, int e, const __bf16* p) { r.v[e] = *p; }
__device__ __forceinline__ void set(Eight<float>& r, int e, const float* p) {
  if (e < 4)
    r.lo[e] = *p;
  else
    r.hi[e - 4] = *p;
}
__device__ __forceinline__ void set(Eight<int8_t>& r, int e, const int8_t* p) {
  r.v[e >> 2] |= (uint32_t)(uint8_t)*p << (8 * (e & 3));
}
// The first n (all of them from 8 on) columns at p; zeros behind them.
template <class X>
__device__ __forceinline__ void load8(Eight<X>& r, const X* p, int n) {
  if (n >= 8) {
    get(r, p);
  } else {
    r = Eight<X>{};
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < n) set(r, e, p + e);
  }
}

__device__ __forceinline__ void put(__bf16* p, const float* x) {
  bf16x8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (__bf16)x[e];
  *(bf16x8_any*)p = v;
}
__device__ __forceinline__ void put(float* p, const float* x) {
  *(f32x4_any*)p = f32x4{x[0], x[1], x[2], x[3]};
  *(f32x4_any*)(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
}
// The first n of x, each rounded once to the type.
template <class X>
__device__ __forceinline__ void store8(X* p, const float* x, int n) {
  if (n >= 8) {
    put(p, x);
  } else {
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < n) p[e] = (X)x[e];
  }
}
// Columns of a parameter or gradient vector whose type only the call knows.
__device__ __forceinline__ void load8p(float* out, const void* p, bool f32, int64_t at, int n, float other) {
#pragma unroll
  for (int e = 0; e < 8; ++e) out[e] = other;
  if (!p || n <= 0) return;
  if (f32) {
    Eight<float> r;
    load8(r, (const float*)p + at, n);
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = e < n ? r[e] : other;
  } else {
    Eight<__bf16> r;
    load8(r, (const __bf16*)p + at, n);
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = e < n ? r[e] : other;
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
__device__ __forceinline__ uint32_t max16(uint32_t x) {  // over the 16 lanes of a row
  x = max(x, dpp<kSwap1>(x));
  x = max(x, dpp<kSwap2>(x));
  x = max(x, dpp<kHalfMirror>(x));
  return max(x, dpp<kMirror>(x));
}

// The 8-bit form of a block of 128 columns, eight in each of 16 lanes (zeros behind a row's end): whole steps of
// a 127th of the largest magnitude, at least 2^-100. The largest is found over the bits of |x|, where a NaN is larger than an
// infinity and that than any number: such a block's scale is NaN, and so is all that is unpacked from it.
// |x (127 / top)| is at most 127 (1 + 2^-23), which rounds to 127.
struct Kept {
  u32x2 q;
  float scale;
};
__device__ __forceinline__ Kept keep8(const float* x) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
  top = max16(top);
  const bool finite = top < 0x7f800000u;
  const float m = finite ? fmaxf(__uint_as_float(top), 0x1p-100f) : 1.0f;
  const float inv = 127.0f / m;
  Kept k;
  k.scale = finite ? m / 127.0f : __uint_as_float(0x7fc00000u);
  uint32_t q[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) q[e] = (uint32_t)(int)rintf(finite ? x[e] * inv : 0.0f) & 0xffu;
  k.q = u32x2{q[0] | q[1] << 8 | q[2] << 16 | q[3] << 24, q[4] | q[5] << 8 | q[6] << 16 | q[7] << 24};
  return k;
}
__device__ __forceinline__ void store_q8(int8_t* p, u32x2 q, int n) {
  if (n >= 8) {
    *(u32x2_any*)p = q;
  } else {
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < n) p[e] = (int8_t)(q[e >> 2] >> (8 * (e & 3)));
  }
}

}  // namespace vcja
