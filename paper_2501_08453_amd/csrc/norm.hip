// Layer norm for gfx950, forward and backward: y = (x - mean) rstd w + b over the columns of
// each row, rstd = 1 / sqrt(mean of (x - mean)^2 + eps). Sums in fp32, the variance of the
// differences to the mean (never as a difference of squares, which cancels far from 0).
//
// Memory-bound: a row is read once and kept in registers, by one wave up to 1,536 columns (no
// barrier), by a workgroup of 4 waves up to 6,144 and of 16 up to 8,192; wider rows are read again
// for each sum, from the caches. (24 columns a thread at most: 32 spilled in the backward.) A wave (workgroup) takes every so many rows, so that the weights are loaded once
// and, backward, the column sums of dout xhat and of dout stay in its registers; the workgroups'
// sums are then added up in order by a second kernel. Rows wider than 8,192 columns are far from
// the memory's rate (one element a load): 5,000 x 16,384 in bf16 forward 212 us, 1.5 TB/s, backward 285, 1.7. 57,856 x 1,536 in bf16: forward 76 us, 4.7 TB/s,
// backward 127 us, 4.2 TB/s (a copy reaches 5.0 to 5.2).
#include "norm.hpp"

#include <algorithm>
#include <type_traits>

namespace vcja {
namespace {

constexpr int kThreads = 256;      // of a workgroup, unless one row takes more
constexpr int kWaveCols = 1536;    // widest row of one wave
constexpr int kBlockCols = 8192;   // ... of one workgroup that keeps it
template <int TPR>
constexpr int kWg = TPR > kThreads ? TPR : kThreads;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// VE consecutive elements of type X as they lie in memory (16 bytes, or one).
template <class X, int VE>
struct Raw {
  typedef X type __attribute__((ext_vector_type(VE)));
};
template <class X>
struct Raw<X, 1> {
  typedef X type;
};
template <class X, int VE>
__device__ __forceinline__ float elem(const typename Raw<X, VE>::type& r, int e) {
  if constexpr (VE == 1)
    return (float)r;
  else
    return (float)r[e];
}

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}
// Sum over the TPR threads of a row. red: a float per wave that no thread still reads.
template <int TPR>
__device__ __forceinline__ float waves_sum(const float* red) {
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < TPR / 64; i += 4) s += (red[i] + red[i + 1]) + (red[i + 2] + red[i + 3]);
  return s;
}
template <int TPR>
__device__ __forceinline__ float row_sum(float x, float* red) {
  x = wave_sum(x);
  if constexpr (TPR == 64) return x;
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  return waves_sum<TPR>(red);
}

// The parameters of this thread's columns (`other` without them).
template <int VE, int NV, int TPR>
__device__ __forceinline__ void load_params(const void* p, bool f32, float other, int C, int t, float* out) {
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * TPR + t) * VE;
#pragma unroll
    for (int e = 0; e < VE; ++e) out[v * VE + e] = other;
    if (p && c < C) {
#pragma unroll
      for (int e = 0; e < VE; ++e) out[v * VE + e] = f32 ? ((const float*)p)[c + e] : (float)((const __bf16*)p)[c + e];
    }
  }
}

template <class X, int VE, int EPT, int TPR>
__global__ __launch_bounds__(kWg<TPR>) void norm_fwd_kernel(NormArgs a) {
  constexpr int NV = EPT / VE;
  using R = typename Raw<X, VE>::type;
  __shared__ float red[2][16];
  const int t = threadIdx.x % TPR, C = a.cols;
  float w[EPT], b[EPT];
  load_params<VE, NV, TPR>(a.w, a.p_f32, 1.0f, C, t, w);
  load_params<VE, NV, TPR>(a.b, a.p_f32, 0.0f, C, t, b);
  const int step = gridDim.x * (kWg<TPR> / TPR);
  R r[NV];
  auto load = [&](int row, R* to) {
    const X* x = (const X*)a.x + row * a.stride;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * TPR + t) * VE;
      if (c < C) to[v] = *(const R*)(x + c);
    }
  };
  int row = blockIdx.x * (kWg<TPR> / TPR) + threadIdx.x / TPR;
  if (row < a.rows) load(row, r);
  for (; row < a.rows; row += step) {
    R next[NV];
    if (row + step < a.rows) load(row + step, next);  // in flight during this row
    float s = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if ((v * TPR + t) * VE < C)
#pragma unroll
        for (int e = 0; e < VE; ++e) s += elem<X, VE>(r[v], e);
    const float mean = row_sum<TPR>(s, red[0]) / C;
    s = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if ((v * TPR + t) * VE < C)
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const float d = elem<X, VE>(r[v], e) - mean;
          s = fmaf(d, d, s);
        }
    const float rstd = 1.0f / sqrtf(row_sum<TPR>(s, red[1]) / C + a.eps);
    X* y = (X*)a.y + (int64_t)row * C;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * TPR + t) * VE;
      if (c < C) {
        R o;
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const X z = (X)fmaf((elem<X, VE>(r[v], e) - mean) * rstd, w[v * VE + e], b[v * VE + e]);
          if constexpr (VE == 1)
            o = z;
          else
            o[e] = z;
        }
        *(R*)(y + c) = o;
      }
    }
    if (t == 0) {
      a.mean[row] = mean;
      a.rstd[row] = rstd;
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) r[v] = next[v];
  }
}

template <class X, int VE, int EPT, int TPR>
__global__ __launch_bounds__(kWg<TPR>, TPR > kThreads ? 1 : 2) void norm_bwd_kernel(NormArgs a) {
  constexpr int NV = EPT / VE;
  using R = typename Raw<X, VE>::type;
  __shared__ float red[2][2][16];
  __shared__ float comb[TPR == 64 ? EPT * kThreads : 1];
  const int t = threadIdx.x % TPR, C = a.cols;
  float w[EPT], dw[EPT], db[EPT];
  load_params<VE, NV, TPR>(a.w, a.p_f32, 1.0f, C, t, w);
#pragma unroll
  for (int i = 0; i < EPT; ++i) dw[i] = db[i] = 0.0f;
  const int step = gridDim.x * (kWg<TPR> / TPR);
  R x[NV], dy[NV];
  float mean = 0.0f, rstd = 0.0f;
  auto load = [&](int row, R* px, R* pd, float& m, float& q) {
    const X *rx = (const X*)a.x + row * a.stride, *rd = (const X*)a.dout + row * a.dout_stride;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * TPR + t) * VE;
      if (c < C) {
        px[v] = *(const R*)(rx + c);
        pd[v] = *(const R*)(rd + c);
      }
    }
    m = a.mean[row];
    q = a.rstd[row];
  };
  int row = blockIdx.x * (kWg<TPR> / TPR) + threadIdx.x / TPR, par = 0;
  if (row < a.rows) load(row, x, dy, mean, rstd);
  for (; row < a.rows; row += step, par ^= 1) {
    R nx[NV], nd[NV];
    float nm = 0.0f, nr = 0.0f;
    if (row + step < a.rows) load(row + step, nx, nd, nm, nr);  // in flight during this row
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if ((v * TPR + t) * VE < C)
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const int i = v * VE + e;
          const float d = elem<X, VE>(dy[v], e), xh = (elem<X, VE>(x[v], e) - mean) * rstd, g = d * w[i];
          s1 += g;
          s2 = fmaf(g, xh, s2);
          db[i] += d;
          dw[i] = fmaf(d, xh, dw[i]);
        }
    s1 = wave_sum(s1);
    s2 = wave_sum(s2);
    if constexpr (TPR != 64) {  // both sums behind one barrier; the buffers alternate
      if ((threadIdx.x & 63) == 0) {
        red[par][0][threadIdx.x >> 6] = s1;
        red[par][1][threadIdx.x >> 6] = s2;
      }
      __syncthreads();
      s1 = waves_sum<TPR>(red[par][0]);
      s2 = waves_sum<TPR>(red[par][1]);
    }
    s1 /= C;
    s2 /= C;
    X* dx = (X*)a.dx + (int64_t)row * C;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * TPR + t) * VE;
      if (c < C) {
        R o;
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const float xh = (elem<X, VE>(x[v], e) - mean) * rstd;
          const X z = (X)(rstd * (elem<X, VE>(dy[v], e) * w[v * VE + e] - s1 - xh * s2));
          if constexpr (VE == 1)
            o = z;
          else
            o[e] = z;
        }
        *(R*)(dx + c) = o;
      }
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      x[v] = nx[v];
      dy[v] = nd[v];
    }
    mean = nm;
    rstd = nr;
  }
  if (!a.dw && !a.db) return;
  // Column sums of the workgroup (its waves' in order) to its row of the partials.
  auto write = [&](const float* sums, float* out) {
    if constexpr (TPR == 64) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < EPT; ++i) comb[i * kThreads + threadIdx.x] = sums[i];
      __syncthreads();
      for (int i = threadIdx.x >> 6; i < EPT; i += kThreads / 64) {
        const int c = (i / VE * TPR + t) * VE + i % VE;
        const float* p = comb + i * kThreads + t;
        if (c < C) out[c] = (p[0] + p[64]) + (p[128] + p[192]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < EPT; ++i) {
        const int c = (i / VE * TPR + t) * VE + i % VE;
        if (c < C) out[c] = sums[i];
      }
    }
  };
  write(dw, a.part + (size_t)blockIdx.x * C);
  write(db, a.part + ((size_t)a.groups + blockIdx.x) * C);
}

// Rows of more than kBlockCols columns: a workgroup per row, read again for each sum.
__device__ __forceinline__ float block_sum(float x, float* red) {
  __syncthreads();
  return row_sum<kThreads>(x, red);
}
__device__ __forceinline__ float param(const void* p, bool f32, int c, float other) {
  return !p ? other : f32 ? ((const float*)p)[c] : (float)((const __bf16*)p)[c];
}
template <class X>
__global__ __launch_bounds__(kThreads) void norm_wide_fwd_kernel(NormArgs a) {
  __shared__ float red[4];
  const int row = blockIdx.x, C = a.cols;
  const X* x = (const X*)a.x + row * a.stride;
  X* y = (X*)a.y + (int64_t)row * C;
  float s = 0.0f;
  for (int c = threadIdx.x; c < C; c += kThreads) s += (float)x[c];
  const float mean = block_sum(s, red) / C;
  s = 0.0f;
  for (int c = threadIdx.x; c < C; c += kThreads) {
    const float d = (float)x[c] - mean;
    s = fmaf(d, d, s);
  }
  const float rstd = 1.0f / sqrtf(block_sum(s, red) / C + a.eps);
  for (int c = threadIdx.x; c < C; c += kThreads)
    y[c] = (X)fmaf(((float)x[c] - mean) * rstd, param(a.w, a.p_f32, c, 1.0f), param(a.b, a.p_f32, c, 0.0f));
  if (threadIdx.x == 0) {
    a.mean[row] = mean;
    a.rstd[row] = rstd;
  }
}
template <class X>
__global__ __launch_bounds__(kThreads) void norm_wide_dx_kernel(NormArgs a) {
  __shared__ float red[4];
  const int row = blockIdx.x, C = a.cols;
  const X* x = (const X*)a.x + row * a.stride;
  const X* dy = (const X*)a.dout + row * a.dout_stride;
  X* dx = (X*)a.dx + (int64_t)row * C;
  const float mean = a.mean[row], rstd = a.rstd[row];
  float s1 = 0.0f, s2 = 0.0f;
  for (int c = threadIdx.x; c < C; c += kThreads) {
    const float g = (float)dy[c] * param(a.w, a.p_f32, c, 1.0f);
    s1 += g;
    s2 = fmaf(g, ((float)x[c] - mean) * rstd, s2);
  }
  s1 = block_sum(s1, red) / C;
  s2 = block_sum(s2, red) / C;
  for (int c = threadIdx.x; c < C; c += kThreads) {
    const float g = (float)dy[c] * param(a.w, a.p_f32, c, 1.0f);
    dx[c] = (X)(rstd * (g - s1 - ((float)x[c] - mean) * rstd * s2));
  }
}
// Column sums over one run of rows.
template <class X>
__global__ __launch_bounds__(kThreads) void norm_wide_columns_kernel(NormArgs a) {
  const int c = blockIdx.x * kThreads + threadIdx.x, C = a.cols;
  if (c >= C) return;
  const int per = (a.rows + a.groups - 1) / a.groups;
  const int r0 = blockIdx.y * per, r1 = min(a.rows, r0 + per);
  float sw = 0.0f, sb = 0.0f;
#pragma unroll 4
  for (int r = r0; r < r1; ++r) {
    const float d = (float)((const X*)a.dout)[r * a.dout_stride + c];
    sw = fmaf(d, ((float)((const X*)a.x)[r * a.stride + c] - a.mean[r]) * a.rstd[r], sw);
    sb += d;
  }
  a.part[(size_t)blockIdx.y * C + c] = sw;
  a.part[((size_t)a.groups + blockIdx.y) * C + c] = sb;
}

// dw (blockIdx.y = 0) and db from the workgroups' sums: 64 columns a workgroup, 16 runs of groups.
__global__ __launch_bounds__(1024) void norm_reduce_kernel(NormArgs a) {
  void* out = blockIdx.y ? a.db : a.dw;
  if (!out) return;
  __shared__ float sum[16][64];
  const int c = blockIdx.x * 64 + (threadIdx.x & 63), run = threadIdx.x >> 6;
  const int per = (a.groups + 15) / 16, g1 = min(a.groups, (run + 1) * per);
  const float* p = a.part + (size_t)blockIdx.y * a.groups * a.cols + c;
  float s = 0.0f;
  if (c < a.cols) {
#pragma unroll 8
    for (int g = run * per; g < g1; ++g) s += p[(size_t)g * a.cols];
  }
  sum[run][threadIdx.x & 63] = s;
  __syncthreads();
  if (run == 0 && c < a.cols) {
    s = 0.0f;
    for (int i = 0; i < 16; ++i) s += sum[i][threadIdx.x];
    if (a.p_f32)
      ((float*)out)[c] = s;
    else
      ((__bf16*)out)[c] = (__bf16)s;
  }
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Calls go(X{}, VE, EPT, TPR) with the constants of the least form that holds a row.
template <class X, class F>
void pick(int cols, bool vec, F go) {
  constexpr int V = 16 / sizeof(X);
  auto width = [&](auto ve) {
    using std::integral_constant;
    if (cols <= 512)
      go(X{}, ve, integral_constant<int, 8>{}, integral_constant<int, 64>{});
    else if (cols <= 1024)
      go(X{}, ve, integral_constant<int, 16>{}, integral_constant<int, 64>{});
    else if (cols <= kWaveCols)
      go(X{}, ve, integral_constant<int, 24>{}, integral_constant<int, 64>{});
    else if (cols <= 2048)
      go(X{}, ve, integral_constant<int, 8>{}, integral_constant<int, 256>{});
    else if (cols <= 4096)
      go(X{}, ve, integral_constant<int, 16>{}, integral_constant<int, 256>{});
    else if (cols <= 6144)
      go(X{}, ve, integral_constant<int, 24>{}, integral_constant<int, 256>{});
    else
      go(X{}, ve, integral_constant<int, 8>{}, integral_constant<int, 1024>{});
  };
  if (vec)
    width(std::integral_constant<int, V>{});
  else
    width(std::integral_constant<int, 1>{});
}

// Workgroups of a launch over rows (four rows a workgroup up to kWaveCols columns), at most as many as
// 256 compute units hold at once by the registers of the form (see pick), or fewer: a second round would
// load the weights again and wait for its rows anew. Forward, 57,856 x 1,536 in bf16: 81.8 us at 1,024, 82.3 at
// 2,048, 111 at 4,096; 20,000 x 4,096 69.5, 75.4, 93.8. Backward with the forward, 100,000 x 512: 113 us at 1,024,
// 119 at 768, 137 at 512; 57,856 x 1,536 213, 229, 202; 20,000 x 4,096 218, 192, 195.
int row_groups(int64_t rows, int cols, bool backward) {
  const int most = cols > 6144                                  ? (backward ? 256 : 512)
                   : cols <= 512 || (cols > 1536 && cols <= 2048) ? (backward ? 1024 : 2048)
                   : cols <= 1024 || (cols > 1536 && cols <= 4096) ? (backward ? 768 : 1024)
                                                                  : (backward ? 512 : 1024);
  return (int)std::min<int64_t>(most, cols <= kWaveCols ? (rows + 3) / 4 : rows);
}

}  // namespace

int64_t norm_max_rows(int cols) { return cols > kBlockCols ? (((int64_t)1 << 32) - 1) / kThreads : (int64_t)1 << 30; }

int norm_groups(int64_t rows, int cols) {
  if (cols > kBlockCols) return (int)std::max<int64_t>(1, std::min<int64_t>(256, rows / 16));
  return row_groups(rows, cols, true);
}

hipError_t launch_norm_fwd(const NormArgs& a, hipStream_t s) {
  const dim3 block(kThreads);
  if (a.cols > kBlockCols) {
    if (a.x_f32)
      hipLaunchKernelGGL(norm_wide_fwd_kernel<float>, dim3(a.rows), block, 0, s, a);
    else
      hipLaunchKernelGGL(norm_wide_fwd_kernel<__bf16>, dim3(a.rows), block, 0, s, a);
    return hipGetLastError();
  }
  const int size = a.x_f32 ? 4 : 2, per = 16 / size;
  const bool vec = a.cols % per == 0 && a.stride % per == 0 && aligned16(a.x) && aligned16(a.y);
  auto go = [&](auto x, auto ve, auto ept, auto tpr) {
    hipLaunchKernelGGL((norm_fwd_kernel<decltype(x), decltype(ve)::value, decltype(ept)::value, decltype(tpr)::value>),
                       dim3(row_groups(a.rows, a.cols, false)), dim3(kWg<decltype(tpr)::value>), 0, s, a);
  };
  if (a.x_f32)
    pick<float>(a.cols, vec, go);
  else
    pick<__bf16>(a.cols, vec, go);
  return hipGetLastError();
}

hipError_t launch_norm_bwd(const NormArgs& a, hipStream_t s) {
  const dim3 block(kThreads);
  if (a.cols > kBlockCols) {
    const dim3 columns((a.cols + kThreads - 1) / kThreads, a.groups);
    if (a.x_f32)
      hipLaunchKernelGGL(norm_wide_dx_kernel<float>, dim3(a.rows), block, 0, s, a);
    else
      hipLaunchKernelGGL(norm_wide_dx_kernel<__bf16>, dim3(a.rows), block, 0, s, a);
    if (a.dw || a.db) {
      if (a.x_f32)
        hipLaunchKernelGGL(norm_wide_columns_kernel<float>, columns, block, 0, s, a);
      else
        hipLaunchKernelGGL(norm_wide_columns_kernel<__bf16>, columns, block, 0, s, a);
    }
  } else {
    const int size = a.x_f32 ? 4 : 2, per = 16 / size;
    const bool vec = a.cols % per == 0 && a.stride % per == 0 && a.dout_stride % per == 0 && aligned16(a.x) && aligned16(a.dout) &&
                     aligned16(a.dx);
    auto go = [&](auto x, auto ve, auto ept, auto tpr) {
      hipLaunchKernelGGL((norm_bwd_kernel<decltype(x), decltype(ve)::value, decltype(ept)::value, decltype(tpr)::value>),
                         dim3(a.groups), dim3(kWg<decltype(tpr)::value>), 0, s, a);
    };
    if (a.x_f32)
      pick<float>(a.cols, vec, go);
    else
      pick<__bf16>(a.cols, vec, go);
  }
  if (a.dw || a.db) hipLaunchKernelGGL(norm_reduce_kernel, dim3((a.cols + 63) / 64, 2), dim3(1024), 0, s, a);
  return hipGetLastError();
}

}  // namespace vcja
