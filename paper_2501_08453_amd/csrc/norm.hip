// Layer norm for gfx950, forward and backward: y = (x - mean) rstd w + b over the columns of
// each row, rstd = 1 / sqrt(mean of (x - mean)^2 + eps). Sums in fp32, the variance of the
// differences to the mean (never as a difference of squares, which cancels far from 0).
#include "norm.hpp"

#include <algorithm>

namespace vcja {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float block_sum(float x, float* red) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  x = red[0];
#pragma unroll
  for (int i = 1; i < kThreads / 64; ++i) x += red[i];
  return x;
}

template <class X, class P>
__global__ __launch_bounds__(kThreads) void norm_fwd_kernel(NormArgs a) {
  __shared__ float red[kThreads / 64];
  const int row = blockIdx.x, C = a.cols;
  const X* x = (const X*)a.x + row * a.stride;
  X* y = (X*)a.y + (int64_t)row * C;
  const P *w = (const P*)a.w, *b = (const P*)a.b;
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
    y[c] = (X)fmaf(((float)x[c] - mean) * rstd, w ? (float)w[c] : 1.0f, b ? (float)b[c] : 0.0f);
  if (threadIdx.x == 0) {
    a.mean[row] = mean;
    a.rstd[row] = rstd;
  }
}

template <class X, class P>
__global__ __launch_bounds__(kThreads) void norm_dx_kernel(NormArgs a) {
  __shared__ float red[kThreads / 64];
  const int row = blockIdx.x, C = a.cols;
  const X* x = (const X*)a.x + row * a.stride;
  const X* dy = (const X*)a.dout + row * a.dout_stride;
  X* dx = (X*)a.dx + (int64_t)row * C;
  const P* w = (const P*)a.w;
  const float mean = a.mean[row], rstd = a.rstd[row];
  float s1 = 0.0f, s2 = 0.0f;
  for (int c = threadIdx.x; c < C; c += kThreads) {
    const float g = (float)dy[c] * (w ? (float)w[c] : 1.0f);
    s1 += g;
    s2 = fmaf(g, ((float)x[c] - mean) * rstd, s2);
  }
  s1 = block_sum(s1, red) / C;
  s2 = block_sum(s2, red) / C;
  for (int c = threadIdx.x; c < C; c += kThreads) {
    const float g = (float)dy[c] * (w ? (float)w[c] : 1.0f);
    dx[c] = (X)(rstd * (g - s1 - ((float)x[c] - mean) * rstd * s2));
  }
}

// Column sums of dout xhat and of dout over one run of rows.
template <class X>
__global__ __launch_bounds__(kThreads) void norm_columns_kernel(NormArgs a) {
  const int c = blockIdx.x * kThreads + threadIdx.x, C = a.cols;
  if (c >= C) return;
  const int per = (a.rows + a.groups - 1) / a.groups;
  const int r0 = blockIdx.y * per, r1 = min(a.rows, r0 + per);
  float sw = 0.0f, sb = 0.0f;
  for (int r = r0; r < r1; ++r) {
    const float d = (float)((const X*)a.dout)[r * a.dout_stride + c];
    sw = fmaf(d, ((float)((const X*)a.x)[r * a.stride + c] - a.mean[r]) * a.rstd[r], sw);
    sb += d;
  }
  a.part[(size_t)blockIdx.y * C + c] = sw;
  a.part[((size_t)a.groups + blockIdx.y) * C + c] = sb;
}

template <class P>
__global__ __launch_bounds__(kThreads) void norm_reduce_kernel(NormArgs a) {
  const int c = blockIdx.x * kThreads + threadIdx.x;
  if (c >= a.cols) return;
  P* out = (P*)(blockIdx.y ? a.db : a.dw);
  if (!out) return;
  float s = 0.0f;
  for (int g = 0; g < a.groups; ++g) s += a.part[((size_t)blockIdx.y * a.groups + g) * a.cols + c];
  out[c] = (P)s;
}

}  // namespace

int norm_groups(int64_t rows, int /*cols*/) { return (int)std::max<int64_t>(1, std::min<int64_t>(256, rows / 16)); }

hipError_t launch_norm_fwd(const NormArgs& a, hipStream_t s) {
  const dim3 grid(a.rows), block(kThreads);
  if (a.x_f32 && a.p_f32)
    hipLaunchKernelGGL((norm_fwd_kernel<float, float>), grid, block, 0, s, a);
  else if (a.x_f32)
    hipLaunchKernelGGL((norm_fwd_kernel<float, __bf16>), grid, block, 0, s, a);
  else if (a.p_f32)
    hipLaunchKernelGGL((norm_fwd_kernel<__bf16, float>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((norm_fwd_kernel<__bf16, __bf16>), grid, block, 0, s, a);
  return hipGetLastError();
}

hipError_t launch_norm_bwd(const NormArgs& a, hipStream_t s) {
  const dim3 grid(a.rows), block(kThreads);
  if (a.x_f32 && a.p_f32)
    hipLaunchKernelGGL((norm_dx_kernel<float, float>), grid, block, 0, s, a);
  else if (a.x_f32)
    hipLaunchKernelGGL((norm_dx_kernel<float, __bf16>), grid, block, 0, s, a);
  else if (a.p_f32)
    hipLaunchKernelGGL((norm_dx_kernel<__bf16, float>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((norm_dx_kernel<__bf16, __bf16>), grid, block, 0, s, a);
  if (a.dw || a.db) {
    const int cb = (a.cols + kThreads - 1) / kThreads;
    if (a.x_f32)
      hipLaunchKernelGGL(norm_columns_kernel<float>, dim3(cb, a.groups), block, 0, s, a);
    else
      hipLaunchKernelGGL(norm_columns_kernel<__bf16>, dim3(cb, a.groups), block, 0, s, a);
    if (a.p_f32)
      hipLaunchKernelGGL(norm_reduce_kernel<float>, dim3(cb, 2), block, 0, s, a);
    else
      hipLaunchKernelGGL(norm_reduce_kernel<__bf16>, dim3(cb, 2), block, 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace vcja
