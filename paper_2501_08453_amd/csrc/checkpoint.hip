// Checkpoints in 8 bits for gfx950: x to whole steps of a scale for each 128 columns of a row, and back.
//
// Bound by memory: 2 or 4 bytes an element on one side, 1 + 1/32 on the other. 16 lanes hold a block, eight columns each, so that its largest value
// is found by four steps within a row of DPP lanes.
#include "checkpoint.hpp"

#include <algorithm>

#include "rows.hpp"

namespace vcja {
namespace {

constexpr int kThreads = 256;

template <class X>
__global__ __launch_bounds__(kThreads) void checkpoint_pack_kernel(CheckpointArgs a) {
  const int64_t all = a.rows * a.blocks;
  const int lane = threadIdx.x & 15;
  for (int64_t b = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> 4; b < all; b += (int64_t)gridDim.x * (kThreads / 16)) {
    const int64_t row = b / a.blocks;
    const int col = (int)(b - row * a.blocks) * kBlockOf8 + lane * 8, n = a.cols - col;
    Eight<X> r;
    load8(r, (const X*)a.x + row * a.stride + col, n);
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = r[e];
    const Kept k = keep8(x);
    store_q8(a.q + row * a.cols + col, k.q, n);
    if (lane == 0) a.scales[b] = k.scale;
  }
}

template <class X>
__global__ __launch_bounds__(kThreads) void checkpoint_unpack_kernel(CheckpointArgs a) {
  const int64_t all = a.rows * a.blocks;
  const int lane = threadIdx.x & 15;
  for (int64_t b = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> 4; b < all; b += (int64_t)gridDim.x * (kThreads / 16)) {
    const int64_t row = b / a.blocks;
    const int col = (int)(b - row * a.blocks) * kBlockOf8 + lane * 8, n = a.cols - col;
    Eight<int8_t> r;
    load8(r, (const int8_t*)a.q + row * a.cols + col, n);
    const float scale = a.scales[b];
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = r[e] * scale;
    store8((X*)a.y + row * a.cols + col, x, n);
  }
}

int groups(const CheckpointArgs& a) {
  return (int)std::min<int64_t>(2048, (a.rows * a.blocks + kThreads / 16 - 1) / (kThreads / 16));
}

}  // namespace

hipError_t launch_checkpoint_pack(const CheckpointArgs& a, hipStream_t s) {
  if (a.f32)
    hipLaunchKernelGGL(checkpoint_pack_kernel<float>, dim3(groups(a)), dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL(checkpoint_pack_kernel<__bf16>, dim3(groups(a)), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_checkpoint_unpack(const CheckpointArgs& a, hipStream_t s) {
  if (a.f32)
    hipLaunchKernelGGL(checkpoint_unpack_kernel<float>, dim3(groups(a)), dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL(checkpoint_unpack_kernel<__bf16>, dim3(groups(a)), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace vcja
