// Checkpoints in 8 bits for gfx950: x to whole steps of a scale for each 128 columns of a row, and back.
//
// Bound by memory: 2 or 4 bytes an element on one side, 1 + 1/32 on the other. 16 lanes hold a block, eight columns each (fp32: 32 lanes, four), so that
// its largest value is found by four steps within a row of DPP lanes.
#include "checkpoint.hpp"

#include <algorithm>
#include <type_traits>

#include "rows.hpp"

namespace vcja {
namespace {

constexpr int kThreads = 256;
template <class X>
constexpr int kCols = sizeof(X) == 2 ? 8 : 4;  // of a thread
template <class X>
constexpr int kLanes = kBlockOf8 / kCols<X>;   // of a block of 128 columns

template <class X, bool ONCE>
__global__ __launch_bounds__(kThreads) void checkpoint_pack_kernel(CheckpointArgs a) {
  constexpr int N = kCols<X>, L = kLanes<X>;
  const int64_t all = a.rows * a.blocks;
  const int lane = threadIdx.x % L;
  for (int64_t b = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / L; b < all; b += (int64_t)gridDim.x * (kThreads / L)) {
    const int64_t row = b / a.blocks;
    const Span<N> s = span_at<N>((int)(b - row * a.blocks) * kBlockOf8 + lane * N, a.cols);
    Cols<X, N> r;
    load_cols<true, ONCE>(r, (const X*)a.x + row * a.stride, s);
    float x[N];
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = s.has(e) ? r[e] : 0.0f;
    const Kept<N> k = keep<N>(x);
    store_kept(a.q + row * a.cols, k, s);
    if (lane == 0) a.scales[b] = k.scale;
  }
}

template <class X, bool ONCE>
__global__ __launch_bounds__(kThreads) void checkpoint_unpack_kernel(CheckpointArgs a) {
  constexpr int N = kCols<X>, L = kLanes<X>;
  const int64_t all = a.rows * a.blocks;
  const int lane = threadIdx.x % L;
  for (int64_t b = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / L; b < all; b += (int64_t)gridDim.x * (kThreads / L)) {
    const int64_t row = b / a.blocks;
    const Span<N> s = span_at<N>((int)(b - row * a.blocks) * kBlockOf8 + lane * N, a.cols);
    Cols<int8_t, N> r;
    load_cols(r, (const int8_t*)a.q + row * a.cols, s);
    const float scale = a.scales[b];
    float x[N];
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = r[e] * scale;
    store_cols<true, ONCE>((X*)a.y + row * a.cols, x, s);
  }
}

int groups(const CheckpointArgs& a) {
  const int of = kThreads / (a.f32 ? kLanes<float> : kLanes<__bf16>);
  return (int)std::min<int64_t>(2048, (a.rows * a.blocks + of - 1) / of);
}

// Whether x (y) goes past the caches, as it is more than half of what the last one holds: the 8 bits may stay there. 1,388,544 x 128 bf16:
// pack 109 us so and 127 otherwise, unpack 81 and 91.
bool once(const CheckpointArgs& a) { return a.rows * a.cols * (a.f32 ? 4 : 2) > ((int64_t)128 << 20); }

// Calls go(X{}, past the caches).
template <class F>
void typed(const CheckpointArgs& a, F go) {
  auto with = [&](auto x) {
    if (once(a))
      go(x, std::true_type{});
    else
      go(x, std::false_type{});
  };
  if (a.f32)
    with(float{});
  else
    with(__bf16{});
}

}  // namespace

hipError_t launch_checkpoint_pack(const CheckpointArgs& a, hipStream_t s) {
  typed(a, [&](auto x, auto past) {
    hipLaunchKernelGGL((checkpoint_pack_kernel<decltype(x), decltype(past)::value>), dim3(groups(a)), dim3(kThreads), 0, s, a);
  });
  return hipGetLastError();
}

hipError_t launch_checkpoint_unpack(const CheckpointArgs& a, hipStream_t s) {
  typed(a, [&](auto x, auto past) {
    hipLaunchKernelGGL((checkpoint_unpack_kernel<decltype(x), decltype(past)::value>), dim3(groups(a)), dim3(kThreads), 0, s, a);
  });
  return hipGetLastError();
}

}  // namespace vcja
