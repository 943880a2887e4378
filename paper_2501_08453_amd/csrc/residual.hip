// Gated residual with the norms before and after a block for gfx950, forward and backward. Of each row, with the
// vectors gate, scale and shift of its sample,
//   h = c x + gate P(a), y = N(h) (1 + scale) + shift,
// P and N a layer norm, an RMS norm or nothing. Backward, with xh = N(h), xa = P(a) before its weight wp, e = 1 + scale,
// r and ra the reciprocal deviations of h and a:
//   G = dy e, H = dh + r (G - mean G - xh mean(G xh)), dx = c H,
//   K = H gate wp, da = ra (K - mean K - xa mean(K xa)),
//   sums over a sample's rows: A = H xa, dscale = dy xh, dshift = dy; dgate = wp A, dwp = the sum over samples of gate A.
// (An RMS norm has no terms of the mean; without P, da = H gate.) A serves two gradients, as wp is the same in all rows
// and gate in all rows of a sample.
//
// Bound by memory: a thread holds eight columns of a row, a workgroup a run of rows one behind the other, so that
// parameters are loaded once a sample and the column sums stay in its registers. Each run's sums of
// each sample go to a row of their own, run + sample, which is free for every pair that occurs as both only grow; a
// second kernel adds them in order. No atomics. 57,856 x 1,536 bf16: forward 142 us (5.0 TB/s), backward 208 (5.1) and 6 for the sums, as a
// copy of 1 GiB does; with h and a kept in 8 bits 195 and 196.
#include "residual.hpp"

#include <algorithm>
#include <type_traits>

#include "rows.hpp"
#include "vc_jointattn.h"

namespace vcja {
namespace {

// A run of rows that belong to one sample, or to none.
struct Piece {
  int sample, end;
  bool live, outside;
};
// The piece that begins with row r of a chunk ending at r1. Whatever the arrays hold, it is of one row at least
// and its sample exists. Every lane of a wave calls it: 64 offsets a step are looked at, one or two steps for most batches.
__device__ __forceinline__ Piece piece_at(const ResidualArgs& a, int r, int r1) {
  int s, b, e;  // sample, and its slot
  if (a.cu) {
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = a.samples;  // the first sample whose slot ends behind r is one of these, or `samples` if none is
    while (lo < hi) {
      const int step = (hi - lo + 63) >> 6, m = lo + lane * step + step - 1;
      const uint64_t behind = __ballot(a.cu[min(m, hi - 1) + 1] > r);
      if (!behind) {
        lo = hi;
        break;
      }
      const int at = lo + (__ffsll((unsigned long long)behind) - 1) * step;  // of this step's samples, the last is behind
      lo = min(at, hi - 1);
      hi = min(at + step - 1, hi - 1);
    }
    s = lo;
    if (s == a.samples) return Piece{a.samples - 1, r1, false, true};
    b = a.cu[s];
    e = a.cu[s + 1];
    if (b > r) return Piece{s, min(b, r1), false, true};
  } else {
    s = r / a.per;
    b = s * a.per;
    e = b + a.per;
  }
  if (a.lens) {
    const int n = min(max(a.lens[s], 0), e - b);
    if (r >= b + n) return Piece{s, min(max(e, r + 1), r1), false, false};
    e = b + n;
  }
  return Piece{s, min(max(e, r + 1), r1), true, false};
}

// Sums over the `waves` waves of a row of N values a thread, the same in every thread. red: two buffers in turn, so that one
// barrier a call is enough: a buffer is written again only behind the barrier of the call between. first: the row's first wave.
template <int N, int W>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*red)[W][N], int& turn, int first, int waves) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
  if (waves == 1) return;
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) red[turn][threadIdx.x >> 6][i] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = 0.0f;
  for (int w = first; w < first + waves; ++w)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += red[turn][w][i];
  turn ^= 1;
}

__device__ __forceinline__ const void* at_sample(const void* p, bool f32, int64_t stride, int s) {
  return !p ? p : f32 ? (const void*)((const float*)p + stride * s) : (const void*)((const __bf16*)p + stride * s);
}

// Columns of a thread's vector, by the types of the stream and of the block.
template <class X, class Y>
constexpr int kCols = sizeof(X) == 2 || sizeof(Y) == 2 ? 8 : 4;
// The columns of thread t of a row's `across`: V vectors.
template <int N, int V>
__device__ __forceinline__ void spans_of(Span<N>* s, int t, int across, int C) {
#pragma unroll
  for (int v = 0; v < V; ++v) s[v] = span_at<N>((v * across + t) * N, C);
}
template <bool ODD, int N, int V>
__device__ __forceinline__ void params(float* out, const void* p, bool f32, int64_t stride, int sample, const Span<N>* s, float other) {
  p = at_sample(p, f32, stride, sample);
#pragma unroll
  for (int v = 0; v < V; ++v) load_param<ODD>(out + N * v, p, f32, s[v], other);
}

// Waves a SIMD: not more than a launch has workgroups for (residual_groups), or some compute units would get one more of them
// and others one less.
constexpr int kFwdWaves = 4;

// A thread has eight columns. FEW: up to 2,048 columns, two rows a step where
// registers allow it (128).
template <class X, class Y, bool POST, bool ODD, bool ONCE, bool FEW>
__global__ __launch_bounds__(FEW ? 256 : 1024) __attribute__((amdgpu_waves_per_eu(kFwdWaves, kFwdWaves))) void residual_fwd_kernel(ResidualArgs a) {
  constexpr int N = kCols<X, Y>, V = 8 / N, W = 8, R = FEW && !(POST && N == 4) ? 2 : 1;
  __shared__ float red[2][FEW ? 4 : 16][R];
  int turn = 0;
  const int C = a.cols, waves = blockDim.x >> 6, t = threadIdx.x;
  Span<N> sp[V];
  spans_of<N, V>(sp, t, blockDim.x, C);
  const float inv = 1.0f / C;
  const int r1 = min(a.rows, ((int)blockIdx.x + 1) * a.chunk), blocks = (C + kBlockOf8 - 1) / kBlockOf8;
  // The 8-bit form of a row's x: the first lane of each block of 128 columns writes the scale.
  auto keep_row = [&](int8_t* q, float* scales, int64_t row, const float* x) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const Kept<N> k = keep<N>(x + N * v);
      store_kept<ODD>(q + row * C, k, sp[v]);
      const int c = (v * (int)blockDim.x + t) * N;
      if ((c & 127) == 0 && c < C) scales[row * blocks + (c >> 7)] = k.scale;
    }
  };
  for (int r = blockIdx.x * a.chunk; r < r1;) {
    Cols<X, N> x[R][V];
    Cols<Y, N> b[R][V];
    auto load = [&]() {
#pragma unroll
      for (int j = 0; j < R; ++j) {
        const int64_t row = min(r + j, r1 - 1);
#pragma unroll
        for (int v = 0; v < V; ++v) {
          load_cols<ODD, ONCE>(x[j][v], (const X*)a.x + row * a.x_stride, sp[v]);
          if (a.a) load_cols<ODD, ONCE>(b[j][v], (const Y*)a.a + row * a.a_stride, sp[v]);
        }
      }
    };
    load();  // in flight while the sample is looked up
    const Piece p = piece_at(a, r, r1);
    if (!p.live) {
      if (!p.outside || a.clear) {
        const float zero[N] = {};
        for (; r < p.end; ++r)
#pragma unroll
          for (int v = 0; v < V; ++v) {
            if (a.h) store_cols<ODD>((X*)a.h + (int64_t)r * C, zero, sp[v]);
            if (a.y) store_cols<ODD>((Y*)a.y + (int64_t)r * C, zero, sp[v]);
          }
      }
      r = p.end;
      continue;
    }
    float g[W], e[W], f[W];  // g: gate, with P's weight where there is one
    params<ODD, N, V>(g, a.gate, a.p_f32, a.gate_stride, p.sample, sp, 1.0f);
    if constexpr (POST) {
      float w[W];
      params<ODD, N, V>(w, a.wp, a.p_f32, 0, 0, sp, 1.0f);
#pragma unroll
      for (int i = 0; i < W; ++i) g[i] *= w[i];
    }
    params<ODD, N, V>(e, a.scale, a.p_f32, a.scale_stride, p.sample, sp, a.plus_one ? 0.0f : 1.0f);
    params<ODD, N, V>(f, a.shift, a.p_f32, a.shift_stride, p.sample, sp, 0.0f);
    if (a.plus_one)
#pragma unroll
      for (int i = 0; i < W; ++i) e[i] += 1.0f;
    for (bool first = true; r < p.end; r += R, first = false) {
      const int m = min(R, p.end - r);
      float h[R][W], s[R], mean[R], rstd[R];
      if (!first) load();
      if (a.a8)
#pragma unroll
        for (int j = 0; j < R; ++j)
          if (j < m) {
            float u[W];
#pragma unroll
            for (int i = 0; i < W; ++i) u[i] = own<ODD>(sp[i / N], i % N) ? b[j][i / N][i % N] : 0.0f;
            keep_row(a.a8, a.a8s, r + j, u);
          }
      if constexpr (POST) {
#pragma unroll
        for (int j = 0; j < R; ++j) mean[j] = 0.0f;
        if (a.post == VC_NORM_LAYER) {
#pragma unroll
          for (int j = 0; j < R; ++j) {
            s[j] = 0.0f;
#pragma unroll
            for (int i = 0; i < W; ++i) s[j] += own<ODD>(sp[i / N], i % N) ? b[j][i / N][i % N] : 0.0f;
          }
          row_sums(s, red, turn, 0, waves);
#pragma unroll
          for (int j = 0; j < R; ++j) mean[j] = s[j] * inv;
        }
#pragma unroll
        for (int j = 0; j < R; ++j) {
          s[j] = 0.0f;
#pragma unroll
          for (int i = 0; i < W; ++i) {
            const float d = b[j][i / N][i % N] - mean[j];
            s[j] = own<ODD>(sp[i / N], i % N) ? fmaf(d, d, s[j]) : s[j];
          }
        }
        row_sums(s, red, turn, 0, waves);
#pragma unroll
        for (int j = 0; j < R; ++j) {
          rstd[j] = 1.0f / sqrtf(fmaf(s[j], inv, a.eps));
          if (t == 0 && j < m) {
            a.pmean[r + j] = mean[j];
            a.prstd[r + j] = rstd[j];
          }
#pragma unroll
          for (int i = 0; i < W; ++i) h[j][i] = fmaf(g[i], (b[j][i / N][i % N] - mean[j]) * rstd[j], a.c * x[j][i / N][i % N]);
        }
      } else {
#pragma unroll
        for (int j = 0; j < R; ++j)
#pragma unroll
          for (int i = 0; i < W; ++i) {
            h[j][i] = a.c * x[j][i / N][i % N];
            if (a.a) h[j][i] = fmaf(g[i], b[j][i / N][i % N], h[j][i]);
          }
      }
#pragma unroll
      for (int j = 0; j < R; ++j) {
        // The norm takes h as it is kept: the next block and the backward read that, not the sum before its rounding.
#pragma unroll
        for (int i = 0; i < W; ++i) h[j][i] = own<ODD>(sp[i / N], i % N) ? (float)(X)h[j][i] : 0.0f;
        if (j < m) {
          if (a.h)
#pragma unroll
            for (int v = 0; v < V; ++v) store_cols<ODD, ONCE>((X*)a.h + (int64_t)(r + j) * C, h[j] + N * v, sp[v]);
          if (a.h8) keep_row(a.h8, a.h8s, r + j, h[j]);
        }
      }
      if (a.norm == VC_NORM_NONE) continue;
#pragma unroll
      for (int j = 0; j < R; ++j) mean[j] = 0.0f;
      if (a.norm == VC_NORM_LAYER) {
#pragma unroll
        for (int j = 0; j < R; ++j) {
          s[j] = 0.0f;
#pragma unroll
          for (int i = 0; i < W; ++i) s[j] += h[j][i];
        }
        row_sums(s, red, turn, 0, waves);
#pragma unroll
        for (int j = 0; j < R; ++j) mean[j] = s[j] * inv;
      }
#pragma unroll
      for (int j = 0; j < R; ++j) {
        s[j] = 0.0f;
#pragma unroll
        for (int i = 0; i < W; ++i) {
          h[j][i] -= mean[j];
          s[j] = own<ODD>(sp[i / N], i % N) ? fmaf(h[j][i], h[j][i], s[j]) : s[j];
        }
      }
      row_sums(s, red, turn, 0, waves);
#pragma unroll
      for (int j = 0; j < R; ++j) {
        rstd[j] = 1.0f / sqrtf(fmaf(s[j], inv, a.eps));
        if (j >= m) break;
        if (t == 0) {
          a.mean[r + j] = mean[j];
          a.rstd[r + j] = rstd[j];
        }
        float y[W];
#pragma unroll
        for (int i = 0; i < W; ++i) y[i] = fmaf(h[j][i] * rstd[j], e[i], f[i]);
#pragma unroll
        for (int v = 0; v < V; ++v) store_cols<ODD, ONCE>((Y*)a.y + (int64_t)(r + j) * C, y + N * v, sp[v]);
      }
    }
    r = p.end;
  }
}

// Sources of h and a in the backward: as they are, or from 8 bits.
template <class X, class Y, bool K8>
struct From {
  typedef X H;
  typedef Y A;
};
template <class X, class Y>
struct From<X, Y, true> {
  typedef int8_t H;
  typedef int8_t A;
};

// The backward up to 2,048 columns (FEW): eight of them a thread, three waves a SIMD (168 registers). 57,856 x 1,536 through the caches, h and a
// read as they are: 227 us at three, 233 at two with two rows a step, 233 at four; from 8 bits 202, 225, 209. (The next row's loads
// in flight during this one: the same at three.) Wider rows: 16 columns a thread, two waves a SIMD (256
// registers, of which some forms spill up to 24).
constexpr int kBwdWaves = 3, kBwdThreads = 256, kWideThreads = 512;

template <class X, class Y, bool K8, bool POST, bool ODD, bool ONCE, bool FEW>
__global__ __launch_bounds__(FEW ? kBwdThreads : kWideThreads) __attribute__((amdgpu_waves_per_eu(FEW ? kBwdWaves : 2, FEW ? kBwdWaves : 2)))
void residual_bwd_kernel(ResidualArgs a, int across) {
  using HT = typename From<X, Y, K8>::H;
  using AT = typename From<X, Y, K8>::A;
  constexpr int N = kCols<X, Y>, W = FEW ? 8 : 16, V = W / N;
  __shared__ float red[2][(FEW ? kBwdThreads : kWideThreads) / 64][2];
  constexpr int kOthers = 192;  // threads of all rows of a step but the first, at most
  __shared__ float comb[FEW ? 24 * kOthers : 1];
  int turn = 0;
  // `across` threads a row; the workgroup's rows of a step one behind the other
  const int abreast = FEW ? blockDim.x / across : 1, which = FEW ? __builtin_amdgcn_readfirstlane(threadIdx.x / across) : 0;
  const int t = threadIdx.x - which * across, waves = across >> 6, first = which * waves;
  const int C = a.cols;
  Span<N> sp[V];
  spans_of<N, V>(sp, t, across, C);
  int block[V];  // of 128 columns, whose scale in 8 bits is this vector's
#pragma unroll
  for (int v = 0; v < V; ++v) block[v] = min((v * across + t) * N, C - 1) >> 7;
  const float inv = 1.0f / C, inv1 = a.norm == VC_NORM_LAYER ? inv : 0.0f, pinv1 = a.post == VC_NORM_LAYER ? inv : 0.0f;
  const int r1 = min(a.rows, ((int)blockIdx.x + 1) * a.chunk), blocks = (C + kBlockOf8 - 1) / kBlockOf8;
  const HT* hp = K8 ? (const HT*)a.h8 : (const HT*)a.h_in;
  const AT* ap = K8 ? (const AT*)a.a8 : (const AT*)a.a;
  const int64_t h_stride = K8 ? C : a.h_stride, a_stride = K8 ? C : a.a_stride;
  const bool has_a = ap != nullptr, has_norm = a.norm != VC_NORM_NONE && a.dy;
  float sa[W] = {}, se[W] = {}, sf[W] = {};
  // This run's sums to the row `to` of the partials: those of the rows abreast added in order.
  auto flush = [&](int64_t to) {
    if constexpr (FEW) {
      if (abreast > 1) {
        const int at = threadIdx.x - across;
        __syncthreads();
        if (which)
#pragma unroll
          for (int i = 0; i < W; ++i) {
            comb[i * kOthers + at] = sa[i];
            comb[(8 + i) * kOthers + at] = se[i];
            comb[(16 + i) * kOthers + at] = sf[i];
          }
        __syncthreads();
        if (!which)
          for (int k = 0; k < abreast - 1; ++k)
#pragma unroll
            for (int i = 0; i < W; ++i) {
              sa[i] += comb[i * kOthers + k * across + t];
              se[i] += comb[(8 + i) * kOthers + k * across + t];
              sf[i] += comb[(16 + i) * kOthers + k * across + t];
            }
      }
    }
    if (!which) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float* out = a.part + to * 3 * C;
        store_cols<ODD>(out, sa + N * v, sp[v]);
        store_cols<ODD>(out + C, se + N * v, sp[v]);
        store_cols<ODD>(out + 2 * C, sf + N * v, sp[v]);
      }
    }
#pragma unroll
    for (int i = 0; i < W; ++i) sa[i] = se[i] = sf[i] = 0.0f;
  };
  for (int r = blockIdx.x * a.chunk; r < r1;) {
    Cols<X, N> dh[V] = {};
    Cols<Y, N> dy[V];
    Cols<HT, N> h[V];
    Cols<AT, N> b[V];
    float hs[V], as[V], mean, rstd, pmean, prstd;
    auto load = [&](int r) {
      const int64_t row = min(r + which, r1 - 1);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        hs[v] = as[v] = 1.0f;
        if (a.dh) load_cols<ODD, ONCE>(dh[v], (const X*)a.dh + row * a.dh_stride, sp[v]);
        if (has_norm) {
          load_cols<ODD, ONCE>(dy[v], (const Y*)a.dy + row * a.dy_stride, sp[v]);
          load_cols<ODD, ONCE>(h[v], hp + row * h_stride, sp[v]);
          if (K8) hs[v] = a.h8s[row * blocks + block[v]];
        }
        if (has_a) {
          load_cols<ODD, ONCE>(b[v], ap + row * a_stride, sp[v]);
          if (K8) as[v] = a.a8s[row * blocks + block[v]];
        }
      }
      mean = pmean = 0.0f;
      if (has_norm) {
        if (a.norm == VC_NORM_LAYER) mean = a.mean[row];
        rstd = a.rstd[row];
      }
      if constexpr (POST) {
        if (a.post == VC_NORM_LAYER) pmean = a.pmean[row];
        prstd = a.prstd[row];
      }
    };
    load(r);  // in flight while the sample is looked up
    const Piece p = piece_at(a, r, r1);
    if (!p.live && (!p.outside || a.clear)) {
      const float zero[N] = {};
      for (int row = r + which; row < p.end; row += abreast)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          if (a.dx) store_cols<ODD>((X*)a.dx + (int64_t)row * C, zero, sp[v]);
          if (a.da) store_cols<ODD>((Y*)a.da + (int64_t)row * C, zero, sp[v]);
        }
    }
    if (!p.live) r = p.end;
    float g[W], e[W];  // g: gate, with P's weight where there is one
    auto gates = [&]() {
      params<ODD, N, V>(g, a.gate, a.p_f32, a.gate_stride, p.sample, sp, 1.0f);
      if constexpr (POST) {
        float w[W];
        params<ODD, N, V>(w, a.wp, a.p_f32, 0, 0, sp, 1.0f);
#pragma unroll
        for (int i = 0; i < W; ++i) g[i] *= w[i];
      }
    };
    auto scales = [&]() {
      params<ODD, N, V>(e, a.scale, a.p_f32, a.scale_stride, p.sample, sp, a.plus_one ? 0.0f : 1.0f);
      if (a.plus_one)
#pragma unroll
        for (int i = 0; i < W; ++i) e[i] += 1.0f;
    };
    gates();
    scales();
    for (; r < p.end; r += abreast) {
      const bool mine = r + which < p.end;  // else this row is the next sample's, or none
      const int64_t row = r + which;
      float H[W], s[2];
      if (has_norm) {
        s[0] = s[1] = 0.0f;
#pragma unroll
        for (int i = 0; i < W; ++i) {
          const float d = own<ODD>(sp[i / N], i % N) ? dy[i / N][i % N] : 0.0f, xh = (h[i / N][i % N] * hs[i / N] - mean) * rstd;
          const float G = d * e[i];
          s[0] += G;
          s[1] = fmaf(G, xh, s[1]);
          if (mine) {
            se[i] = fmaf(d, xh, se[i]);
            sf[i] += d;
          }
        }
        row_sums(s, red, turn, first, waves);
        const float m1 = s[0] * inv1, m2 = s[1] * inv;
#pragma unroll
        for (int i = 0; i < W; ++i) {
          const float xh = (h[i / N][i % N] * hs[i / N] - mean) * rstd;
          H[i] = fmaf(rstd, fmaf(dy[i / N][i % N], e[i], -m1) - xh * m2, dh[i / N][i % N]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < W; ++i) H[i] = dh[i / N][i % N];
      }
      float o[W];
#pragma unroll
      for (int i = 0; i < W; ++i) {
        H[i] = own<ODD>(sp[i / N], i % N) ? H[i] : 0.0f;
        o[i] = a.c * H[i];
      }
      if (mine && a.dx)
#pragma unroll
        for (int v = 0; v < V; ++v) store_cols<ODD, ONCE>((X*)a.dx + row * C, o + N * v, sp[v]);
      if constexpr (POST) {
        s[0] = s[1] = 0.0f;
#pragma unroll
        for (int i = 0; i < W; ++i) {
          const float xa = (b[i / N][i % N] * as[i / N] - pmean) * prstd, K = H[i] * g[i];
          s[0] += K;
          s[1] = fmaf(K, xa, s[1]);
          if (mine) sa[i] = fmaf(H[i], xa, sa[i]);
        }
        row_sums(s, red, turn, first, waves);
        const float m1 = s[0] * pinv1, m2 = s[1] * inv;
#pragma unroll
        for (int i = 0; i < W; ++i) {
          const float xa = (b[i / N][i % N] * as[i / N] - pmean) * prstd;
          o[i] = prstd * (fmaf(H[i], g[i], -m1) - xa * m2);
        }
      } else if (has_a) {
#pragma unroll
        for (int i = 0; i < W; ++i) {
          if (mine) sa[i] = fmaf(H[i], b[i / N][i % N] * as[i / N], sa[i]);
          o[i] = H[i] * g[i];
        }
      }
      if (mine && a.da)
#pragma unroll
        for (int v = 0; v < V; ++v) store_cols<ODD, ONCE>((Y*)a.da + row * C, o + N * v, sp[v]);
      if (r + abreast < p.end) load(r + abreast);
    }
    r = p.end;
    if (a.part && (a.flat ? r == r1 : p.live)) flush((int64_t)blockIdx.x + (a.flat ? 0 : p.sample));
  }
}

__device__ __forceinline__ float param(const void* p, bool f32, int64_t at, float other) {
  return !p ? other : f32 ? ((const float*)p)[at] : (float)((const __bf16*)p)[at];
}
__device__ __forceinline__ void write(void* p, bool f32, int64_t at, float x) {
  if (!p) return;
  if (f32)
    ((float*)p)[at] = x;
  else
    ((__bf16*)p)[at] = (__bf16)x;
}

// Columns of a workgroup that adds up sums, a line of them, and its shares a wave. 57,856 x 1,536: 6.4 us, with 16 columns 9.3, with 64 9.9.
constexpr int kSumCols = 32, kSumWave = 64 / kSumCols;

// Sums over the workgroup's shares of K values a thread, in order, for the threads of its first K shares each one. sum: [K] [waves][columns].
template <int K>
__device__ __forceinline__ float shares_sum(float (&v)[K], float (*sum)[16][kSumCols]) {
#pragma unroll
  for (int k = 0; k < K; ++k) {
#pragma unroll
    for (int o = kSumCols; o < 64; o <<= 1) v[k] += __shfl_xor(v[k], o, 64);
    if (threadIdx.y % kSumWave == 0) sum[k][threadIdx.y / kSumWave][threadIdx.x] = v[k];
  }
  __syncthreads();
  float s = 0.0f;
  if (threadIdx.y < K)
#pragma unroll 4
    for (int w = 0; w < (int)blockDim.y / kSumWave; ++w) s += sum[threadIdx.y][w][threadIdx.x];
  return s;
}

// One of the three sums of one sample from those of its runs, in order: blockDim.y shares of the runs a workgroup.
__global__ __launch_bounds__(1024) void residual_sample_kernel(ResidualArgs a) {
  __shared__ float sum[1][16][kSumCols];
  const int C = a.cols, across = (C + kSumCols - 1) / kSumCols, k = blockIdx.x % 3, at_s = blockIdx.x / 3;
  const int s = at_s / across, col = (at_s - s * across) * kSumCols + threadIdx.x;
  int b, e;
  if (a.flat) {
    b = 0;
    e = a.rows;
  } else if (a.cu) {
    b = min(max(a.cu[s], 0), a.rows);
    e = min(max(a.cu[s + 1], b), a.rows);
  } else {
    b = s * a.per;
    e = b + a.per;
  }
  if (a.lens && !a.flat) e = b + min(max(a.lens[s], 0), e - b);
  const int g0 = b / a.chunk, g1 = e > b ? (e - 1) / a.chunk + 1 : g0, share = (g1 - g0 + blockDim.y - 1) / blockDim.y;
  const int last = min(g1, g0 + ((int)threadIdx.y + 1) * share);
  float v[1] = {};
  if (col < C)
#pragma unroll 8
    for (int g = g0 + threadIdx.y * share; g < last; ++g) v[0] += a.part[(((int64_t)g + s) * 3 + k) * C + col];
  const float t = shares_sum(v, sum);
  if (col >= C || threadIdx.y) return;
  const int64_t at = (int64_t)s * C + col;
  const bool one = a.flat;
  if (a.sums) a.sums[((int64_t)s * 3 + k) * C + col] = t;
  if (k == 0) {
    if (a.gate_stride || one) write(a.dgate, a.p_f32, at, t * param(a.wp, a.p_f32, col, 1.0f));
    if (one) write(a.dwp, a.p_f32, col, t * param(a.gate, a.p_f32, col, 1.0f));
  } else if (k == 1) {
    if (a.scale_stride || one) write(a.dscale, a.p_f32, at, t);
  } else {
    if (a.shift_stride || one) write(a.dshift, a.p_f32, at, t);
  }
}

// What all samples share, from the samples' sums.
__global__ __launch_bounds__(1024) void residual_shared_kernel(ResidualArgs a) {
  __shared__ float sum[4][16][kSumCols];
  const int C = a.cols, col = blockIdx.x * kSumCols + threadIdx.x;
  const int share = (a.samples + blockDim.y - 1) / blockDim.y, last = min(a.samples, ((int)threadIdx.y + 1) * share);
  float v[4] = {};
  if (col < C)
#pragma unroll 2
    for (int s = threadIdx.y * share; s < last; ++s) {
      const float* p = a.sums + (int64_t)s * 3 * C + col;
      const float t = p[0];
      v[0] += t;
      v[1] += p[C];
      v[2] += p[2 * C];
      v[3] = fmaf(t, param(a.gate, a.p_f32, a.gate_stride * s + col, 1.0f), v[3]);
    }
  const float t = shares_sum(v, sum);
  if (col >= C) return;
  if (threadIdx.y == 0 && !a.gate_stride) write(a.dgate, a.p_f32, col, t * param(a.wp, a.p_f32, col, 1.0f));
  if (threadIdx.y == 1 && !a.scale_stride) write(a.dscale, a.p_f32, col, t);
  if (threadIdx.y == 2 && !a.shift_stride) write(a.dshift, a.p_f32, col, t);
  if (threadIdx.y == 3) write(a.dwp, a.p_f32, col, t);
}

constexpr int kFewCols = 2048;
// Whether a call reads and writes its rows past the caches, as these are more than the last one's 256 MiB: the backward, and a forward
// that keeps 8 bits, which then stay there for the backward. 57,856 x 1,536: backward 208 us so and 230 otherwise, with 8 bits 197
// and 230, their forward 198 and 203; a forward without them 147 so and 142 otherwise, and its backward 221 behind it instead of 208.
bool once_of(const ResidualArgs& a, bool backward) {
  const int64_t bytes = (int64_t)a.rows * a.cols * ((a.x_f32 ? 4 : 2) + (a.y_f32 ? 4 : 2)) * (backward ? 3 : 2);
  return (backward || a.h8 || a.a8) && bytes > ((int64_t)256 << 20);
}
int threads_of(int cols) { return (cols + 511) / 512 * 64; }
// Threads of a row in the backward, and the rows that a workgroup has abreast there, whose column sums it adds up itself: fewer runs'
// sums to write and to read again.
int bwd_across(int cols) { return cols <= kFewCols ? threads_of(cols) : (cols + 1023) / 1024 * 64; }
int bwd_abreast(int cols) { return cols <= 512 ? 4 : cols <= 1024 ? 2 : 1; }

template <bool B>
using flag = std::integral_constant<bool, B>;
// Calls go(X{}, Y{}, has P, rows end within a thread's columns, past the caches, few columns) with the stream's and the block's types.
template <class F>
void typed(const ResidualArgs& a, bool once, F go) {
  auto sized = [&](auto x, auto y, auto post) {
    auto odd = [&](auto few) {
      if (a.cols % kCols<decltype(x), decltype(y)>) {
        go(x, y, post, flag<true>{}, flag<false>{}, few);
      } else {
        if constexpr (sizeof(x) == sizeof(y))
          if (once) return go(x, y, post, flag<false>{}, flag<true>{}, few);
        go(x, y, post, flag<false>{}, flag<false>{}, few);
      }
    };
    if (a.cols > kFewCols)
      odd(flag<false>{});
    else
      odd(flag<true>{});
  };
  auto with = [&](auto x, auto y) {
    if (a.post != VC_NORM_NONE)
      sized(x, y, flag<true>{});
    else
      sized(x, y, flag<false>{});
  };
  if (!a.x_f32)
    with(__bf16{}, __bf16{});
  else if (!a.y_f32)
    with(float{}, __bf16{});
  else
    with(float{}, float{});
}

}  // namespace

void residual_groups(int64_t rows, int cols, bool backward, int* groups, int* chunk) {
  const int threads = backward ? bwd_across(cols) : threads_of(cols), abreast = backward ? bwd_abreast(cols) : 1;
  const int waves = !backward ? kFwdWaves : cols <= kFewCols ? kBwdWaves : 2;
  const int64_t most = 256 * std::max(1, 4 * waves / (threads / 64 * abreast));  // as many as 256 compute units hold
  // a run of the backward has four rows at least, or its sums weigh more than they: 780 x 3,568 28.7 us so, 34.9 with one, 29.9 with eight
  const int64_t c = (std::max<int64_t>((rows + most - 1) / most, backward ? 4 : 1) + abreast - 1) / abreast * abreast;
  *chunk = (int)c;
  *groups = (int)((rows + c - 1) / c);
}

hipError_t launch_residual_fwd(const ResidualArgs& a, hipStream_t s) {
  typed(a, once_of(a, false), [&](auto x, auto y, auto post, auto odd, auto once, auto few) {
    constexpr bool kFew = decltype(few)::value;
    hipLaunchKernelGGL((residual_fwd_kernel<decltype(x), decltype(y), decltype(post)::value, decltype(odd)::value, decltype(once)::value, kFew>), dim3(a.groups),
                       dim3(threads_of(a.cols)), 0, s, a);
  });
  return hipGetLastError();
}

hipError_t launch_residual_bwd(const ResidualArgs& a, bool kept, hipStream_t s) {
  typed(a, once_of(a, true), [&](auto x, auto y, auto post, auto odd, auto once, auto few) {
    constexpr bool kPost = decltype(post)::value, kOdd = decltype(odd)::value, kFew = decltype(few)::value;
    const int across = bwd_across(a.cols);
    const dim3 grid(a.groups), block(across * bwd_abreast(a.cols));
    if (kept)
      hipLaunchKernelGGL((residual_bwd_kernel<decltype(x), decltype(y), true, kPost, kOdd, decltype(once)::value, kFew>), grid, block, 0, s, a, across);
    else
      hipLaunchKernelGGL((residual_bwd_kernel<decltype(x), decltype(y), false, kPost, kOdd, decltype(once)::value, kFew>), grid, block, 0, s, a, across);
  });
  if (a.part) {
    const int across = (a.cols + kSumCols - 1) / kSumCols, samples = a.flat ? 1 : a.samples;
    auto shares = [](int of, int least) { return std::max(least, std::min(1024 / kSumCols, (of + 3) / 4 * 4)); };
    hipLaunchKernelGGL(residual_sample_kernel, dim3(3 * across * samples), dim3(kSumCols, shares(a.groups / samples, kSumWave)), 0, s, a);
    if (a.sums) hipLaunchKernelGGL(residual_shared_kernel, dim3(across), dim3(kSumCols, shares(samples, 4)), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace vcja
