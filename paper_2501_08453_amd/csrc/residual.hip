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
// second kernel adds them in order. No atomics.
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
// and its sample exists.
__device__ __forceinline__ Piece piece_at(const ResidualArgs& a, int r, int r1) {
  int s, b, e;  // sample, and its slot
  if (a.cu) {
    int lo = 0, hi = a.samples;  // the first sample whose slot ends behind r
    while (lo < hi) {
      const int m = (lo + hi) >> 1;
      if (a.cu[m + 1] > r)
        hi = m;
      else
        lo = m + 1;
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

// Sums over the workgroup of N values a thread, the same in every thread. red: two buffers in turn, so that one barrier a call is
// enough: a buffer is written again only behind the barrier of the call between.
template <int N, int W>
__device__ __forceinline__ void block_sum(float* v, float (*red)[W][N], int& turn) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
  const int waves = blockDim.x >> 6;
  if (waves == 1) return;
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) red[turn][threadIdx.x >> 6][i] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = 0.0f;
  for (int w = 0; w < waves; ++w)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += red[turn][w][i];
  turn ^= 1;
}

__device__ __forceinline__ const void* at_sample(const void* p, bool f32, int64_t stride, int s) {
  return !p ? p : f32 ? (const void*)((const float*)p + stride * s) : (const void*)((const __bf16*)p + stride * s);
}

// Threads of a workgroup, at most: up to 2,048 columns 256, which leaves a thread 256 registers, else 1,024.
template <class X, class Y, bool POST, int MAXT, int R>
__global__ __launch_bounds__(MAXT) void residual_fwd_kernel(ResidualArgs a) {
  __shared__ float red[2][MAXT / 64][R];
  int turn = 0;
  const int C = a.cols, col = threadIdx.x * 8, n = C - col;
  const float inv = 1.0f / C;
  const int r1 = min(a.rows, ((int)blockIdx.x + 1) * a.chunk), blocks = (C + kBlockOf8 - 1) / kBlockOf8;
  for (int r = blockIdx.x * a.chunk; r < r1;) {
    const Piece p = piece_at(a, r, r1);
    if (!p.live) {
      if (!p.outside || a.clear) {
        const float zero[8] = {};
        for (; r < p.end; ++r) {
          if (a.h) store8((X*)a.h + (int64_t)r * C + col, zero, n);
          if (a.y) store8((Y*)a.y + (int64_t)r * C + col, zero, n);
        }
      }
      r = p.end;
      continue;
    }
    float g[8], e[8], f[8];  // g: gate, with P's weight where there is one
    load8p(g, at_sample(a.gate, a.p_f32, a.gate_stride, p.sample), a.p_f32, col, n, 1.0f);
    if constexpr (POST) {
      float w[8];
      load8p(w, a.wp, a.p_f32, col, n, 1.0f);
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] *= w[i];
    }
    load8p(e, at_sample(a.scale, a.p_f32, a.scale_stride, p.sample), a.p_f32, col, n, a.plus_one ? 0.0f : 1.0f);
    load8p(f, at_sample(a.shift, a.p_f32, a.shift_stride, p.sample), a.p_f32, col, n, 0.0f);
    if (a.plus_one)
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] += 1.0f;
    for (; r < p.end; r += R) {
      const int m = min(R, p.end - r);
      float h[R][8], s[R], mean[R], rstd[R];
      Eight<X> x[R];
      Eight<Y> b[R];
#pragma unroll
      for (int j = 0; j < R; ++j) {
        const int64_t row = min(r + j, p.end - 1);
        load8(x[j], (const X*)a.x + row * a.x_stride + col, n);
        if (a.a) load8(b[j], (const Y*)a.a + row * a.a_stride + col, n);
      }
      if (a.a8) {
#pragma unroll
        for (int j = 0; j < R; ++j)
          if (j < m) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = b[j][i];
            const Kept k = keep8(v);
            store_q8(a.a8 + (int64_t)(r + j) * C + col, k.q, n);
            if ((threadIdx.x & 15) == 0 && n > 0) a.a8s[(int64_t)(r + j) * blocks + (threadIdx.x >> 4)] = k.scale;
          }
      }
      if constexpr (POST) {
#pragma unroll
        for (int j = 0; j < R; ++j) mean[j] = 0.0f;
        if (a.post == VC_NORM_LAYER) {
#pragma unroll
          for (int j = 0; j < R; ++j) {
            s[j] = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s[j] += b[j][i];
          }
          block_sum<R>(s, red, turn);
#pragma unroll
          for (int j = 0; j < R; ++j) mean[j] = s[j] * inv;
        }
#pragma unroll
        for (int j = 0; j < R; ++j) {
          s[j] = 0.0f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float d = b[j][i] - mean[j];
            s[j] = i < n ? fmaf(d, d, s[j]) : s[j];
          }
        }
        block_sum<R>(s, red, turn);
#pragma unroll
        for (int j = 0; j < R; ++j) {
          rstd[j] = 1.0f / sqrtf(fmaf(s[j], inv, a.eps));
          if (threadIdx.x == 0 && j < m) {
            a.pmean[r + j] = mean[j];
            a.prstd[r + j] = rstd[j];
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) h[j][i] = fmaf(g[i], (b[j][i] - mean[j]) * rstd[j], a.c * x[j][i]);
        }
      } else if (a.a) {
#pragma unroll
        for (int j = 0; j < R; ++j)
#pragma unroll
          for (int i = 0; i < 8; ++i) h[j][i] = fmaf(g[i], b[j][i], a.c * x[j][i]);
      } else {
#pragma unroll
        for (int j = 0; j < R; ++j)
#pragma unroll
          for (int i = 0; i < 8; ++i) h[j][i] = a.c * x[j][i];
      }
#pragma unroll
      for (int j = 0; j < R; ++j) {
        // The norm takes h as it is kept: the next block and the backward read that, not the sum before its rounding.
#pragma unroll
        for (int i = 0; i < 8; ++i) h[j][i] = i < n ? (float)(X)h[j][i] : 0.0f;
        if (j < m) {
          if (a.h) store8((X*)a.h + (int64_t)(r + j) * C + col, h[j], n);
          if (a.h8) {
            const Kept k = keep8(h[j]);
            store_q8(a.h8 + (int64_t)(r + j) * C + col, k.q, n);
            if ((threadIdx.x & 15) == 0 && n > 0) a.h8s[(int64_t)(r + j) * blocks + (threadIdx.x >> 4)] = k.scale;
          }
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
          for (int i = 0; i < 8; ++i) s[j] += h[j][i];
        }
        block_sum<R>(s, red, turn);
#pragma unroll
        for (int j = 0; j < R; ++j) mean[j] = s[j] * inv;
      }
#pragma unroll
      for (int j = 0; j < R; ++j) {
        s[j] = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          h[j][i] -= mean[j];
          s[j] = i < n ? fmaf(h[j][i], h[j][i], s[j]) : s[j];
        }
      }
      block_sum<R>(s, red, turn);
#pragma unroll
      for (int j = 0; j < R; ++j) {
        rstd[j] = 1.0f / sqrtf(fmaf(s[j], inv, a.eps));
        if (j >= m) break;
        if (threadIdx.x == 0) {
          a.mean[r + j] = mean[j];
          a.rstd[r + j] = rstd[j];
        }
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = fmaf(h[j][i] * rstd[j], e[i], f[i]);
        store8((Y*)a.y + (int64_t)(r + j) * C + col, y, n);
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

template <class X, class Y, bool K8, bool POST, int MAXT, int R>
__global__ __launch_bounds__(MAXT) void residual_bwd_kernel(ResidualArgs a) {
  using HT = typename From<X, Y, K8>::H;
  using AT = typename From<X, Y, K8>::A;
  __shared__ float red[2][MAXT / 64][2 * R];
  int turn = 0;
  const int C = a.cols, col = threadIdx.x * 8, n = C - col;
  const float inv = 1.0f / C, inv1 = a.norm == VC_NORM_LAYER ? inv : 0.0f, pinv1 = a.post == VC_NORM_LAYER ? inv : 0.0f;
  const int r1 = min(a.rows, ((int)blockIdx.x + 1) * a.chunk), blocks = (C + kBlockOf8 - 1) / kBlockOf8;
  const HT* hp = K8 ? (const HT*)a.h8 : (const HT*)a.h_in;
  const AT* ap = K8 ? (const AT*)a.a8 : (const AT*)a.a;
  const int64_t a_stride = K8 ? C : a.a_stride;
  const bool has_a = ap != nullptr, has_norm = a.norm != VC_NORM_NONE && a.dy;
  for (int r = blockIdx.x * a.chunk; r < r1;) {
    const Piece p = piece_at(a, r, r1);
    if (!p.live) {
      if (!p.outside || a.clear) {
        const float zero[8] = {};
        for (; r < p.end; ++r) {
          if (a.dx) store8((X*)a.dx + (int64_t)r * C + col, zero, n);
          if (a.da) store8((Y*)a.da + (int64_t)r * C + col, zero, n);
        }
      }
      r = p.end;
      continue;
    }
    float g[8], e[8], sa[8] = {}, se[8] = {}, sf[8] = {};  // g: gate, with P's weight where there is one
    load8p(g, at_sample(a.gate, a.p_f32, a.gate_stride, p.sample), a.p_f32, col, n, 1.0f);
    if constexpr (POST) {
      float w[8];
      load8p(w, a.wp, a.p_f32, col, n, 1.0f);
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] *= w[i];
    }
    load8p(e, at_sample(a.scale, a.p_f32, a.scale_stride, p.sample), a.p_f32, col, n, a.plus_one ? 0.0f : 1.0f);
    if (a.plus_one)
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] += 1.0f;
    for (; r < p.end; r += R) {
      const int m = min(R, p.end - r);
      float H[R][8], s[2 * R], hs[R], as[R], mean[R], rstd[R];
      Eight<X> dh[R];
      Eight<Y> dy[R];
      Eight<HT> h[R];
      Eight<AT> b[R];
#pragma unroll
      for (int j = 0; j < R; ++j) {
        const int row = min(r + j, p.end - 1);
        hs[j] = as[j] = 1.0f;
        dh[j] = Eight<X>{};
        if (a.dh) load8(dh[j], (const X*)a.dh + row * a.dh_stride + col, n);
        if (has_norm) {
          load8(dy[j], (const Y*)a.dy + row * a.dy_stride + col, n);
          load8(h[j], hp + (int64_t)row * C + col, n);
          if (K8 && n > 0) hs[j] = a.h8s[(int64_t)row * blocks + (threadIdx.x >> 4)];
        }
        if (has_a) {
          load8(b[j], ap + row * a_stride + col, n);
          if (K8 && n > 0) as[j] = a.a8s[(int64_t)row * blocks + (threadIdx.x >> 4)];
        }
      }
      if (has_norm) {
#pragma unroll
        for (int j = 0; j < R; ++j) {
          const int row = min(r + j, p.end - 1);
          rstd[j] = a.rstd[row];
          mean[j] = a.norm == VC_NORM_LAYER ? a.mean[row] : 0.0f;
          s[2 * j] = s[2 * j + 1] = 0.0f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float d = dy[j][i], xh = (h[j][i] * hs[j] - mean[j]) * rstd[j], G = d * e[i];
            s[2 * j] += G;
            s[2 * j + 1] = i < n ? fmaf(G, xh, s[2 * j + 1]) : s[2 * j + 1];
            if (j < m) {
              se[i] = fmaf(d, xh, se[i]);
              sf[i] += d;
            }
          }
        }
        block_sum<2 * R>(s, red, turn);
#pragma unroll
        for (int j = 0; j < R; ++j) {
          const float m1 = s[2 * j] * inv1, m2 = s[2 * j + 1] * inv;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float xh = (h[j][i] * hs[j] - mean[j]) * rstd[j];
            H[j][i] = fmaf(rstd[j], fmaf(dy[j][i], e[i], -m1) - xh * m2, dh[j][i]);
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < R; ++j)
#pragma unroll
          for (int i = 0; i < 8; ++i) H[j][i] = dh[j][i];
      }
#pragma unroll
      for (int j = 0; j < R; ++j) {
        float dx[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          H[j][i] = i < n ? H[j][i] : 0.0f;
          dx[i] = a.c * H[j][i];
        }
        if (j < m && a.dx) store8((X*)a.dx + (int64_t)(r + j) * C + col, dx, n);
      }
      if constexpr (!POST) {
        if (!has_a) continue;
#pragma unroll
        for (int j = 0; j < R; ++j) {
          if (j >= m) break;
          float da[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            sa[i] = fmaf(H[j][i], b[j][i] * as[j], sa[i]);
            da[i] = H[j][i] * g[i];
          }
          if (a.da) store8((Y*)a.da + (int64_t)(r + j) * C + col, da, n);
        }
      } else {
#pragma unroll
        for (int j = 0; j < R; ++j) {
          const int row = min(r + j, p.end - 1);
          mean[j] = a.post == VC_NORM_LAYER ? a.pmean[row] : 0.0f;
          rstd[j] = a.prstd[row];
          s[2 * j] = s[2 * j + 1] = 0.0f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float xa = (b[j][i] * as[j] - mean[j]) * rstd[j], K = H[j][i] * g[i];
            s[2 * j] += K;
            s[2 * j + 1] = i < n ? fmaf(K, xa, s[2 * j + 1]) : s[2 * j + 1];
            if (j < m) sa[i] = fmaf(H[j][i], xa, sa[i]);
          }
        }
        block_sum<2 * R>(s, red, turn);
#pragma unroll
        for (int j = 0; j < R; ++j) {
          if (j >= m) break;
          const float m1 = s[2 * j] * pinv1, m2 = s[2 * j + 1] * inv;
          float da[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float xa = (b[j][i] * as[j] - mean[j]) * rstd[j];
            da[i] = rstd[j] * (fmaf(H[j][i], g[i], -m1) - xa * m2);
          }
          if (a.da) store8((Y*)a.da + (int64_t)(r + j) * C + col, da, n);
        }
      }
    }
    r = p.end;
    if (a.part) {
      float* out = a.part + ((int64_t)blockIdx.x + p.sample) * 3 * C + col;
      store8(out, sa, n);
      store8(out + C, se, n);
      store8(out + 2 * C, sf, n);
    }
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

constexpr int kSumCols = 64;

// The sums of one sample from those of its runs, in order: 64 columns a workgroup, blockDim.y shares of the runs.
__global__ __launch_bounds__(1024) void residual_sample_kernel(ResidualArgs a) {
  __shared__ float sum[3][16][kSumCols];
  const int C = a.cols, across = (C + kSumCols - 1) / kSumCols;
  const int s = blockIdx.x / across, col = (blockIdx.x - s * across) * kSumCols + threadIdx.x;
  int b, e;
  if (a.cu) {
    b = min(max(a.cu[s], 0), a.rows);
    e = min(max(a.cu[s + 1], b), a.rows);
  } else {
    b = s * a.per;
    e = b + a.per;
  }
  if (a.lens) e = b + min(max(a.lens[s], 0), e - b);
  const int g0 = b / a.chunk, g1 = e > b ? (e - 1) / a.chunk + 1 : g0, share = (g1 - g0 + blockDim.y - 1) / blockDim.y;
  const int last = min(g1, g0 + ((int)threadIdx.y + 1) * share);
  float v[3] = {};
  if (col < C)
    for (int g = g0 + threadIdx.y * share; g < last; ++g) {
      const float* p = a.part + ((int64_t)g + s) * 3 * C + col;
#pragma unroll
      for (int k = 0; k < 3; ++k) v[k] += p[(int64_t)k * C];
    }
#pragma unroll
  for (int k = 0; k < 3; ++k) sum[k][threadIdx.y][threadIdx.x] = v[k];
  __syncthreads();
  if (threadIdx.y || col >= C) return;
  for (int y = 1; y < (int)blockDim.y; ++y)
#pragma unroll
    for (int k = 0; k < 3; ++k) v[k] += sum[k][y][threadIdx.x];
  const int64_t at = (int64_t)s * C + col;
  if (a.sums) {
#pragma unroll
    for (int k = 0; k < 3; ++k) a.sums[((int64_t)s * 3 + k) * C + col] = v[k];
  }
  const bool one = a.samples == 1;
  if (a.gate_stride || one) write(a.dgate, a.p_f32, at, v[0] * param(a.wp, a.p_f32, col, 1.0f));
  if (a.scale_stride || one) write(a.dscale, a.p_f32, at, v[1]);
  if (a.shift_stride || one) write(a.dshift, a.p_f32, at, v[2]);
  if (one) write(a.dwp, a.p_f32, col, v[0] * param(a.gate, a.p_f32, col, 1.0f));
}

// What all samples share, from the samples' sums.
__global__ __launch_bounds__(1024) void residual_shared_kernel(ResidualArgs a) {
  __shared__ float sum[4][16][kSumCols];
  const int C = a.cols, col = blockIdx.x * kSumCols + threadIdx.x;
  const int share = (a.samples + 15) / 16, last = min(a.samples, ((int)threadIdx.y + 1) * share);
  float v[4] = {};
  if (col < C)
    for (int s = threadIdx.y * share; s < last; ++s) {
      const float* p = a.sums + (int64_t)s * 3 * C + col;
      const float t = p[0];
      v[0] += t;
      v[1] += p[C];
      v[2] += p[2 * C];
      v[3] = fmaf(t, param(a.gate, a.p_f32, a.gate_stride * s + col, 1.0f), v[3]);
    }
#pragma unroll
  for (int k = 0; k < 4; ++k) sum[k][threadIdx.y][threadIdx.x] = v[k];
  __syncthreads();
  if (threadIdx.y || col >= C) return;
  for (int y = 1; y < 16; ++y)
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] += sum[k][y][threadIdx.x];
  if (!a.gate_stride) write(a.dgate, a.p_f32, col, v[0] * param(a.wp, a.p_f32, col, 1.0f));
  if (!a.scale_stride) write(a.dscale, a.p_f32, col, v[1]);
  if (!a.shift_stride) write(a.dshift, a.p_f32, col, v[2]);
  write(a.dwp, a.p_f32, col, v[3]);
}

int threads_of(int cols) { return (cols + 511) / 512 * 64; }

template <bool B>
using flag = std::integral_constant<bool, B>;
// Calls go(X{}, Y{}, has P, most threads) with the stream's and the block's types.
template <class F>
void typed(const ResidualArgs& a, F go) {
  auto sized = [&](auto x, auto y, auto post) {
    if (threads_of(a.cols) <= 256)
      go(x, y, post, std::integral_constant<int, 256>{});
    else
      go(x, y, post, std::integral_constant<int, 1024>{});
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
  const int64_t most = 256 * std::max(1, 16 / (threads_of(cols) / 64));
  const int64_t c = (rows + most - 1) / most;
  *chunk = (int)c;
  *groups = (int)((rows + c - 1) / c);
}

hipError_t launch_residual_fwd(const ResidualArgs& a, hipStream_t s) {
  typed(a, [&](auto x, auto y, auto post, auto most) {
    constexpr int kMost = decltype(most)::value, kRows = kMost == 256 ? 2 : 1;
    hipLaunchKernelGGL((residual_fwd_kernel<decltype(x), decltype(y), decltype(post)::value, kMost, kRows>), dim3(a.groups),
                       dim3(threads_of(a.cols)), 0, s, a);
  });
  return hipGetLastError();
}

hipError_t launch_residual_bwd(const ResidualArgs& a, bool kept, hipStream_t s) {
  typed(a, [&](auto x, auto y, auto post, auto most) {
    constexpr int kMost = decltype(most)::value, kRows = kMost == 256 ? 2 : 1;
    constexpr bool kPost = decltype(post)::value;
    const dim3 grid(a.groups), block(threads_of(a.cols));
    if (kept)
      hipLaunchKernelGGL((residual_bwd_kernel<decltype(x), decltype(y), true, kPost, kMost, kRows>), grid, block, 0, s, a);
    else
      hipLaunchKernelGGL((residual_bwd_kernel<decltype(x), decltype(y), false, kPost, kMost, kRows>), grid, block, 0, s, a);
  });
  if (a.part) {
    const int across = (a.cols + kSumCols - 1) / kSumCols;
    const int shares = std::max(1, std::min(16, a.groups / a.samples));
    hipLaunchKernelGGL(residual_sample_kernel, dim3(across * a.samples), dim3(kSumCols, shares), 0, s, a);
    if (a.sums) hipLaunchKernelGGL(residual_shared_kernel, dim3(across), dim3(kSumCols, 16), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace vcja
