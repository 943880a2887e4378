// Embedding of tokens for gfx950, and its gradient: out_t = scale table[id_t], and dtable_v = scale times the sum of the
// rows dout_t of the tokens t with id v, in the order of t. No atomics on the sums: the tokens are sorted by their ids
// (stably, so that equal ones keep their order), and shares of the sorted list are summed each by itself.
//
// Bound by memory: rows of the table, rows of dout, and every row of the gradient, which is written whole (zeros where no token met it).
// Sort: digits of up to nine bits, the last first. A wave finds the lanes of the same digit by ballots and counts for itself, so that
// the order is that of the tokens. Up to 8,192 tokens one workgroup sorts in LDS; more take two launches a digit.
// Sums: a share of the sorted list writes the rows of ids that begin and end in it; the sums of ids that go on beyond it are
// kept apart and added in order by the last kernel, however many shares a frequent id fills.
#include "embedding.hpp"

#include <algorithm>

#include "rows.hpp"

namespace vcja {
namespace {

constexpr int kRowThreads = 256;   // threads of a workgroup, where a row takes fewer
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kDigits = 512;
constexpr int kOneBlock = 8192;   // most tokens that one workgroup sorts
constexpr int kFillRows = 64;      // rows of the table that a workgroup looks through for zeros

// The id of token t; `vocab`, which is none, where it is the padding's or none of the table's.
__device__ __forceinline__ int64_t id_of(const EmbeddingArgs& a, int64_t t) {
  const int64_t id = a.ids64 ? ((const int64_t*)a.ids)[t] : (int64_t)((const int32_t*)a.ids)[t];
  return id < 0 || id >= a.vocab || id == a.padding ? a.vocab : id;
}

template <class T, class O>
__global__ __launch_bounds__(1024) void embedding_fwd_kernel(EmbeddingArgs a) {
  constexpr int U = 4;  // tokens of a thread in flight
  const int across = (a.cols + 7) / 8, rows = blockDim.x / across;
  const int ty = threadIdx.x / across, col = (threadIdx.x - ty * across) * 8, n = a.cols - col;
  if (ty >= rows) return;
  const int64_t step = (int64_t)gridDim.x * rows;
  for (int64_t t = (int64_t)blockIdx.x * rows + ty; t < a.tokens; t += U * step) {
    Eight<T> r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      r[u] = Eight<T>{};
      const int64_t id = t + u * step < a.tokens ? id_of(a, t + u * step) : a.vocab;
      if (id < a.vocab) load8(r[u], (const T*)a.table + id * a.table_stride + col, n);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (t + u * step >= a.tokens) break;
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = r[u][e] * a.scale;
      store8((O*)a.out + (t + u * step) * a.cols + col, x, n);
    }
  }
}

// --- sort ---------------------------------------------------------------------------------------

// Ranks of this wave's ITEMS x 64 digits (item k of lane l is number 64 k + l) among those before with the same digit;
// count: the wave's own counters, zeros before.
template <int ITEMS>
__device__ __forceinline__ void wave_ranks(const uint32_t* digit, const bool* real, uint32_t* rank, uint32_t* count, int bits) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    uint64_t same = __ballot(real[k]);
    for (int b = 0; b < bits; ++b) {
      const bool one = digit[k] >> b & 1;
      const uint64_t m = __ballot(one);
      same &= one ? m : ~m;
    }
    const int first = real[k] ? __ffsll((unsigned long long)same) - 1 : lane;
    uint32_t base = 0;
    if (real[k] && lane == first) base = atomicAdd(&count[digit[k]], (uint32_t)__popcll(same));
    base = __shfl(base, first, 64);
    rank[k] = base + __popcll(same & (((uint64_t)1 << lane) - 1));
  }
}

// Exclusive sums over the 512 values v of the first 512 threads. Every thread of the workgroup calls it. tmp: 8 values.
__device__ __forceinline__ uint32_t scan512(uint32_t v, uint32_t* tmp) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t s = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t t = __shfl_up(s, o, 64);
    if (lane >= o) s += t;
  }
  if (lane == 63 && wave < 8) tmp[wave] = s;
  __syncthreads();
  for (int w = 0; w < wave && w < 8; ++w) s += tmp[w];
  return s - v;
}

// One workgroup: all passes in LDS.
template <int ITEMS>
__global__ __launch_bounds__(kSortThreads) void embedding_sort_one_kernel(EmbeddingArgs a) {
  __shared__ uint32_t keys[kSortThreads * ITEMS], pos[kSortThreads * ITEMS];
  __shared__ uint32_t count[kSortWaves][kDigits];
  __shared__ uint32_t tmp[8];
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63, T = (int)a.tokens;
  const int at = wave * 64 * ITEMS + lane;
  uint32_t key[ITEMS], p[ITEMS], rank[ITEMS], digit[ITEMS];
  bool real[ITEMS];
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    p[k] = at + 64 * k;
    real[k] = (int)p[k] < T;
    key[k] = real[k] ? (uint32_t)id_of(a, p[k]) : 0;
  }
  for (int pass = 0; pass < a.passes; ++pass) {
    for (int i = lane; i < kDigits; i += 64) count[wave][i] = 0;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) digit[k] = key[k] >> (pass * a.digits) & ((1u << a.digits) - 1);
    __syncthreads();
    wave_ranks<ITEMS>(digit, real, rank, count[wave], a.digits);
    __syncthreads();
    uint32_t all = 0;
    if (t < kDigits)
      for (int w = 0; w < kSortWaves; ++w) {
        const uint32_t c = count[w][t];
        count[w][t] = all;
        all += c;
      }
    const uint32_t before = scan512(t < kDigits ? all : 0, tmp);
    if (t < kDigits)
      for (int w = 0; w < kSortWaves; ++w) count[w][t] += before;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
      if (real[k]) {
        const uint32_t to = count[wave][digit[k]] + rank[k];
        keys[to] = key[k];
        pos[to] = p[k];
      }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
      if (real[k]) {
        key[k] = keys[at + 64 * k];
        p[k] = pos[at + 64 * k];
      }
  }
#pragma unroll
  for (int k = 0; k < ITEMS; ++k)
    if (real[k]) {
      a.keys[0][at + 64 * k] = key[k];
      a.pos[0][at + 64 * k] = p[k];
    }
}

__device__ __forceinline__ uint32_t sort_key(const EmbeddingArgs& a, int pass, int64_t i) {
  return pass == 0 ? (uint32_t)id_of(a, i) : a.keys[pass & 1][i];
}

// Several workgroups: how often each digit stands in each block's tokens.
template <int ITEMS>
__global__ __launch_bounds__(kSortThreads) void embedding_count_kernel(EmbeddingArgs a, int pass) {
  __shared__ uint32_t count[kDigits];
  const int t = threadIdx.x;
  if (t < kDigits) count[t] = 0;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    const int64_t i = (int64_t)blockIdx.x * kSortThreads * ITEMS + k * kSortThreads + t;
    if (i < a.tokens) atomicAdd(&count[sort_key(a, pass, i) >> (pass * a.digits) & ((1u << a.digits) - 1)], 1u);
  }
  __syncthreads();
  if (t < kDigits) a.hist[(int64_t)blockIdx.x * kDigits + t] = count[t];
}

// ... and each block's tokens to their places of this pass.
template <int ITEMS>
__global__ __launch_bounds__(kSortThreads) void embedding_move_kernel(EmbeddingArgs a, int pass) {
  __shared__ uint32_t count[kSortWaves][kDigits];
  __shared__ uint32_t tmp[8];
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
  const int64_t at = (int64_t)blockIdx.x * kSortThreads * ITEMS + wave * 64 * ITEMS + lane;
  uint32_t key[ITEMS], p[ITEMS], rank[ITEMS], digit[ITEMS];
  bool real[ITEMS];
  for (int i = lane; i < kDigits; i += 64) count[wave][i] = 0;
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    const int64_t i = at + 64 * k;
    real[k] = i < a.tokens;
    key[k] = real[k] ? sort_key(a, pass, i) : 0;
    p[k] = !real[k] ? 0 : pass == 0 ? (uint32_t)i : a.pos[pass & 1][i];
    digit[k] = key[k] >> (pass * a.digits) & ((1u << a.digits) - 1);
  }
  __syncthreads();
  wave_ranks<ITEMS>(digit, real, rank, count[wave], a.digits);
  __syncthreads();
  uint32_t total = 0, mine = 0;  // of this digit: in all blocks, in those before
  if (t < kDigits)
#pragma unroll 8
    for (int b = 0; b < (int)gridDim.x; ++b) {
      const uint32_t c = a.hist[(int64_t)b * kDigits + t];
      total += c;
      mine += b < (int)blockIdx.x ? c : 0;
    }
  const uint32_t before = scan512(t < kDigits ? total : 0, tmp) + mine;
  if (t < kDigits) {
    uint32_t all = before;
    for (int w = 0; w < kSortWaves; ++w) {
      const uint32_t c = count[w][t];
      count[w][t] = all;
      all += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < ITEMS; ++k)
    if (real[k]) {
      const uint32_t to = count[wave][digit[k]] + rank[k];
      a.keys[(pass + 1) & 1][to] = key[k];
      a.pos[(pass + 1) & 1][to] = p[k];
    }
}

// --- sums ---------------------------------------------------------------------------------------

// The first of the sorted keys that is at least v (past, more than v).
__device__ __forceinline__ int64_t lower(const uint32_t* keys, int64_t lo, int64_t hi, uint32_t v) {
  while (lo < hi) {
    const int64_t m = (lo + hi) >> 1;
    if (keys[m] < v)
      lo = m + 1;
    else
      hi = m;
  }
  return lo;
}

template <class G>
__device__ __forceinline__ void write_row(const EmbeddingArgs& a, int64_t v, int col, int n, float* sum) {
  G* g = (G*)a.grad + v * a.cols + col;
#pragma unroll
  for (int e = 0; e < 8; ++e) sum[e] *= a.scale;
  if (a.add) {
    Eight<G> old;
    load8(old, (const G*)g, n);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] += old[e];
  }
  store8(g, sum, n);
}

// The first `sums` workgroups sum shares of the sorted tokens, the others write zeros to the rows that no token met.
template <class D, class G>
__global__ __launch_bounds__(1024) void embedding_sum_kernel(EmbeddingArgs a, int sums) {
  const uint32_t *keys = a.keys[0], *pos = a.pos[0];
  const uint32_t V = (uint32_t)a.vocab;
  const int64_t T = a.tokens;
  if ((int)blockIdx.x >= sums) {
    const int64_t v0 = ((int64_t)blockIdx.x - sums) * kFillRows;
    const int waves = blockDim.x >> 6, lane = threadIdx.x & 63;
    const int64_t v = v0 + lane;
    bool none = false;
    if (v < a.vocab) {
      const int64_t i = lower(keys, 0, T, (uint32_t)v);
      none = i == T || keys[i] != (uint32_t)v;
    }
    uint64_t rows = __ballot(none);
    const float zero[8] = {};
    for (int i = 0; rows; ++i, rows &= rows - 1) {
      if (i % waves != (int)(threadIdx.x >> 6)) continue;
      G* g = (G*)a.grad + (v0 + __ffsll((unsigned long long)rows) - 1) * a.cols;
      for (int c = lane * 8; c < a.cols; c += 512) store8(g + c, zero, a.cols - c);
    }
    return;
  }
  constexpr int U = 8;  // rows of a thread in flight
  const int across = (a.cols + 7) / 8, shares = blockDim.x / across;
  const int ty = threadIdx.x / across, col = (threadIdx.x - ty * across) * 8, n = a.cols - col;
  const int64_t c = (int64_t)blockIdx.x * shares + ty;
  if (ty >= shares || c >= a.chunks) return;
  const int64_t i0 = c * a.chunk, i1 = min(T, i0 + a.chunk);
  uint32_t cur = keys[i0];
  bool from = i0 > 0 && keys[i0 - 1] == cur;  // goes on from the share before
  float sum[8] = {};
  float* part = a.part + c * 2 * a.cols + col;
  auto done = [&](bool on) {  // on: goes on in the next share
    if (cur >= V) return;
    if (from)
      store8(part, sum, n);
    else if (on)
      store8(part + a.cols, sum, n);
    else
      write_row<G>(a, cur, col, n, sum);
  };
  for (int64_t i = i0; i < i1; i += U) {
    uint32_t k[U];
    Eight<D> r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = min(i + u, i1 - 1);
      k[u] = keys[at];
      r[u] = Eight<D>{};
      if (k[u] < V) load8(r[u], (const D*)a.dout + (int64_t)pos[at] * a.dout_stride + col, n);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u >= i1) break;
      if (k[u] != cur) {
        done(false);
        cur = k[u];
        from = false;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += r[u][e];
    }
  }
  done(i1 < T && keys[i1] == cur);
}

// The row of an id whose tokens begin in share c and go on beyond it: its sums of all shares, in order.
template <class G>
__global__ __launch_bounds__(1024) void embedding_join_kernel(EmbeddingArgs a) {
  __shared__ float sums[1024 * 8];
  const uint32_t* keys = a.keys[0];
  const int64_t T = a.tokens, c = blockIdx.x, i0 = c * a.chunk, i1 = i0 + a.chunk;
  if (i1 >= T) return;
  const uint32_t v = keys[i1 - 1];
  if (v >= (uint32_t)a.vocab || keys[i1] != v || (keys[i0] == v && i0 > 0 && keys[i0 - 1] == v)) return;
  const int count = (int)((lower(keys, i1, T, v + 1) - 1) / a.chunk - c) + 1;  // shares of this id
  const int across = (a.cols + 7) / 8, runs = blockDim.x / across;
  const int ty = threadIdx.x / across, col = (threadIdx.x - ty * across) * 8, n = a.cols - col;
  const int per = (count + runs - 1) / runs, last = min(count, (ty + 1) * per);
  float sum[8] = {};
  if (ty < runs) {
#pragma unroll 4
    for (int j = ty * per; j < last; ++j) {
      Eight<float> r;
      load8(r, (const float*)a.part + (c + j) * 2 * a.cols + (j ? 0 : a.cols) + col, n);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += r[e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[e * 1024 + threadIdx.x] = sum[e];
  }
  __syncthreads();
  if (ty) return;
  for (int y = 1; y < runs; ++y)
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] += sums[e * 1024 + y * across + threadIdx.x];
  write_row<G>(a, v, col, n, sum);
}

// Threads of a workgroup whose rows take `across` threads each.
int row_threads(int cols, int most) {
  const int across = (cols + 7) / 8;
  return std::min(1024, (std::max(across, most / across * across) + 63) / 64 * 64);
}
template <class F>
void pick(bool first, bool second, F go) {
  auto with = [&](auto x) {
    if (second)
      go(x, float{});
    else
      go(x, __bf16{});
  };
  if (first)
    with(float{});
  else
    with(__bf16{});
}
int items(int64_t tokens) { return tokens <= 131072 ? 4 : 16; }

}  // namespace

EmbeddingPlan embedding_plan(int64_t tokens, int64_t vocab, int cols) {
  EmbeddingPlan p;
  int bits = 1;
  while (vocab >> bits) ++bits;  // of keys up to `vocab` itself
  p.passes = (bits + 8) / 9;
  p.digits = (bits + p.passes - 1) / p.passes;
  const int per = kSortThreads * items(tokens);
  p.blocks = tokens <= kOneBlock ? 1 : (int)((tokens + per - 1) / per);
  p.chunk = (int)std::max<int64_t>(8, (tokens + 8 * 4096 - 1) / (8 * 4096) * 8);
  p.chunks = (int)((tokens + p.chunk - 1) / p.chunk);
  return p;
}

hipError_t launch_embedding_fwd(const EmbeddingArgs& a, hipStream_t s) {
  const int threads = row_threads(a.cols, kRowThreads), rows = threads / ((a.cols + 7) / 8);
  const int64_t blocks = std::min<int64_t>(4096, (a.tokens + rows - 1) / rows);
  pick(a.table_f32, a.out_f32, [&](auto t, auto o) {
    hipLaunchKernelGGL((embedding_fwd_kernel<decltype(t), decltype(o)>), dim3(blocks), dim3(threads), 0, s, a);
  });
  return hipGetLastError();
}

hipError_t launch_embedding_bwd(EmbeddingArgs a, hipStream_t s) {
  const EmbeddingPlan p = embedding_plan(a.tokens, a.vocab, a.cols);
  a.passes = p.passes;
  a.digits = p.digits;
  a.chunk = p.chunk;
  a.chunks = p.chunks;
  if (p.blocks == 1) {
    if (a.tokens <= 1024)
      hipLaunchKernelGGL(embedding_sort_one_kernel<1>, dim3(1), dim3(kSortThreads), 0, s, a);
    else if (a.tokens <= 4096)
      hipLaunchKernelGGL(embedding_sort_one_kernel<4>, dim3(1), dim3(kSortThreads), 0, s, a);
    else
      hipLaunchKernelGGL(embedding_sort_one_kernel<8>, dim3(1), dim3(kSortThreads), 0, s, a);
  } else {
    for (int pass = 0; pass < p.passes; ++pass) {
      if (items(a.tokens) == 4) {
        hipLaunchKernelGGL(embedding_count_kernel<4>, dim3(p.blocks), dim3(kSortThreads), 0, s, a, pass);
        hipLaunchKernelGGL(embedding_move_kernel<4>, dim3(p.blocks), dim3(kSortThreads), 0, s, a, pass);
      } else {
        hipLaunchKernelGGL(embedding_count_kernel<16>, dim3(p.blocks), dim3(kSortThreads), 0, s, a, pass);
        hipLaunchKernelGGL(embedding_move_kernel<16>, dim3(p.blocks), dim3(kSortThreads), 0, s, a, pass);
      }
    }
    if (p.passes & 1) {  // the last pass wrote the second of the two
      std::swap(a.keys[0], a.keys[1]);
      std::swap(a.pos[0], a.pos[1]);
    }
  }
  const int threads = row_threads(a.cols, kRowThreads), shares = threads / ((a.cols + 7) / 8);
  const int sums = (p.chunks + shares - 1) / shares;
  const int fill = a.add ? 0 : (int)((a.vocab + kFillRows - 1) / kFillRows);
  pick(a.out_f32, a.grad_f32, [&](auto d, auto g) {
    hipLaunchKernelGGL((embedding_sum_kernel<decltype(d), decltype(g)>), dim3(sums + fill), dim3(threads), 0, s, a, sums);
  });
  if (p.chunks > 1) {
    if (a.grad_f32)
      hipLaunchKernelGGL(embedding_join_kernel<float>, dim3(p.chunks), dim3(row_threads(a.cols, 1024)), 0, s, a);
    else
      hipLaunchKernelGGL(embedding_join_kernel<__bf16>, dim3(p.chunks), dim3(row_threads(a.cols, 1024)), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace vcja
