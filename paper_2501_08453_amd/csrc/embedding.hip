// Embedding of tokens for gfx950, and its gradient: out_t = scale table[id_t], and dtable_v = scale times the sum of the
// rows dout_t of the tokens t with id v, in the order of t. No atomics on the sums: the tokens are sorted by their ids
// (stably, so that equal ones keep their order), and shares of the sorted list are summed each by itself.
//
// Bound by memory: rows of the table, rows of dout, and every row of the gradient, which is written whole (zeros where no token met it).
// Sort: digits of up to nine bits, the last first. A wave finds the lanes of the same digit by ballots and counts for itself, so that
// the order is that of the tokens. Up to 8,192 tokens one workgroup sorts in LDS; more take two launches a digit. Up to 64 need no sort.
// Sums: a share of the sorted list writes the rows of ids that begin and end in it; the sums of ids that go on beyond it are
// kept apart and added in order by the last kernel, however many shares a frequent id fills.
// 65,536 tokens of 50,000 ids as words come, 1,536 columns, bf16 rows, fp32 gradient: lookup 47 us (5.3 TB/s), sort and zeros 44, sums 71, joins 10.
#include "embedding.hpp"

#include <algorithm>

#include "rows.hpp"

namespace vcja {
namespace {

constexpr int kRowThreads = 256;   // threads of a workgroup, where a row takes fewer
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;
constexpr int kOneBlock = 8192;   // most tokens that one workgroup sorts
constexpr int kFewTokens = 64;    // most that need no sort
// Bytes of zeros of a workgroup then. 64 tokens of 2,000 ids of 2,048 columns in fp32, 50,000 of 1,536, 100,000 of 64: 9, 64 and 15 us on the GPU, with
// 16 KiB 12, 134 and 15; by three launches 12, 67 and 14, and 17 us of the host for a small call instead of 11.
constexpr int64_t kFewFill = 65536;
constexpr int kFillRows = 64;      // rows of the table that a workgroup looks through for zeros
// Bytes of zeros beside the sort of one workgroup, or beside a pass of several, and most workgroups that write them. Lookup and gradient
// with ids as words come, bf16 rows, fp32 gradients of 1,536 columns, at 16, 32, 64, 96 and 128 MiB a pass: 65,536 tokens of 50,000 ids 180,
// 176, 176, 173 and 171 us, of 32,128 162, 159, 147, 153 and 153, 16,384 of 50,000 121, 117, 109, 104 and 108. (Where nearly every row is met, what
// was written beside the sort is written twice.)
constexpr int64_t kFillOne = (int64_t)128 << 20, kFillPass = (int64_t)96 << 20;
constexpr int kFillGroups = 512;

// The ids of K tokens at(0), at(1), ..., all in flight at once (so no branch stands between two of them, and every place exists);
// `vocab`, which is none, where it is the padding's or none of the table's.
template <int K, class At>
__device__ __forceinline__ void ids_of(const EmbeddingArgs& a, uint32_t* key, At at) {
  int64_t id[K];
  if (a.ids64) {
#pragma unroll
    for (int k = 0; k < K; ++k) id[k] = ((const int64_t*)a.ids)[at(k)];
  } else {
#pragma unroll
    for (int k = 0; k < K; ++k) id[k] = ((const int32_t*)a.ids)[at(k)];
  }
#pragma unroll
  for (int k = 0; k < K; ++k) key[k] = (uint32_t)(id[k] < 0 || id[k] >= a.vocab || id[k] == a.padding ? a.vocab : id[k]);
}

// A row of threads: `across` of them, V vectors of N columns each.
template <class A, class B>
struct Form {
  static constexpr int N = sizeof(A) == 2 || sizeof(B) == 2 ? 8 : 4, V = 8 / N;
};
template <int N, int V>
__device__ __forceinline__ void spans_of(Span<N>* s, int t, int across, int C) {
#pragma unroll
  for (int v = 0; v < V; ++v) s[v] = span_at<N>((v * across + t) * N, C);
}

template <class T, class O, bool ONCE>
__global__ __launch_bounds__(1024) void embedding_fwd_kernel(EmbeddingArgs a) {
  constexpr int U = 4, N = Form<T, O>::N, V = Form<T, O>::V;  // U: tokens of a thread in flight
  const int across = (a.cols + 7) / 8, rows = blockDim.x / across, ty = threadIdx.x / across;
  if (ty >= rows) return;
  Span<N> s[V];
  spans_of<N, V>(s, threadIdx.x - ty * across, across, a.cols);
  const int64_t step = (int64_t)gridDim.x * rows;
  for (int64_t t = (int64_t)blockIdx.x * rows + ty; t < a.tokens; t += U * step) {
    Cols<T, N> r[U][V];
    uint32_t id[U];
    ids_of<U>(a, id, [&](int u) { return min(t + u * step, a.tokens - 1); });
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        r[u][v] = Cols<T, N>{};
        if (id[u] < (uint32_t)a.vocab && t + u * step < a.tokens) load_cols(r[u][v], (const T*)a.table + id[u] * a.table_stride, s[v]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (t + u * step >= a.tokens) break;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float x[N];
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = r[u][v][e] * a.scale;
        store_cols<true, ONCE>((O*)a.out + (t + u * step) * a.cols, x, s[v]);
      }
    }
  }
}

// Zeros to rows [v0, v1) of the gradient: by workgroup `at` of `of` that do so.
template <bool ONCE>
__device__ __forceinline__ void fill_rows_as(const EmbeddingArgs& a, int64_t v0, int64_t v1, int at, int of) {
  const int64_t n = (v1 - v0) * a.cols * (a.grad_f32 ? 4 : 2);  // bytes, whole elements
  char* p = (char*)a.grad + v0 * a.cols * (a.grad_f32 ? 4 : 2);
  typedef f32x4 any __attribute__((aligned(2)));
  const int64_t step = (int64_t)of * blockDim.x * 16;
  for (int64_t i = ((int64_t)at * blockDim.x + threadIdx.x) * 16; i < n; i += step) {
    if (i + 16 > n)
      for (int64_t j = i; j < n; j += 2) *(uint16_t*)(p + j) = 0;
    else if constexpr (ONCE)
      __builtin_nontemporal_store(f32x4{}, (any*)(p + i));
    else
      *(any*)(p + i) = f32x4{};
  }
}
__device__ __forceinline__ void fill_rows(const EmbeddingArgs& a, int64_t v0, int64_t v1, int at, int of) {
  if (a.once)
    fill_rows_as<true>(a, v0, v1, at, of);
  else
    fill_rows_as<false>(a, v0, v1, at, of);
}

// --- sort ---------------------------------------------------------------------------------------
//
// One workgroup, or a few, sort while the others of the launch write zeros to rows of the gradient, whichever tokens
// there are: of the last ids, which are the rare ones where ids are numbered by how often they come.

// Ranks of this wave's ITEMS x 64 digits (item k of lane l is number 64 k + l) among those before with the same digit;
// count: the wave's own counters, zeros before.
template <int ITEMS>
__device__ __forceinline__ void wave_ranks(const uint32_t* digit, const bool* real, uint32_t* rank, uint32_t* count, int bits) {
  const int lane = threadIdx.x & 63;
  uint32_t lo[ITEMS], hi[ITEMS], base[ITEMS];  // the lanes of the same digit
  int first[ITEMS];
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    const uint64_t m = __ballot(real[k]);
    lo[k] = (uint32_t)m;
    hi[k] = (uint32_t)(m >> 32);
  }
  for (int b = 0; b < bits; ++b)
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const uint32_t one = (uint32_t)__builtin_amdgcn_sbfe((int)digit[k], b, 1);  // all of its bits
      const uint64_t m = __ballot(one != 0);
      lo[k] &= ~((uint32_t)m ^ one);
      hi[k] &= ~((uint32_t)(m >> 32) ^ one);
    }
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    first[k] = !real[k] ? lane : lo[k] ? __ffs((int)lo[k]) - 1 : __ffs((int)hi[k]) + 31;
    base[k] = 0;
    if (real[k] && lane == first[k]) base[k] = atomicAdd(&count[digit[k]], (uint32_t)(__popc(lo[k]) + __popc(hi[k])));
  }
#pragma unroll
  for (int k = 0; k < ITEMS; ++k)
    rank[k] = __shfl(base[k], first[k], 64) + __builtin_amdgcn_mbcnt_hi(hi[k], __builtin_amdgcn_mbcnt_lo(lo[k], 0));
}

// The waves' counts of each digit to where their tokens of it begin: behind `before`, the wave before and all smaller digits.
// total: of the digit, in all waves. For the first 512 threads, one a digit.
__device__ __forceinline__ uint32_t waves_total(const uint32_t (*count)[kDigits], uint32_t* c) {
  uint32_t total = 0;
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) c[w] = count[w][threadIdx.x];
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) total += c[w];
  return total;
}
__device__ __forceinline__ void waves_begin(uint32_t (*count)[kDigits], const uint32_t* c, uint32_t before) {
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) {
    count[w][threadIdx.x] = before;
    before += c[w];
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
  if (blockIdx.x) return fill_rows(a, a.filled, a.vocab, blockIdx.x - 1, gridDim.x - 1);
  __shared__ uint32_t keys[kSortThreads * ITEMS], pos[kSortThreads * ITEMS];
  __shared__ uint32_t count[kSortWaves][kDigits];
  __shared__ uint32_t tmp[8];
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63, T = (int)a.tokens;
  const int at = wave * 64 * ITEMS + lane;
  const int digits = 1 << a.digits;
  uint32_t key[ITEMS], p[ITEMS], rank[ITEMS], digit[ITEMS];
  bool real[ITEMS];
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    p[k] = at + 64 * k;
    real[k] = (int)p[k] < T;
  }
  ids_of<ITEMS>(a, key, [&](int k) { return min((int)p[k], T - 1); });
  for (int pass = 0; pass < a.passes; ++pass) {
    for (int i = lane; i < digits; i += 64) count[wave][i] = 0;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) digit[k] = key[k] >> (pass * a.digits) & ((1u << a.digits) - 1);
    __syncthreads();
    wave_ranks<ITEMS>(digit, real, rank, count[wave], a.digits);
    __syncthreads();
    uint32_t c[kSortWaves];
    const uint32_t before = scan512(t < digits ? waves_total(count, c) : 0, tmp);
    if (t < digits) waves_begin(count, c, before);
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

// The keys of K tokens at a pass, at places that exist.
template <int K, class At>
__device__ __forceinline__ void sort_keys(const EmbeddingArgs& a, int pass, uint32_t* key, At at) {
  if (pass == 0) return ids_of<K>(a, key, at);
#pragma unroll
  for (int k = 0; k < K; ++k) key[k] = a.keys[pass & 1][at(k)];
}

// Several workgroups: how often each digit stands in each block's tokens.
template <int ITEMS>
__global__ __launch_bounds__(kSortThreads) void embedding_count_kernel(EmbeddingArgs a, int pass, int blocks, int64_t v0, int64_t v1) {
  if ((int)blockIdx.x >= blocks) return fill_rows(a, v0, v1, blockIdx.x - blocks, gridDim.x - blocks);
  __shared__ uint32_t count[kDigits];
  const int t = threadIdx.x;
  if (t < kDigits) count[t] = 0;
  __syncthreads();
  const int64_t at = (int64_t)blockIdx.x * kSortThreads * ITEMS + t;
  uint32_t key[ITEMS];
  sort_keys<ITEMS>(a, pass, key, [&](int k) { return min(at + k * kSortThreads, a.tokens - 1); });
#pragma unroll
  for (int k = 0; k < ITEMS; ++k)
    if (at + k * kSortThreads < a.tokens) atomicAdd(&count[key[k] >> (pass * a.digits) & ((1u << a.digits) - 1)], 1u);
  __syncthreads();
  if (t < kDigits) a.hist[(int64_t)blockIdx.x * kDigits + t] = count[t];
}

// ... and each block's tokens to their places of this pass.
template <int ITEMS>
__global__ __launch_bounds__(kSortThreads) void embedding_move_kernel(EmbeddingArgs a, int pass, int blocks, int64_t v0, int64_t v1) {
  if ((int)blockIdx.x >= blocks) return fill_rows(a, v0, v1, blockIdx.x - blocks, gridDim.x - blocks);
  __shared__ uint32_t count[kSortWaves][kDigits];
  __shared__ uint32_t tmp[8];
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
  const int64_t at = (int64_t)blockIdx.x * kSortThreads * ITEMS + wave * 64 * ITEMS + lane;
  uint32_t key[ITEMS], p[ITEMS], rank[ITEMS], digit[ITEMS];
  bool real[ITEMS];
  for (int i = lane; i < kDigits; i += 64) count[wave][i] = 0;
  auto place = [&](int k) { return min(at + 64 * k, a.tokens - 1); };
  sort_keys<ITEMS>(a, pass, key, place);
  if (pass) {
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) p[k] = a.pos[pass & 1][place(k)];
  } else {
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) p[k] = (uint32_t)place(k);
  }
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    real[k] = at + 64 * k < a.tokens;
    digit[k] = key[k] >> (pass * a.digits) & ((1u << a.digits) - 1);
  }
  __syncthreads();
  wave_ranks<ITEMS>(digit, real, rank, count[wave], a.digits);
  __syncthreads();
  uint32_t total = 0, mine = 0;  // of this digit: in all blocks, in those before
  if (t < kDigits)
#pragma unroll 8
    for (int b = 0; b < blocks; ++b) {
      const uint32_t c = a.hist[(int64_t)b * kDigits + t];
      total += c;
      mine += b < (int)blockIdx.x ? c : 0;
    }
  const uint32_t before = scan512(t < kDigits ? total : 0, tmp) + mine;
  if (t < kDigits) {
    uint32_t c[kSortWaves];
    waves_total(count, c);
    waves_begin(count, c, before);
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

template <class G, int N, int V, bool ODD = true>
__device__ __forceinline__ void write_row(const EmbeddingArgs& a, int64_t id, const Span<N>* s, float* sum) {
  G* g = (G*)a.grad + id * a.cols;
#pragma unroll
  for (int v = 0; v < V; ++v) {
#pragma unroll
    for (int e = 0; e < N; ++e) sum[N * v + e] *= a.scale;
    if (a.add) {
      Cols<G, N> old;
      load_cols<ODD>(old, (const G*)g, s[v]);
#pragma unroll
      for (int e = 0; e < N; ++e) sum[N * v + e] += old[e];
    }
    store_cols<ODD>(g, sum + N * v, s[v]);
  }
}

// Waits for all loads at once. Loads and stores are counted by one counter, and whether a row is written between two tokens only the
// keys say: left to itself, the compiler waits for everything, the stores' round trips too, before each next token.
__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0f70); }  // vmcnt(0), the other counters as they are

// Zeros to those of the rows [v0, v0 + kFillRows) whose lane says that no token met them.
template <class G, bool ONCE>
__device__ __forceinline__ void zero_rows(const EmbeddingArgs& a, int64_t v0, bool unmet) {
  const int waves = blockDim.x >> 6, lane = threadIdx.x & 63;
  uint64_t rows = __ballot(unmet);
  constexpr int M = 16 / sizeof(G);
  const float zero[M] = {};
  if (a.cols % M == 0) {  // rows of whole vectors: one behind the other
    const int per = a.cols / M, n = rows ? (64 - __builtin_clzll(rows)) * per : 0;
    G* g = (G*)a.grad + v0 * a.cols;
    for (int i = threadIdx.x; i < n; i += blockDim.x)
      if (rows >> (i / per) & 1) put<ONCE, M>(g + (int64_t)i * M, zero);
    return;
  }
  for (int i = 0; rows; ++i, rows &= rows - 1) {
    if (i % waves != (int)(threadIdx.x >> 6)) continue;
    G* g = (G*)a.grad + (v0 + __ffsll((unsigned long long)rows) - 1) * a.cols;
    for (int c = lane * M; c < a.cols; c += 64 * M) store_cols<true, ONCE>(g, zero, span_at<M>(c, a.cols));
  }
}

// ... of those before `filled`, by the sorted tokens.
template <class G, bool ONCE>
__device__ __forceinline__ void fill_unmet(const EmbeddingArgs& a, int64_t v0) {
  const uint32_t* keys = a.keys[0];
  const int64_t id = v0 + (threadIdx.x & 63);
  bool unmet = false;
  if (id < a.filled) {
    const int64_t i = lower(keys, 0, a.tokens, (uint32_t)id);
    unmet = i == a.tokens || keys[i] != (uint32_t)id;
  }
  zero_rows<G, ONCE>(a, v0, unmet);
}

// Up to 64 tokens, without a sort: every wave has all of them in its lanes. A workgroup for each token sums the rows of all that
// have its id, in order, if it is the first of these; the others write zeros to `fill` rows each.
template <class D, class G, bool ONCE>
__global__ __launch_bounds__(1024) void embedding_few_kernel(EmbeddingArgs a, int fill) {
  constexpr int N = Form<D, G>::N, V = Form<D, G>::V, U = 8;  // U: rows of a thread in flight
  const int T = (int)a.tokens, lane = threadIdx.x & 63, t = blockIdx.x;
  uint32_t key[1];
  ids_of<1>(a, key, [&](int) { return (int64_t)min(lane, T - 1); });
  if (t >= T) {
    const int64_t v0 = (int64_t)(t - T) * fill, id = v0 + lane;
    bool unmet = lane < fill && id < a.vocab;
    for (int j = 0; j < T; ++j) unmet = unmet && (uint32_t)__builtin_amdgcn_readlane(key[0], j) != (uint32_t)id;
    return zero_rows<G, ONCE>(a, v0, unmet);
  }
  const uint32_t id = __builtin_amdgcn_readlane(key[0], t);
  uint64_t mine = __ballot(lane < T && key[0] == id);
  if (id >= (uint32_t)a.vocab || __ffsll((unsigned long long)mine) - 1 != t) return;
  Span<N> s[V];
  spans_of<N, V>(s, threadIdx.x, blockDim.x, a.cols);
  float sum[8] = {};
  while (mine) {
    const int n = __popcll(mine);
    Cols<D, N> r[U][V];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = mine ? __ffsll((unsigned long long)mine) - 1 : t;  // behind the last, one that is there already
      mine &= mine - 1;
#pragma unroll
      for (int v = 0; v < V; ++v) load_cols(r[u][v], (const D*)a.dout + at * a.dout_stride, s[v]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (u < n)
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int e = 0; e < N; ++e) sum[N * v + e] += r[u][v][e];
  }
  write_row<G, N, V>(a, id, s, sum);
}

// The first `sums` workgroups sum shares of the sorted tokens, the others write zeros. `across` threads a share; WHOLE: these are whole
// waves, whose keys and positions lie in their lanes, 64 at a time, so that every row's address is a scalar and 16 rows are in
// flight behind one load of positions. ODD: rows may end within a vector. (The code that writes a row stands behind each of the rows in
// flight, and with that of odd ends it is more than the instruction cache holds.)
template <class D, class G, bool WHOLE, bool ODD, bool ONCE>
__global__ __launch_bounds__(1024) void embedding_sum_kernel(EmbeddingArgs a, int sums, int across) {
  constexpr int N = Form<D, G>::N, V = Form<D, G>::V, U = WHOLE && !ODD && sizeof(D) == 2 ? 16 : 8;  // U: rows of a thread in flight
  if ((int)blockIdx.x >= sums) return fill_unmet<G, ONCE>(a, ((int64_t)blockIdx.x - sums) * kFillRows);
  const uint32_t *keys = a.keys[0], *pos = a.pos[0];
  const uint32_t none = (uint32_t)a.vocab;
  const int64_t T = a.tokens;
  const int shares = blockDim.x / across, ty = WHOLE ? __builtin_amdgcn_readfirstlane(threadIdx.x / across) : threadIdx.x / across;
  const int64_t c = (int64_t)blockIdx.x * shares + ty;
  if (ty >= shares || c >= a.chunks) return;
  Span<N> s[V];
  spans_of<N, V>(s, threadIdx.x - ty * across, across, a.cols);
  const int64_t i0 = c * a.chunk, i1 = min(T, i0 + a.chunk);
  uint32_t cur = keys[i0];
  bool from = i0 > 0 && keys[i0 - 1] == cur;  // goes on from the share before
  float sum[8] = {};
  float* part = a.part + c * 2 * a.cols;
  auto done = [&](bool on) {  // on: goes on in the next share
    if (cur >= none) return;
    if (from || on) {
#pragma unroll
      for (int v = 0; v < V; ++v) store_cols<ODD>(from ? part : part + a.cols, sum + N * v, s[v]);
    } else {
      write_row<G, N, V, ODD>(a, cur, s, sum);
    }
  };
  auto add = [&](uint32_t k, const Cols<D, N>* r) {
    if (k != cur) {
      done(false);
      cur = k;
      from = false;
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < N; ++e) sum[N * v + e] += r[v][e];
  };
  // the rows of tokens that have no id are not read; they stand behind all others
  if constexpr (WHOLE) {
    const int lane = threadIdx.x & 63;
    for (int64_t i = i0; i < i1; i += 64) {
      const int n = (int)min((int64_t)64, i1 - i);
      const int64_t at = i + min(lane, n - 1);
      const uint32_t ks = keys[at], ps = pos[at];
      const int real = __popcll(__ballot(ks < none && lane < n));
      for (int u0 = 0; u0 < real; u0 += U) {
        Cols<D, N> r[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const uint32_t p = __builtin_amdgcn_readlane(ps, min(u0 + u, real - 1));
#pragma unroll
          for (int v = 0; v < V; ++v) load_cols<false, ONCE>(r[u][v], (const D*)a.dout + (int64_t)p * a.dout_stride, s[v]);
        }
        wait_loads();
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (u0 + u >= real) break;
          add(__builtin_amdgcn_readlane(ks, u0 + u), r[u]);
        }
      }
      if (real < n) {  // the last id ends here
        done(false);
        return;
      }
    }
  } else {
    for (int64_t i = i0; i < i1; i += U) {
      uint32_t k[U];
      Cols<D, N> r[U][V];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t at = min(i + u, i1 - 1);
        k[u] = keys[at];
#pragma unroll
        for (int v = 0; v < V; ++v) {
          r[u][v] = Cols<D, N>{};
          if (k[u] < none) load_cols(r[u][v], (const D*)a.dout + (int64_t)pos[at] * a.dout_stride, s[v]);
        }
      }
      wait_loads();
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i + u >= i1) break;
        add(k[u], r[u]);
      }
    }
  }
  done(i1 < T && keys[i1] == cur);
}

constexpr int kJoinThreads = 32, kJoinRuns = 8;  // of a workgroup that joins 256 columns of a row

// The row of an id whose tokens begin in share c and go on beyond it: its sums of all shares, in order.
template <class G>
__global__ __launch_bounds__(kJoinThreads * kJoinRuns) void embedding_join_kernel(EmbeddingArgs a) {
  __shared__ float sums[8][kJoinRuns][kJoinThreads];
  const uint32_t* keys = a.keys[0];
  const int64_t T = a.tokens, c = blockIdx.x, i0 = c * a.chunk, i1 = i0 + a.chunk;
  if (i1 >= T) return;
  const int t = threadIdx.x, y = threadIdx.y, lane = (y * kJoinThreads + t) & 63;
  const int64_t behind = i1 + (int64_t)lane * a.chunk;
  const uint32_t id = keys[i1 - 1], next = keys[i1], begin = keys[i0], before = keys[max(i0 - 1, (int64_t)0)];
  uint32_t first = keys[min(behind, T - 1)];
  if (id >= (uint32_t)a.vocab || next != id || (begin == id && i0 > 0 && before == id)) return;
  int count = 1;  // shares of this id: those behind begin with it; 64 of them a step
  for (int64_t at = behind;;) {
    const uint64_t other = ~__ballot(at < T && first == id);
    count += other ? __ffsll((unsigned long long)other) - 1 : 64;
    if (other) break;
    at += (int64_t)64 * a.chunk;
    first = keys[min(at, T - 1)];
  }
  Span<4> s[2];
#pragma unroll
  for (int v = 0; v < 2; ++v) s[v] = span_at<4>((blockIdx.y * 64 + v * kJoinThreads + t) * 4, a.cols);
  const int per = (count + kJoinRuns - 1) / kJoinRuns, last = min(count, (y + 1) * per);
  float sum[8] = {};
#pragma unroll 8
  for (int j = y * per; j < last; ++j)
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      Cols<float, 4> r;
      load_cols(r, (const float*)a.part + (c + j) * 2 * a.cols + (j ? 0 : a.cols), s[v]);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[4 * v + e] += r[e];
    }
#pragma unroll
  for (int e = 0; e < 8; ++e) sums[e][y][t] = sum[e];
  __syncthreads();
  if (y) return;
#pragma unroll
  for (int k = 1; k < kJoinRuns; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] += sums[e][k][t];
  write_row<G, 4, 2>(a, id, s, sum);
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
// Whether a call's streams (a lookup's output; the zeros beside the sort and the rows of dout) go past the caches: where these are in the
// way of what is used again, rows of the table or of the gradient. ids as words come, bf16 rows, us without and with, alternating
// with the other direction and by themselves: 65,536 x 1,536 lookups (384 MiB read and written) 62 and 46, 32,768 (192) 26 and 25; gradients of
// 65,536 tokens in 32,128 x 1,536 fp32 (380 MiB) 128 and 110, with the lookup 208 and 154; of 30,000 in 60,000 x 1,024 bf16 (176) 60 and 60, 87 and 74;
// of 8,192 in 32,128 x 1,024 fp32 (142) 35 and 42, 44 and 50. Not where a thread's vector takes two instructions, half of a line each.
constexpr int64_t kOnceFwd = (int64_t)256 << 20, kOnceBwd = (int64_t)160 << 20;
template <class X, class Y>
constexpr bool kWholeLines = sizeof(X) * Form<X, Y>::N <= 16;
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
  // about 1,024 shares: 65,536 tokens as above take sums of 71 us and joins of 10, with 2,048 of them 77 and 15 (an id's shares are joined in a row)
  p.chunk = (int)std::max<int64_t>(8, (tokens + 8 * 1024 - 1) / (8 * 1024) * 8);
  p.chunks = (int)((tokens + p.chunk - 1) / p.chunk);
  return p;
}

hipError_t launch_embedding_fwd(const EmbeddingArgs& a, hipStream_t s) {
  const int threads = row_threads(a.cols, kRowThreads), rows = threads / ((a.cols + 7) / 8);
  const int64_t blocks = std::min<int64_t>(4096, (a.tokens + rows - 1) / rows);
  const bool once = a.tokens * a.cols * ((a.table_f32 ? 4 : 2) + (a.out_f32 ? 4 : 2)) > kOnceFwd;
  pick(a.table_f32, a.out_f32, [&](auto t, auto o) {
    using T = decltype(t);
    using O = decltype(o);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(threads), 0, s, a); };
    if constexpr (kWholeLines<O, T>)
      if (once) return launch(embedding_fwd_kernel<T, O, true>);
    launch(embedding_fwd_kernel<T, O, false>);
  });
  return hipGetLastError();
}

hipError_t launch_embedding_bwd(EmbeddingArgs a, hipStream_t s) {
  const EmbeddingPlan p = embedding_plan(a.tokens, a.vocab, a.cols);
  a.passes = p.passes;
  a.digits = p.digits;
  a.chunk = p.chunk;
  a.chunks = p.chunks;
  a.once = a.cols * (a.tokens * (a.out_f32 ? 4 : 2) + a.vocab * (a.grad_f32 ? 4 : 2)) > kOnceBwd;
  const int64_t row_bytes = (int64_t)a.cols * (a.grad_f32 ? 4 : 2);
  const int few_threads = std::max(kRowThreads, ((a.cols + 7) / 8 + 63) / 64 * 64);
  const int fill_each = (int)std::min<int64_t>(64, std::max<int64_t>(1, kFewFill / row_bytes));
  const int64_t few_groups = a.tokens + (a.add ? 0 : (a.vocab + fill_each - 1) / fill_each);
  if (a.tokens <= kFewTokens && few_groups * few_threads < (int64_t)1 << 32) {  // a launch has less threads than that
    pick(a.out_f32, a.grad_f32, [&](auto d, auto g) {
      auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(few_groups), dim3(few_threads), 0, s, a, fill_each); };
      if (a.once)
        launch(embedding_few_kernel<decltype(d), decltype(g), true>);
      else
        launch(embedding_few_kernel<decltype(d), decltype(g), false>);
    });
    return hipGetLastError();
  }
  // Rows that the sort's launches write zeros to: as many as take about the time of the sort.
  const int64_t most = p.blocks == 1 ? kFillOne : kFillPass * p.passes;
  a.filled = a.add ? a.vocab : std::max<int64_t>(0, a.vocab - most / row_bytes);
  auto fills = [&](int64_t rows) { return (int)std::min<int64_t>(kFillGroups, (rows * row_bytes + 65535) / 65536); };
  if (p.blocks == 1) {
    const dim3 grid(1 + fills(a.vocab - a.filled));
    if (a.tokens <= 1024)
      hipLaunchKernelGGL(embedding_sort_one_kernel<1>, grid, dim3(kSortThreads), 0, s, a);
    else if (a.tokens <= 4096)
      hipLaunchKernelGGL(embedding_sort_one_kernel<4>, grid, dim3(kSortThreads), 0, s, a);
    else
      hipLaunchKernelGGL(embedding_sort_one_kernel<8>, grid, dim3(kSortThreads), 0, s, a);
  } else {
    const int64_t rows = a.vocab - a.filled;
    int64_t v0 = a.filled;
    for (int k = 0; k < 2 * p.passes; ++k) {
      const int64_t v1 = a.filled + rows * (k + 1) / (2 * p.passes);
      const dim3 grid(p.blocks + fills(v1 - v0));
      const int pass = k / 2;
      auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kSortThreads), 0, s, a, pass, p.blocks, v0, v1); };
      if (items(a.tokens) == 4) {
        if (k % 2)
          launch(embedding_move_kernel<4>);
        else
          launch(embedding_count_kernel<4>);
      } else {
        if (k % 2)
          launch(embedding_move_kernel<16>);
        else
          launch(embedding_count_kernel<16>);
      }
      v0 = v1;
    }
    if (p.passes & 1) {  // the last pass wrote the second of the two
      std::swap(a.keys[0], a.keys[1]);
      std::swap(a.pos[0], a.pos[1]);
    }
  }
  // Shares of whole waves where a row takes more than half of one.
  const int least = (a.cols + 7) / 8, across = least > 32 ? (least + 63) / 64 * 64 : least;
  const int threads = least > 32 ? std::max(across, 256 / across * across) : 256, shares = threads / across;
  const int sums = (p.chunks + shares - 1) / shares;
  const int fill = a.add ? 0 : (int)((a.filled + kFillRows - 1) / kFillRows);
  pick(a.out_f32, a.grad_f32, [&](auto d, auto g) {
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(sums + fill), dim3(threads), 0, s, a, sums, across); };
    using D = decltype(d);
    using G = decltype(g);
    if (least <= 32) return launch(embedding_sum_kernel<D, G, false, true, false>);
    if constexpr (kWholeLines<D, G>)
      if (a.once)
        return a.cols % Form<D, G>::N ? launch(embedding_sum_kernel<D, G, true, true, true>) : launch(embedding_sum_kernel<D, G, true, false, true>);
    if (a.cols % Form<D, G>::N)
      launch(embedding_sum_kernel<D, G, true, true, false>);
    else
      launch(embedding_sum_kernel<D, G, true, false, false>);
  });
  if (p.chunks > 1) {
    const dim3 grid(p.chunks, (a.cols + 255) / 256), block(kJoinThreads, kJoinRuns);
    if (a.grad_f32)
      hipLaunchKernelGGL(embedding_join_kernel<float>, grid, block, 0, s, a);
    else
      hipLaunchKernelGGL(embedding_join_kernel<__bf16>, grid, block, 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace vcja
