// Device-side types and helpers shared by the packed-attention kernels (gfx950).
#pragma once

#include "common.hpp"

namespace vcja {

constexpr int kPackedWaves = 4;                  // of a workgroup
constexpr int kPackedRows = 32 * kPackedWaves;   // query rows (keys) that it owns
constexpr int kMaxBiasDistance = 512;  // largest relative distance with a bucket of its own
constexpr int kMaxBuckets = 1024;
constexpr float kBiasLimit = 65536.0f;  // bias entries below -this shut their pairs out

// Kernel arguments of the packed attention. Sequence s has the query slot [cu_q[s], cu_q[s+1])
// of the Tq rows and the key slot [cu_k[s], cu_k[s+1]) of the Tk rows; the first len_q[s] and
// len_k[s] rows of them (all without the arrays) take part.
struct PackedArgs {
  const __bf16 *q, *k, *v;
  const __bf16* dout;  // backward
  const __bf16* o_in;  // backward: the forward's O
  __bf16 *o, *dq, *dk, *dv;
  float* lse;          // [H, Tq]; the backward reads it
  const int32_t *cu_q, *cu_k, *len_q, *len_k;
  const __bf16* bias;      // [H, nb] or NULL
  const int32_t* buckets;  // [2 R + 1], of the distances -R .. R
  int nb, R;
  int S, H, Hkv, G;        // G = H / Hkv query heads per key head
  int Tq, Tk, max_q, max_k;
  unsigned q_tok, k_tok, v_tok;  // elements between the rows of consecutive tokens
  int causal, clear;  // clear: rows outside every slot, 1 of all outputs (forward: 2 of o, 3 of lse alone)
  float scale, scale_log2;  // softmax scale; times log2(e)
  int nblk, blocks;         // row blocks of the longest slot; of all slots in a grid
  bool compact;             // blocks numbered through (see packed_item)
  int chunks;               // workgroups that share a row block's key tiles (backward: a key block's query tiles)
  int dq_chunks;            // backward: workgroups that share a row block's key tiles
  int pack, span;           // forward: heads of a group in one row block; key tiles of a chunk (dQ pass: of dq_chunks)
  bool few;                 // forward: all rows of a (sequence, key head) in one wave's 32
  float* part;              // forward: the chunks' partial results (see write_partial); dQ pass: [dq_chunks][Tq, H][D] of
                            // dQ / scale, then [dq_chunks][Tq, H] sums of dS
  float* key_part;          // their partial dK, dV: [chunks][2][Tk, Hkv, D]
  // Backward: per query row -LSE / c (-inf on padding) and -D, [H, npad], sequence s from row
  // packed_row(cu_q[s], s) on.
  float *nls, *dd;
  int npad;
  float* dist_part;         // bias gradient: sums per distance, [dist_row][Hkv][chunks][2 R + 1]
};

// A pointer that is the same for the whole wave, in scalar registers.
template <class T>
__device__ __forceinline__ T* uniform_ptr(T* p) {
  const uint64_t x = (uint64_t)p;
  const uint64_t lo = (unsigned)__builtin_amdgcn_readfirstlane((unsigned)x), hi = (unsigned)__builtin_amdgcn_readfirstlane((unsigned)(x >> 32));
  return (T*)(lo | hi << 32);
}

__device__ __forceinline__ float uniform(float x) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x))); }

// The rows of one sequence. Whatever the offsets hold, they stay inside the tensors.
struct SeqRows {
  int q0, sq, nq;  // first row, rows of the slot, rows that take part
  int k0, sk, nk;
  int off;         // query i stands at position i + off of the keys: the last at the last key
};
// (`s` the same for the whole wave.)
__device__ __forceinline__ SeqRows seq_rows(const PackedArgs& a, int s) {
  // the same for the whole wave: in scalar registers
  auto at = [&](const int32_t* p, int i) { return __builtin_amdgcn_readfirstlane(p[i]); };
  SeqRows r;
  r.q0 = min(max(at(a.cu_q, s), 0), a.Tq);
  r.sq = min(max(at(a.cu_q, s + 1), r.q0), a.Tq) - r.q0;
  r.sq = min(r.sq, a.max_q);
  r.nq = a.len_q ? min(max(at(a.len_q, s), 0), r.sq) : r.sq;
  r.k0 = min(max(at(a.cu_k, s), 0), a.Tk);
  r.sk = min(max(at(a.cu_k, s + 1), r.k0), a.Tk) - r.k0;
  r.sk = min(r.sk, a.max_k);
  r.nk = a.len_k ? min(max(at(a.len_k, s), 0), r.sk) : r.sk;
  r.off = r.nk - r.nq;
  return r;
}
// Row of query i; past the sequence's own rows its last one (never another's: those may hold
// anything), and some row of the tensor where there is none.
__device__ __forceinline__ int query_row(const PackedArgs& a, const SeqRows& r, int i) {
  return min(r.q0 + max(min(i, r.nq - 1), 0), a.Tq - 1);
}
// First row of sequence s in the padded row statistics: a multiple of 64, at least the
// sequence's rows rounded up to 64 before the next one's.
__host__ __device__ constexpr int packed_row(int q0, int s) { return ((q0 + 63) & ~63) + 64 * s; }
__host__ __device__ constexpr int64_t packed_rows(int64_t Tq, int64_t S) { return ((Tq + 63) & ~(int64_t)63) + 64 * (S + 1) + 256; }

// Row of the bias gradient's per-distance sums for block `blk` (of bm keys) of the sequence whose
// keys start at k0: a sequence's blocks lie one behind the other, at most Tk / bm + S rows in all, and
// a sequence's rows end at or before the next one's first. (Rows between: zeros.)
__host__ __device__ constexpr int64_t dist_row(int64_t k0, int s, int blk, int bm) { return k0 / bm + s + blk; }

// The sequence that holds block c of the blocks of kPackedRows tokens laid one behind the other (sequence
// s from block cu[s] / kPackedRows + s on), -1 before the first. By the whole wave: 64 sequences a step.
__host__ __device__ constexpr int64_t packed_blocks(int64_t total, int64_t S) { return total / kPackedRows + S; }
__device__ __forceinline__ int find_sequence(const int32_t* cu, int S, int total, int c) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = S;
  for (;;) {
    const int step = (n + 63) / 64, l = min(lo + lane * step, S - 1);
    const int first = min(max(cu[l], 0), total) / kPackedRows + l;
    const int k = __popcll(__ballot(lane * step < n && first <= c)) - 1;
    if (k < 0) return -1;
    lo += k * step;
    if (step == 1) return __builtin_amdgcn_readfirstlane(lo);
    n = min(step, n - k * step);
  }
}

// One (row block, head, sequence) of a 1-D grid: heads and sequences run fastest, key heads before the
// query heads of a group, so that (with 8 key heads or a multiple) the workgroups that read a key
// head's rows sit on one XCD; with `last_first` the last row blocks, the longest under the causal rule,
// are dispatched first. Where one long slot beside short ones would leave most of such a grid empty
// (a.compact), the blocks are numbered through instead and each workgroup looks its sequence up: one
// sequence of 8,192 tokens with 200 of 60, 16 heads, D = 128, forward 520 -> 326 us; a search costs every
// workgroup about a microsecond.
struct PackedItem {
  int blk, h, s;  // s < 0: none
};
__device__ __forceinline__ PackedItem packed_item(const PackedArgs& a, int x, const int32_t* cu, int total, int Hkv, int G,
                                                  bool last_first) {
  const int H = Hkv * G;
  PackedItem r;
  if (!a.compact) {
    const int HS = H * a.S, p = x % HS;
    r.blk = x / HS;
    if (last_first) r.blk = a.nblk - 1 - r.blk;
    r.s = p / H;
  } else {
    const int i = x / H, c = last_first ? a.blocks - 1 - i : i;
    r.s = find_sequence(cu, a.S, total, c);
    r.blk = r.s < 0 ? 0 : c - __builtin_amdgcn_readfirstlane(min(max(cu[r.s], 0), total) / kPackedRows) - r.s;
  }
  const int hx = x % H;
  r.h = (hx % Hkv) * G + hx / Hkv;
  return r;
}

// Bias of one head per distance in LDS, divided by the softmax scale (the scores' own unit):
// entry kBiasPad + R + d for distance d = key position - query position, distances past +-R
// repeating the last, so that no tile that holds a distance inside (-R, R) reads outside. The
// kernels come with tables for distances up to 128 and up to kMaxBiasDistance, as the wide one
// (and the sums per distance, backward) leaves room for fewer workgroups.
constexpr int kSmallBiasDistance = 128;
constexpr int kBiasPad = 96;  // >= 63 + 31, the distances in a tile of 64 keys x 32 queries
template <int RMAX>
struct BiasTable {
  static constexpr int N = 2 * RMAX + 1 + 2 * kBiasPad;
  static constexpr int ROW = 256;  // buckets whose values are loaded along with the bucket numbers
  float tb[N], row[ROW];
  // By the whole workgroup; ends with the table readable.
  __device__ __forceinline__ void load(const PackedArgs& a, int h, int tid, int threads) {
    const __bf16* bias = a.bias + (size_t)h * a.nb;
    const bool staged = a.nb <= ROW;
    int u[(N + 255) / 256];
#pragma unroll
    for (int j = 0; j < (N + 255) / 256; ++j) u[j] = a.buckets[min(max(tid + j * threads - kBiasPad, 0), 2 * a.R)];
    if (staged && tid < a.nb) row[tid] = (float)bias[tid];
    __syncthreads();
    const float inv = 1.0f / a.scale;
#pragma unroll
    for (int j = 0; j < (N + 255) / 256; ++j) {
      const int i = tid + j * threads;
      float b = 0.0f;
      if (u[j] >= 0 && u[j] < a.nb) b = staged ? row[u[j]] : (float)bias[u[j]];
      b = b < -kBiasLimit ? -INFINITY : b > kBiasLimit ? kBiasLimit : b;  // a NaN stays one
      if (i < N) tb[i] = b * inv;
    }
    __syncthreads();
  }
};
template <>
struct BiasTable<0> {  // no bias
  float tb[1];
  __device__ __forceinline__ void load(const PackedArgs&, int, int, int) {}
};

// Where a block of keys [k0, k1] stands to a block of query positions [p0, p1]: every distance
// at or past R (1), at or before -R (-1), or some inside (0).
__device__ __forceinline__ int bias_side(int k0, int k1, int p0, int p1, int R) {
  return k0 - p1 >= R ? 1 : k1 - p0 <= -R ? -1 : 0;
}

}  // namespace vcja

// Host-side launchers.
namespace vcja {
// The row blocks of a grid over S slots of at most `longest` tokens, `total` in all. A search of the sequence is
// worth its time where it saves half of the workgroups and more than a round of them.
struct RowBlocks {
  int64_t longest, blocks;  // of the longest slot; of all slots in the grid
  bool compact;             // numbered through
};
inline RowBlocks row_blocks(int64_t longest, int64_t total, int64_t S, int64_t Hkv) {
  RowBlocks r;
  r.longest = (longest + kPackedRows - 1) / kPackedRows;
  const int64_t all = r.longest * S, through = packed_blocks(total, S);
  r.compact = all > 2 * through && (all - through) * Hkv > 1024;
  r.blocks = r.compact ? through : all;
  return r;
}
inline void set_blocks(PackedArgs& a, int64_t longest, int64_t total) {
  const RowBlocks r = row_blocks(longest, total, a.S, a.Hkv);
  a.nblk = (int)r.longest;
  a.compact = r.compact;
  a.blocks = (int)r.blocks;
}
constexpr int kClearGroups = 32;  // workgroups of a grid that clear the rows outside every slot
hipError_t launch_packed_fwd(const PackedArgs& a, int head_dim, hipStream_t s);
hipError_t launch_packed_bwd(const PackedArgs& a, int head_dim, __bf16* dbias, hipStream_t s);
}  // namespace vcja
