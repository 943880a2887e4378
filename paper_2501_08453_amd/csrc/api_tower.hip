// Host side of the packed attention's and the layer norm's entry points: argument
// validation, workspace layout, launches. Nothing here allocates, frees or synchronises.
#include <math.h>

#include <algorithm>

#include "host.hpp"
#include "norm.hpp"
#include "packed.hpp"

namespace {

using vcja::aligned16;
using vcja::aligned4;

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
inline hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }
inline const __bf16* bf(const void* p) { return static_cast<const __bf16*>(p); }

// A launch takes less than 2^32 threads: workgroups of 256 beside those that clear, waves of a merge.
constexpr int64_t kMaxGroups = (((int64_t)1 << 32) - 1) / 256;
constexpr int64_t kMaxGrid = kMaxGroups - vcja::kClearGroups;
constexpr int64_t kMaxWaves = 4 * kMaxGroups;
constexpr int64_t kMaxRows = (int64_t)1 << 30;
constexpr int64_t kMaxStride = (int64_t)1 << 23;  // elements between tokens: tile offsets of 16 rows stay in 32 bits

int64_t stride_of(int64_t given, int64_t heads, int64_t d) { return given ? given : heads * d; }

vc_status check_packed(const vc_packedattn_desc* d) {
  if (!d) return VC_ERR_NULL;
  if (d->head_dim != 64 && d->head_dim != 128) return VC_ERR_HEAD_DIM;
  if (d->sequences < 1 || d->heads < 1 || d->kv_heads < 1 || d->heads % d->kv_heads) return VC_ERR_SHAPE;
  if (d->sequences > (1 << 20) || d->heads > 4096) return VC_ERR_SHAPE;
  if (d->total_q < 1 || d->total_q > kMaxRows || d->total_k < 1 || d->total_k > kMaxRows) return VC_ERR_SHAPE;
  if (d->max_q < 1 || d->max_q > d->total_q || d->max_k < 1 || d->max_k > d->total_k) return VC_ERR_SHAPE;
  if ((d->causal & ~1) || (d->clear_outside & ~3)) return VC_ERR_SHAPE;
  const int64_t D = d->head_dim;
  for (const int64_t s : {d->q_stride, d->k_stride, d->v_stride})
    if (s < 0 || s > kMaxStride || s % 8) return VC_ERR_SHAPE;
  if (stride_of(d->q_stride, d->heads, D) < d->heads * D || stride_of(d->k_stride, d->kv_heads, D) < d->kv_heads * D ||
      stride_of(d->v_stride, d->kv_heads, D) < d->kv_heads * D)
    return VC_ERR_SHAPE;
  if (d->num_buckets < 0 || d->num_buckets > vcja::kMaxBuckets || d->max_distance < 0 || d->max_distance > vcja::kMaxBiasDistance)
    return VC_ERR_SHAPE;
  // Scores are formed in units of 1 / c; with a bias that quotient is taken of its entries too.
  if (!(d->softmax_scale <= 0.0f)) {
    const float c = d->softmax_scale, lo = d->num_buckets ? 0x1p-24f : 0x1p-60f, hi = d->num_buckets ? 0x1p24f : 0x1p60f;
    if (!(c >= lo && c <= hi)) return VC_ERR_SHAPE;
  }
  // Row counts of the statistics and workgroup counts stay inside 32 bits.
  const int64_t blocks = (int64_t)d->heads * d->sequences * ((std::max(d->max_q, d->max_k) + 31) / 32);
  if (blocks > ((int64_t)1 << 30) || vcja::packed_rows(d->total_q, d->sequences) > ((int64_t)1 << 31) - 1) return VC_ERR_SHAPE;
  return VC_OK;
}

float scale_of(const vc_packedattn_desc* d) {
  return d->softmax_scale > 0.0f ? d->softmax_scale : 1.0f / sqrtf((float)d->head_dim);
}

vcja::PackedArgs packed_args(const vc_packedattn_desc* d, const void* q, const void* k, const void* v, const int32_t* cu_q,
                             const int32_t* cu_k, const int32_t* len_q, const int32_t* len_k, const void* bias,
                             const int32_t* buckets) {
  vcja::PackedArgs a{};
  a.q = bf(q);
  a.k = bf(k);
  a.v = bf(v);
  a.cu_q = cu_q;
  a.cu_k = cu_k;
  a.len_q = len_q;
  a.len_k = len_k;
  if (d->num_buckets) {
    a.bias = bf(bias);
    a.buckets = buckets;
    a.nb = d->num_buckets;
    a.R = d->max_distance;
  }
  a.S = d->sequences;
  a.H = d->heads;
  a.Hkv = d->kv_heads;
  a.G = d->heads / d->kv_heads;
  a.Tq = (int)d->total_q;
  a.Tk = (int)d->total_k;
  a.max_q = d->max_q;
  a.max_k = d->max_k;
  a.q_tok = (unsigned)stride_of(d->q_stride, d->heads, d->head_dim);
  a.k_tok = (unsigned)stride_of(d->k_stride, d->kv_heads, d->head_dim);
  a.v_tok = (unsigned)stride_of(d->v_stride, d->kv_heads, d->head_dim);
  a.causal = d->causal;
  a.clear = d->clear_outside;
  a.scale = scale_of(d);
  a.scale_log2 = a.scale * vcja::kLog2e;
  a.npad = (int)vcja::packed_rows(d->total_q, d->sequences);
  return a;
}

// Blocks of kPackedRows rows (slots of up to `longest`, `total` in all) as so many of the longest slot's, if the
// other S - 1 sequences share the rest evenly and a block takes time by the other side's tokens.
double equal_blocks(const vc_packedattn_desc* d, int64_t longest, int64_t total, int64_t other_longest, int64_t other_total) {
  const double bm = vcja::kPackedRows, rest = d->sequences - 1;
  double blocks = ceil(longest / bm);
  if (rest > 0) {
    const double mean = std::max<int64_t>(0, total - longest) / rest, other = std::max<int64_t>(0, other_total - other_longest) / rest;
    blocks += rest * ceil(mean / bm) * std::min(1.0, other / other_longest);
  }
  return blocks;
}

// Forward: heads of a group packed into a row block, and the chunks of a row block's key tiles.
struct FwdPlan {
  int pack, chunks, span;
  bool few, fits;  // fits: the launches can be made
};
// The chunks of least estimated time, in tiles of 64 keys x 128 rows (about 1.8 us at head_dim 128, half
// of that at 64): rounds over 512 places, two workgroups a compute unit (at head_dim 64 the forward and dK/dV
// hold three, which the model leaves out), each workgroup 3 tiles
// more than its keys for its start and its partial results, and the merge, a launch of about 6 us and
// the partials' way to memory and back. `blocks` count by their keys (equal_blocks); `uneven` ones (the
// causal rule's, longest first) fill their last round. `cost`:
// receives the estimated time unsplit over the least. Measured, us at 1, 2, 4, 8, 16 chunks (32 heads, 8 key heads, D = 128): 512 queries behind 16,384
// keys -, -, 144, 157, 181; 128 behind 16,384 -, -, -, -, 57 (74 at 32); 4 x 64 behind 500 to 9,000 -, -, 62, 46,
// 57; 8,192 causal at 4 heads 134, 113, 110, 107; two texts of 12 heads at D = 64 41, 48, 45 (3), 51 (5).
int fwd_chunks(const vc_packedattn_desc* d, double blocks, double rows, bool uneven, double* cost = nullptr) {
  const int ntile = (d->max_k + vcja::kTileTok - 1) / vcja::kTileTok;
  const double tile_us = d->head_dim == 128 ? 1.8 : 0.9;
  double least = 1e30;
  int best = 1;
  for (int c = 1; c <= std::min(64, std::max(1, ntile / 4)); ++c) {
    const double span = (ntile + c - 1) / c;
    const double load = blocks * c / 512, rounds = uneven ? std::max(load, 1.0) : ceil(load);
    const double merge = c == 1 ? 0 : (6 + rows * c * (d->head_dim + 2) * 8 / 4e6) / tile_us;
    const double time = rounds * (span + 3) + merge;
    if (time < least * 0.98) {
      least = time;
      best = c;
    }
    if (cost && c == 1) *cost = time;
  }
  if (cost) *cost /= least;
  return best;
}
// The same for the few-row kernel, in ns: a workgroup streams about 50 bytes a ns by itself, 20 beside 256
// others, all of them 5,200, a quarter of the longest one's time passes while the others have ended,
// and each takes 3 us besides. Measured, us at 3, 4, 6, 8, 16 chunks, D = 128, 8 key
// heads: 16 sequences of up to 8,000 keys 75, 66, 53, 55, 56; four of 200 to 8,000 42, 35, 26, 23, 22; 64 of
// 100 to 2,431 73, 74, 76, 76, 78 (70 unsplit).
int few_chunks(const vc_packedattn_desc* d, int64_t rows, int64_t blocks) {
  const int ntile = (d->max_k + vcja::kTileTok - 1) / vcja::kTileTok;
  const double tile = 2.0 * 2 * vcja::kTileTok * d->head_dim;
  const double share = std::min(1.0, (double)d->total_k / ((double)d->sequences * d->max_k));
  const double all = 2.0 * 2 * d->total_k * d->kv_heads * d->head_dim / 5200;
  double least = 1e30;
  int best = 1;
  for (int c = 1; c <= std::min(64, std::max(1, ntile / 2)); c += c < 8 ? 1 : c / 4) {
    const double span = (ntile + c - 1) / c * tile;
    const double merge = c == 1 ? 0 : 6000 + rows * c * (d->head_dim + 2) * 8 / 4000.0;
    const double wgs = blocks * (share * c + 0.5), alone = span / (50 - 30 * std::min(1.0, wgs / 256));
    const double time = std::max(all + alone / 4 + std::max(1.0, wgs / 512) * 3000, alone + 3000) + merge;
    if (time < least * 0.995) {
      least = time;
      best = c;
    }
  }
  return best;
}
vcja::RowBlocks query_blocks(const vc_packedattn_desc* d, int pack) {  // heads packed into a block: one block a slot
  return vcja::row_blocks(pack > 1 ? 1 : d->max_q, d->total_q, d->sequences, d->kv_heads);
}
vcja::RowBlocks key_blocks(const vc_packedattn_desc* d) {
  return vcja::row_blocks(d->max_k, d->total_k, d->sequences, d->kv_heads);
}
// Waves of the kernels that join the chunks: one per (query of a slot, head).
int64_t merge_waves(const vc_packedattn_desc* d, const vcja::RowBlocks& b) {
  return (b.compact ? b.blocks * vcja::kPackedRows : (int64_t)d->sequences * d->max_q) * d->heads;
}
FwdPlan fwd_plan(const vc_packedattn_desc* d) {
  const int group = d->heads / d->kv_heads;
  FwdPlan p;
  p.pack = !d->num_buckets && (int64_t)d->max_q * group <= 128 ? group : 1;
  const int64_t rows = (int64_t)d->max_q * p.pack, bm = vcja::kPackedRows;
  const int64_t blocks = std::min<int64_t>(d->sequences * ((rows + bm - 1) / bm), d->total_q * p.pack / bm + d->sequences) *
                         (d->heads / p.pack);
  const bool uneven = d->causal && 2 * (int64_t)d->max_q > d->max_k;
  const double work = equal_blocks(d, rows, d->total_q * p.pack, d->max_k, d->total_k) * (d->heads / p.pack) * (uneven ? 0.5 : 1.0);
  p.few = rows <= 32;
  const vcja::RowBlocks b = query_blocks(d, p.pack);
  const int64_t grid = (p.few ? d->sequences : b.blocks) * (d->heads / p.pack), outs = d->total_q * d->heads;
  const int ntile = (d->max_k + vcja::kTileTok - 1) / vcja::kTileTok;
  p.chunks = (int)std::max<int64_t>(1, std::min<int64_t>(p.few ? few_chunks(d, outs, blocks) : fwd_chunks(d, work, (double)outs, uneven),
                                                          kMaxGrid / grid));
  if (merge_waves(d, b) > kMaxWaves) p.chunks = 1;
  p.fits = grid <= kMaxGrid;
  p.span = (ntile + p.chunks - 1) / p.chunks;
  p.chunks = (ntile + p.span - 1) / p.span;
  return p;
}
size_t fwd_part_bytes(const vc_packedattn_desc* d, const FwdPlan& p) {
  return p.chunks == 1 ? 256 : align256((size_t)p.chunks * d->total_q * d->heads * (d->head_dim + 2) * sizeof(float));
}

// The dQ pass's chunks of a row block's key tiles: as the forward's, where they promise to take less than
// 0.7 of the time. Forward and backward, us unsplit / split, 16 heads, D = 128: 64 queries of 16,384 keys 350 / 93, 300
// and 200 of 8,000 and 3,000 324 / 253, 8,192 causal at 4 heads 435 / 420; not so 2,048 causal 159 / 168, 4,096 389 / 410.
struct DqPlan {
  int chunks, span;
  bool fits;
};
DqPlan dq_plan(const vc_packedattn_desc* d) {
  const vcja::RowBlocks b = query_blocks(d, 1);
  const int64_t grid = b.blocks * d->heads;
  const bool uneven = d->causal && 2 * (int64_t)d->max_q > d->max_k;
  const double work = equal_blocks(d, d->max_q, d->total_q, d->max_k, d->total_k) * d->heads * (uneven ? 0.5 : 1.0);
  const int ntile = (d->max_k + vcja::kTileTok - 1) / vcja::kTileTok;
  double gain = 1;
  int64_t chunks = fwd_chunks(d, work, (double)d->total_q * d->heads, uneven, &gain);
  chunks = gain * 0.7 < 1 || merge_waves(d, b) > kMaxWaves ? 1 : std::max<int64_t>(1, std::min(chunks, kMaxGrid / grid));
  DqPlan p;
  p.fits = grid <= kMaxGrid;
  p.span = (int)((ntile + chunks - 1) / chunks);
  p.chunks = (ntile + p.span - 1) / p.span;
  return p;
}
size_t dq_part_bytes(const vc_packedattn_desc* d, int c) {
  return c == 1 ? 0 : align256((size_t)c * d->total_q * d->heads * (d->head_dim + 1) * sizeof(float));
}

// Backward workspace: -LSE/c | -D | the bias gradient's sums per distance.
size_t stat_bytes(const vc_packedattn_desc* d) {
  return align256((size_t)d->heads * vcja::packed_rows(d->total_q, d->sequences) * sizeof(float));
}
// Backward: the chunks of a key block's query tiles (over all heads of the group). About 512
// workgroups fill the chip twice; up to 1,024 even out the causal rule's unequal blocks where each
// then still has 96 tiles of 32 queries to pay for its partial sums. Measured, forward and backward at D = 128,
// us with 512 / 1,024: 4 x 1,024 tokens, 16 heads, 4 key heads 132 / 162; 16 x 1,024 394 / 432; 1 x 2,048 158 /
// 183; 4 x 4,096 1255 / 1189; 1 x 12,000, 2 key heads 2565 / 2387.
int key_chunks(const vc_packedattn_desc* d) {
  const int bm = vcja::kPackedRows, group = d->heads / d->kv_heads;
  // blocks of all slots, but not many more than their work amounts to
  const int64_t items = d->kv_heads * std::min<int64_t>({(int64_t)d->sequences * ((d->max_k + bm - 1) / bm), d->total_k / bm + d->sequences,
                                                         (int64_t)(2 * equal_blocks(d, d->max_k, d->total_k, d->max_q, d->total_q)) + 1});
  const int64_t steps = (int64_t)group * ((d->max_q + 31) / 32);
  const int64_t want = std::min((1024 + items - 1) / items, std::max((512 + items - 1) / items, steps / 96));
  // the workgroups of a launch, and the threads of the sum over the chunks (one per 4 elements)
  const int64_t grid = key_blocks(d).blocks * d->kv_heads;
  const int64_t most = (d->total_k * d->kv_heads * d->head_dim / 4 + 255) / 256 > kMaxGroups ? 1 : kMaxGrid / grid;
  const int64_t chunks = std::max<int64_t>(1, std::min({want, steps / 8, most}));
  if (!d->num_buckets) return (int)chunks;
  const int64_t whole = (chunks + group - 1) / group * group;  // with a bias none of two heads
  return (int)(whole <= most ? whole : std::max<int64_t>(group, most / group * group));
}
bool key_fits(const vc_packedattn_desc* d, int chunks) {
  return key_blocks(d).blocks * d->kv_heads * chunks <= kMaxGrid &&
         (chunks == 1 || (d->total_k * d->kv_heads * d->head_dim / 4 + 255) / 256 <= kMaxGroups);
}
struct BwdPlan {
  DqPlan dq;
  int key_chunks;
  bool fits;
};
BwdPlan bwd_plan(const vc_packedattn_desc* d) {
  BwdPlan p;
  p.dq = dq_plan(d);
  p.key_chunks = key_chunks(d);
  p.fits = p.dq.fits && key_fits(d, p.key_chunks);
  return p;
}
size_t dist_bytes(const vc_packedattn_desc* d, int chunks) {
  if (!d->num_buckets) return 0;
  const int bm = vcja::kPackedRows;
  const int per_head = chunks / (d->heads / d->kv_heads);
  return align256((size_t)(vcja::dist_row(d->total_k, d->sequences, 0, bm) + 1) * per_head * d->heads * (2 * d->max_distance + 1) *
                  sizeof(float));
}
size_t key_part_bytes(const vc_packedattn_desc* d, int c) {
  return c == 1 ? 0 : align256((size_t)c * 2 * d->total_k * d->kv_heads * d->head_dim * sizeof(float));
}

// The partial results of the two passes take the same room, one after the other.
size_t bwd_ws_bytes(const vc_packedattn_desc* d, const BwdPlan& p) {
  return 2 * stat_bytes(d) + dist_bytes(d, p.key_chunks) + std::max(key_part_bytes(d, p.key_chunks), dq_part_bytes(d, p.dq.chunks));
}

vc_status check_inputs(const vc_packedattn_desc* d, const void* q, const void* k, const void* v, const int32_t* cu_q,
                       const int32_t* cu_k, const int32_t* len_q, const int32_t* len_k, const void* bias,
                       const int32_t* buckets) {
  if (!q || !k || !v || !cu_q || !cu_k || (d->num_buckets && (!bias || !buckets))) return VC_ERR_NULL;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned4(cu_q) || !aligned4(cu_k) || !aligned4(len_q) ||
      !aligned4(len_k) || (d->num_buckets && ((reinterpret_cast<uintptr_t>(bias) & 1u) || !aligned4(buckets))))
    return VC_ERR_ALIGN;
  return VC_OK;
}

// The descriptor, and whether the launches of the call can be made; fills the plan.
vc_status check_fwd(const vc_packedattn_desc* d, FwdPlan* p) {
  const vc_status st = check_packed(d);
  if (st != VC_OK) return st;
  *p = fwd_plan(d);
  return p->fits ? VC_OK : VC_ERR_SHAPE;
}
vc_status check_bwd(const vc_packedattn_desc* d, BwdPlan* p) {
  const vc_status st = check_packed(d);
  if (st != VC_OK) return st;
  if (d->clear_outside > 1) return VC_ERR_SHAPE;
  *p = bwd_plan(d);
  return p->fits ? VC_OK : VC_ERR_SHAPE;
}

vc_status check_ws(const void* ws, size_t have, size_t need) {
  if (!ws) return VC_ERR_WORKSPACE;
  if ((reinterpret_cast<uintptr_t>(ws) & 255u) != 0) return VC_ERR_ALIGN;
  return have < need ? VC_ERR_WORKSPACE : VC_OK;
}

}  // namespace

extern "C" {

size_t vc_packedattn_fwd_workspace_bytes(const vc_packedattn_desc* desc) {
  FwdPlan p;
  return check_fwd(desc, &p) == VC_OK ? fwd_part_bytes(desc, p) : 0;
}

vc_status vc_packedattn_fwd(const vc_packedattn_desc* desc, const void* q, const void* k, const void* v,
                            const int32_t* cu_q, const int32_t* cu_k, const int32_t* len_q, const int32_t* len_k,
                            const void* bias, const int32_t* buckets, void* o, float* lse, void* workspace,
                            size_t workspace_bytes, void* stream) {
  FwdPlan p;
  vc_status st = check_fwd(desc, &p);
  if (st != VC_OK) return st;
  if (!o || !lse) return VC_ERR_NULL;
  if ((st = check_inputs(desc, q, k, v, cu_q, cu_k, len_q, len_k, bias, buckets)) != VC_OK) return st;
  if (!aligned16(o) || !aligned4(lse)) return VC_ERR_ALIGN;
  if ((st = check_ws(workspace, workspace_bytes, fwd_part_bytes(desc, p))) != VC_OK) return st;
  if ((st = vcja::check_device()) != VC_OK) return st;
  vcja::PackedArgs a = packed_args(desc, q, k, v, cu_q, cu_k, len_q, len_k, bias, buckets);
  a.o = static_cast<__bf16*>(o);
  a.lse = lse;
  a.pack = p.pack;
  a.few = p.few;
  a.chunks = p.chunks;
  a.span = p.span;
  a.part = static_cast<float*>(workspace);
  return vcja::launch_packed_fwd(a, desc->head_dim, as_stream(stream)) == hipSuccess ? VC_OK : VC_ERR_HIP;
}

size_t vc_packedattn_bwd_workspace_bytes(const vc_packedattn_desc* desc) {
  BwdPlan p;
  return check_bwd(desc, &p) == VC_OK ? bwd_ws_bytes(desc, p) : 0;
}

vc_status vc_packedattn_bwd(const vc_packedattn_desc* desc, const void* q, const void* k, const void* v, const void* o,
                            const float* lse, const void* dout, const int32_t* cu_q, const int32_t* cu_k,
                            const int32_t* len_q, const int32_t* len_k, const void* bias, const int32_t* buckets, void* dq,
                            void* dk, void* dv, void* dbias, void* workspace, size_t workspace_bytes, void* stream) {
  BwdPlan p;
  vc_status st = check_bwd(desc, &p);
  if (st != VC_OK) return st;
  if (!o || !lse || !dout || !dq || !dk || !dv) return VC_ERR_NULL;
  if ((st = check_inputs(desc, q, k, v, cu_q, cu_k, len_q, len_k, bias, buckets)) != VC_OK) return st;
  if (!aligned16(o) || !aligned4(lse) || !aligned16(dout) || !aligned16(dq) || !aligned16(dk) || !aligned16(dv) ||
      (reinterpret_cast<uintptr_t>(dbias) & 1u))
    return VC_ERR_ALIGN;
  if (dbias && !desc->num_buckets) return VC_ERR_SHAPE;
  if ((st = check_ws(workspace, workspace_bytes, bwd_ws_bytes(desc, p))) != VC_OK) return st;
  if ((st = vcja::check_device()) != VC_OK) return st;
  vcja::PackedArgs a = packed_args(desc, q, k, v, cu_q, cu_k, len_q, len_k, bias, buckets);
  a.o_in = bf(o);
  a.lse = const_cast<float*>(lse);
  a.dout = bf(dout);
  a.dq = static_cast<__bf16*>(dq);
  a.dk = static_cast<__bf16*>(dk);
  a.dv = static_cast<__bf16*>(dv);
  char* ws = static_cast<char*>(workspace);
  a.nls = reinterpret_cast<float*>(ws);
  a.dd = reinterpret_cast<float*>(ws + stat_bytes(desc));
  a.dist_part = reinterpret_cast<float*>(ws + 2 * stat_bytes(desc));
  a.key_part = reinterpret_cast<float*>(ws + 2 * stat_bytes(desc) + dist_bytes(desc, p.key_chunks));
  a.part = a.key_part;
  a.chunks = p.key_chunks;
  a.dq_chunks = p.dq.chunks;
  a.span = p.dq.span;
  return vcja::launch_packed_bwd(a, desc->head_dim, static_cast<__bf16*>(dbias), as_stream(stream)) == hipSuccess ? VC_OK
                                                                                                            : VC_ERR_HIP;
}

}  // extern "C"

namespace {

vc_status check_norm(const vc_layernorm_desc* d) {
  if (!d) return VC_ERR_NULL;
  if (d->rows < 1 || d->cols < 1 || d->cols > (1 << 16) || d->rows > vcja::norm_max_rows(d->cols)) return VC_ERR_SHAPE;
  for (const int t : {d->x_type, d->param_type})
    if (t != VC_BF16 && t != VC_FP32) return VC_ERR_UNSUPPORTED;
  for (const int64_t s : {d->x_stride, d->dout_stride})
    if (s && (s < d->cols || s > ((int64_t)1 << 30))) return VC_ERR_SHAPE;
  if (!(d->eps >= 0.0f && isfinite(d->eps))) return VC_ERR_SHAPE;
  return VC_OK;
}
bool aligned_elem(const void* p, int type) { return (reinterpret_cast<uintptr_t>(p) & (type == VC_BF16 ? 1u : 3u)) == 0; }

vcja::NormArgs norm_args(const vc_layernorm_desc* d, const void* x, const void* weight) {
  vcja::NormArgs a{};
  a.x = x;
  a.w = weight;
  a.rows = (int)d->rows;
  a.cols = d->cols;
  a.stride = d->x_stride ? d->x_stride : d->cols;
  a.dout_stride = d->dout_stride ? d->dout_stride : d->cols;
  a.eps = d->eps;
  a.x_f32 = d->x_type == VC_FP32;
  a.p_f32 = d->param_type == VC_FP32;
  a.groups = vcja::norm_groups(d->rows, d->cols);
  return a;
}

}  // namespace

extern "C" {

vc_status vc_layernorm_fwd(const vc_layernorm_desc* desc, const void* x, const void* weight, const void* bias, void* y,
                           float* mean, float* rstd, void* stream) {
  vc_status st = check_norm(desc);
  if (st != VC_OK) return st;
  if (!x || !y || !mean || !rstd) return VC_ERR_NULL;
  if (!aligned_elem(x, desc->x_type) || !aligned_elem(y, desc->x_type) || !aligned_elem(weight, desc->param_type) ||
      !aligned_elem(bias, desc->param_type) || !aligned4(mean) || !aligned4(rstd))
    return VC_ERR_ALIGN;
  if ((st = vcja::check_device()) != VC_OK) return st;
  vcja::NormArgs a = norm_args(desc, x, weight);
  a.b = bias;
  a.y = y;
  a.mean = mean;
  a.rstd = rstd;
  return vcja::launch_norm_fwd(a, as_stream(stream)) == hipSuccess ? VC_OK : VC_ERR_HIP;
}

size_t vc_layernorm_bwd_workspace_bytes(const vc_layernorm_desc* desc) {
  if (check_norm(desc) != VC_OK) return 0;
  return align256((size_t)2 * vcja::norm_groups(desc->rows, desc->cols) * desc->cols * sizeof(float));
}

vc_status vc_layernorm_bwd(const vc_layernorm_desc* desc, const void* dout, const void* x, const void* weight,
                           const float* mean, const float* rstd, void* dx, void* dweight, void* dbias, void* workspace,
                           size_t workspace_bytes, void* stream) {
  vc_status st = check_norm(desc);
  if (st != VC_OK) return st;
  if (!dout || !x || !mean || !rstd || !dx) return VC_ERR_NULL;
  if (!aligned_elem(dout, desc->x_type) || !aligned_elem(x, desc->x_type) || !aligned_elem(dx, desc->x_type) ||
      !aligned_elem(weight, desc->param_type) || !aligned_elem(dweight, desc->param_type) ||
      !aligned_elem(dbias, desc->param_type) || !aligned4(mean) || !aligned4(rstd))
    return VC_ERR_ALIGN;
  if ((dweight || dbias) && (st = check_ws(workspace, workspace_bytes, vc_layernorm_bwd_workspace_bytes(desc))) != VC_OK)
    return st;
  if ((st = vcja::check_device()) != VC_OK) return st;
  vcja::NormArgs a = norm_args(desc, x, weight);
  a.dout = dout;
  a.mean = const_cast<float*>(mean);
  a.rstd = const_cast<float*>(rstd);
  a.dx = dx;
  a.dw = dweight;
  a.db = dbias;
  a.part = static_cast<float*>(workspace);
  return vcja::launch_norm_bwd(a, as_stream(stream)) == hipSuccess ? VC_OK : VC_ERR_HIP;
}

}  // extern "C"
