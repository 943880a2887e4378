// C ABI of the operators around a block's attention: checks of descriptors, pointers and workspaces, and the
// launches' arguments.
#include <math.h>

#include "checkpoint.hpp"
#include "embedding.hpp"
#include "host.hpp"
#include "residual.hpp"

namespace {

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
hipStream_t as_stream(void* s) { return static_cast<hipStream_t>(s); }
bool type_ok(int t) { return t == VC_BF16 || t == VC_FP32; }
// Aligned to an element of its type; NULL is.
bool aligned_elem(const void* p, int type) { return (reinterpret_cast<uintptr_t>(p) & (type == VC_BF16 ? 1u : 3u)) == 0; }
bool stride_ok(int64_t s, int cols) { return s == 0 || (s >= cols && s <= ((int64_t)1 << 30)); }

vc_status check_ws(const void* ws, size_t have, size_t need) {
  if (!ws || have < need) return VC_ERR_WORKSPACE;
  return (reinterpret_cast<uintptr_t>(ws) & 255u) == 0 ? VC_OK : VC_ERR_ALIGN;
}

// --- residual norm -----------------------------------------------------------------------------

vc_status check_residual(const vc_residualnorm_desc* d) {
  if (!d) return VC_ERR_NULL;
  if (d->rows < 1 || d->rows > ((int64_t)1 << 30) || d->cols < 1 || d->cols > vcja::kResidualCols) return VC_ERR_SHAPE;
  // the launch that adds up the samples' sums: less than 2^32 threads, of workgroups of 64 where there are many
  const int64_t across = (d->cols + 15) / 16;
  if (d->samples < 1 || 3 * across * d->samples >= ((int64_t)1 << 32) / 64) return VC_ERR_SHAPE;
  if (!d->packed && d->rows % d->samples) return VC_ERR_SHAPE;
  if (!type_ok(d->x_type) || !type_ok(d->y_type) || !type_ok(d->param_type)) return VC_ERR_UNSUPPORTED;
  if (d->x_type == VC_BF16 && d->y_type == VC_FP32) return VC_ERR_UNSUPPORTED;
  for (const int k : {d->norm, d->post_norm})
    if (k != VC_NORM_NONE && k != VC_NORM_LAYER && k != VC_NORM_RMS) return VC_ERR_UNSUPPORTED;
  for (const int b : {d->packed, d->plus_one, d->checkpoint, d->clear_outside})
    if (b != 0 && b != 1) return VC_ERR_SHAPE;
  if (!isfinite(d->residual_scale) || !(d->eps >= 0.0f && isfinite(d->eps))) return VC_ERR_SHAPE;
  for (const int64_t s : {d->x_stride, d->a_stride, d->dh_stride, d->dy_stride})
    if (!stride_ok(s, d->cols)) return VC_ERR_SHAPE;
  for (const int64_t s : {d->gate_stride, d->scale_stride, d->shift_stride})
    if (s != VC_SHARED && !stride_ok(s, d->cols)) return VC_ERR_SHAPE;
  return VC_OK;
}

// What the offsets, lengths and parameters of a call have to be.
vc_status check_common(const vc_residualnorm_desc* d, const void* gate, const void* scale, const void* shift, const void* wp,
                       const int32_t* cu, const int32_t* lens) {
  if ((d->packed != 0) != (cu != nullptr)) return d->packed ? VC_ERR_NULL : VC_ERR_SHAPE;
  for (const void* p : {gate, scale, shift, wp})
    if (!aligned_elem(p, d->param_type)) return VC_ERR_ALIGN;
  return vcja::aligned4(cu) && vcja::aligned4(lens) ? VC_OK : VC_ERR_ALIGN;
}

vcja::ResidualArgs residual_args(const vc_residualnorm_desc* d, bool backward) {
  vcja::ResidualArgs a{};
  auto rows = [&](int64_t s) { return s ? s : (int64_t)d->cols; };
  auto samples = [&](int64_t s) { return s == VC_SHARED ? 0 : s ? s : (int64_t)d->cols; };
  a.x_stride = rows(d->x_stride);
  a.a_stride = rows(d->a_stride);
  a.dh_stride = rows(d->dh_stride);
  a.dy_stride = rows(d->dy_stride);
  a.gate_stride = samples(d->gate_stride);
  a.scale_stride = samples(d->scale_stride);
  a.shift_stride = samples(d->shift_stride);
  a.rows = (int)d->rows;
  a.cols = d->cols;
  a.samples = d->samples;
  a.per = d->packed ? 0 : (int)(d->rows / d->samples);
  a.c = d->residual_scale;
  a.eps = d->eps;
  a.norm = d->norm;
  a.post = d->post_norm;
  a.plus_one = d->plus_one;
  a.p_f32 = d->param_type == VC_FP32;
  a.x_f32 = d->x_type == VC_FP32;
  a.y_f32 = d->y_type == VC_FP32;
  a.clear = d->clear_outside;
  vcja::residual_groups(d->rows, d->cols, backward, &a.groups, &a.chunk);
  return a;
}
size_t part_bytes(const vc_residualnorm_desc* d) {
  int groups, chunk;
  vcja::residual_groups(d->rows, d->cols, true, &groups, &chunk);
  return align256(((size_t)groups + d->samples) * 3 * d->cols * sizeof(float));
}
size_t residual_ws_bytes(const vc_residualnorm_desc* d) {
  return part_bytes(d) + (d->samples > 1 ? align256((size_t)d->samples * 3 * d->cols * sizeof(float)) : 0);
}

}  // namespace

extern "C" {

vc_status vc_residualnorm_fwd(const vc_residualnorm_desc* desc, const void* x, const void* a, const void* gate,
                              const void* scale, const void* shift, const void* post_weight, const int32_t* cu,
                              const int32_t* lens, void* h, void* y, float* mean, float* rstd, float* post_mean,
                              float* post_rstd, void* h8, float* h8_scales, void* a8, float* a8_scales, void* stream) {
  vc_status st = check_residual(desc);
  if (st != VC_OK) return st;
  const bool norm = desc->norm != VC_NORM_NONE, post = desc->post_norm != VC_NORM_NONE;
  if (!x || (a && !h) || (norm && (!y || !mean || !rstd))) return VC_ERR_NULL;
  if (a ? post && (!post_mean || !post_rstd) : post || gate || post_weight) return a ? VC_ERR_NULL : VC_ERR_SHAPE;
  if (!a && !norm) return VC_ERR_SHAPE;                      // nothing to compute
  if (!a && desc->residual_scale != 1.0f) return VC_ERR_SHAPE;  // h is x then, whether it is written or not
  if (!post && post_weight) return VC_ERR_SHAPE;
  if (!norm && (scale || shift)) return VC_ERR_SHAPE;
  if (desc->checkpoint && ((norm && (!h8 || !h8_scales)) || (a && (!a8 || !a8_scales)))) return VC_ERR_NULL;
  if ((st = check_common(desc, gate, scale, shift, post_weight, cu, lens)) != VC_OK) return st;
  for (const void* p : {x, (const void*)h})
    if (!aligned_elem(p, desc->x_type)) return VC_ERR_ALIGN;
  for (const void* p : {a, (const void*)y})
    if (!aligned_elem(p, desc->y_type)) return VC_ERR_ALIGN;
  for (const float* p : {mean, rstd, post_mean, post_rstd, h8_scales, a8_scales})
    if (!vcja::aligned4(p)) return VC_ERR_ALIGN;
  if ((st = vcja::check_device()) != VC_OK) return st;
  vcja::ResidualArgs r = residual_args(desc, false);
  r.x = x;
  r.a = a;
  r.gate = gate;
  r.scale = scale;
  r.shift = shift;
  r.wp = post_weight;
  r.cu = cu;
  r.lens = lens;
  r.h = h;
  r.y = norm ? y : nullptr;
  r.mean = mean;
  r.rstd = rstd;
  r.pmean = post_mean;
  r.prstd = post_rstd;
  if (desc->checkpoint) {
    if (norm) {
      r.h8 = static_cast<int8_t*>(h8);
      r.h8s = h8_scales;
    }
    if (a) {
      r.a8 = static_cast<int8_t*>(a8);
      r.a8s = a8_scales;
    }
  }
  return vcja::launch_residual_fwd(r, as_stream(stream)) == hipSuccess ? VC_OK : VC_ERR_HIP;
}

size_t vc_residualnorm_bwd_workspace_bytes(const vc_residualnorm_desc* desc) {
  return check_residual(desc) == VC_OK ? residual_ws_bytes(desc) : 0;
}

vc_status vc_residualnorm_bwd(const vc_residualnorm_desc* desc, const void* dh, const void* dy, const void* h, const void* a,
                              const float* h8_scales, const float* a8_scales, const void* gate, const void* scale,
                              const void* post_weight, const int32_t* cu, const int32_t* lens, const float* mean,
                              const float* rstd, const float* post_mean, const float* post_rstd, void* dx, void* da,
                              void* dgate, void* dscale, void* dshift, void* dpost_weight, void* workspace,
                              size_t workspace_bytes, void* stream) {
  vc_status st = check_residual(desc);
  if (st != VC_OK) return st;
  const bool norm = desc->norm != VC_NORM_NONE, post = desc->post_norm != VC_NORM_NONE;
  if (!dh && !dy) return VC_ERR_NULL;
  if (norm ? dy && (!h || !mean || !rstd) : !dh) return VC_ERR_NULL;
  if (!norm && (dy || scale || dscale || dshift)) return VC_ERR_SHAPE;
  if (a ? post && (!post_mean || !post_rstd) : post || gate || post_weight || da || dgate || dpost_weight)
    return a ? VC_ERR_NULL : VC_ERR_SHAPE;
  if (!a && (!norm || desc->residual_scale != 1.0f)) return VC_ERR_SHAPE;
  if (!post && (post_weight || dpost_weight)) return VC_ERR_SHAPE;
  if (desc->checkpoint && ((dy && !h8_scales) || (a && !a8_scales))) return VC_ERR_NULL;
  if ((st = check_common(desc, gate, scale, nullptr, post_weight, cu, lens)) != VC_OK) return st;
  for (const void* p : {dh, (const void*)dx})
    if (!aligned_elem(p, desc->x_type)) return VC_ERR_ALIGN;
  for (const void* p : {dy, (const void*)da})
    if (!aligned_elem(p, desc->y_type)) return VC_ERR_ALIGN;
  if (!desc->checkpoint && (!aligned_elem(h, desc->x_type) || !aligned_elem(a, desc->y_type))) return VC_ERR_ALIGN;
  for (const void* p : {dgate, dscale, dshift, dpost_weight})
    if (!aligned_elem(p, desc->param_type)) return VC_ERR_ALIGN;
  for (const float* p : {mean, rstd, post_mean, post_rstd, h8_scales, a8_scales})
    if (!vcja::aligned4(p)) return VC_ERR_ALIGN;
  const bool sums = dgate || dscale || dshift || dpost_weight;
  if (!dx && !da && !sums) return VC_ERR_NULL;
  if (sums && (st = check_ws(workspace, workspace_bytes, residual_ws_bytes(desc))) != VC_OK) return st;
  if ((st = vcja::check_device()) != VC_OK) return st;
  vcja::ResidualArgs r = residual_args(desc, true);
  r.dh = dh;
  r.dy = dy;
  if (desc->checkpoint) {
    r.h8 = static_cast<int8_t*>(const_cast<void*>(h));
    r.a8 = static_cast<int8_t*>(const_cast<void*>(a));
    r.h8s = const_cast<float*>(h8_scales);
    r.a8s = const_cast<float*>(a8_scales);
  } else {
    r.h_in = h;
    r.h_stride = a ? desc->cols : r.x_stride;  // without a block output h is x itself
    r.a = a;
  }
  r.gate = gate;
  r.scale = scale;
  r.wp = post_weight;
  r.cu = cu;
  r.lens = lens;
  r.mean = const_cast<float*>(mean);
  r.rstd = const_cast<float*>(rstd);
  r.pmean = const_cast<float*>(post_mean);
  r.prstd = const_cast<float*>(post_rstd);
  r.dx = dx;
  r.da = da;
  r.dgate = dgate;
  r.dscale = dscale;
  r.dshift = dshift;
  r.dwp = dpost_weight;
  if (sums) {
    r.part = static_cast<float*>(workspace);
    // a gate's gradient may be wanted where the gate itself is not given (1); a gate of each sample weighs the sums of dpost_weight
    const bool own = (gate || dgate) && r.gate_stride || dscale && r.scale_stride || dshift && r.shift_stride;
    r.flat = desc->samples == 1 || !own;
    if (!r.flat && (dpost_weight || (dgate && !r.gate_stride) || (dscale && !r.scale_stride) || (dshift && !r.shift_stride)))
      r.sums = reinterpret_cast<float*>(static_cast<char*>(workspace) + part_bytes(desc));
  }
  return vcja::launch_residual_bwd(r, desc->checkpoint != 0, as_stream(stream)) == hipSuccess ? VC_OK : VC_ERR_HIP;
}

}  // extern "C"

// --- checkpoints -------------------------------------------------------------------------------

namespace {

vc_status check_checkpoint(const vc_checkpoint_desc* d) {
  if (!d) return VC_ERR_NULL;
  if (d->rows < 1 || d->rows > ((int64_t)1 << 32) || d->cols < 1 || d->cols > (1 << 24)) return VC_ERR_SHAPE;
  if (!type_ok(d->type)) return VC_ERR_UNSUPPORTED;
  return stride_ok(d->stride, d->cols) ? VC_OK : VC_ERR_SHAPE;
}
vcja::CheckpointArgs checkpoint_args(const vc_checkpoint_desc* d) {
  vcja::CheckpointArgs a{};
  a.rows = d->rows;
  a.cols = d->cols;
  a.blocks = (d->cols + 127) / 128;
  a.stride = d->stride ? d->stride : d->cols;
  a.f32 = d->type == VC_FP32;
  return a;
}

}  // namespace

extern "C" {

vc_status vc_checkpoint_pack(const vc_checkpoint_desc* desc, const void* x, void* q, float* scales, void* stream) {
  vc_status st = check_checkpoint(desc);
  if (st != VC_OK) return st;
  if (!x || !q || !scales) return VC_ERR_NULL;
  if (!aligned_elem(x, desc->type) || !vcja::aligned4(scales)) return VC_ERR_ALIGN;
  if ((st = vcja::check_device()) != VC_OK) return st;
  vcja::CheckpointArgs a = checkpoint_args(desc);
  a.x = x;
  a.q = static_cast<int8_t*>(q);
  a.scales = scales;
  return vcja::launch_checkpoint_pack(a, as_stream(stream)) == hipSuccess ? VC_OK : VC_ERR_HIP;
}

vc_status vc_checkpoint_unpack(const vc_checkpoint_desc* desc, const void* q, const float* scales, void* y, void* stream) {
  vc_status st = check_checkpoint(desc);
  if (st != VC_OK) return st;
  if (!y || !q || !scales) return VC_ERR_NULL;
  if (!aligned_elem(y, desc->type) || !vcja::aligned4(scales)) return VC_ERR_ALIGN;
  if (desc->stride && desc->stride != desc->cols) return VC_ERR_SHAPE;
  if ((st = vcja::check_device()) != VC_OK) return st;
  vcja::CheckpointArgs a = checkpoint_args(desc);
  a.y = y;
  a.q = static_cast<int8_t*>(const_cast<void*>(q));
  a.scales = const_cast<float*>(scales);
  return vcja::launch_checkpoint_unpack(a, as_stream(stream)) == hipSuccess ? VC_OK : VC_ERR_HIP;
}

}  // extern "C"

// --- embedding ---------------------------------------------------------------------------------

namespace {

vc_status check_embedding(const vc_embedding_desc* d, bool backward) {
  if (!d) return VC_ERR_NULL;
  if (d->tokens < 1 || d->tokens > (backward ? vcja::kEmbeddingTokens : (int64_t)1 << 30) || d->vocab < 1 ||
      d->vocab > vcja::kEmbeddingVocab || d->cols < 1 || d->cols > vcja::kResidualCols)
    return VC_ERR_SHAPE;
  if (!type_ok(d->table_type) || !type_ok(d->out_type)) return VC_ERR_UNSUPPORTED;
  if ((d->ids64 != 0 && d->ids64 != 1) || (d->accumulate != 0 && d->accumulate != 1)) return VC_ERR_SHAPE;
  if (!isfinite(d->scale)) return VC_ERR_SHAPE;
  return stride_ok(d->row_stride, d->cols) ? VC_OK : VC_ERR_SHAPE;
}
bool aligned_ids(const void* p, int ids64) { return (reinterpret_cast<uintptr_t>(p) & (ids64 ? 7u : 3u)) == 0; }

vcja::EmbeddingArgs embedding_args(const vc_embedding_desc* d, const void* ids) {
  vcja::EmbeddingArgs a{};
  a.ids = ids;
  a.ids64 = d->ids64;
  a.tokens = d->tokens;
  a.vocab = d->vocab;
  a.cols = d->cols;
  a.padding = d->padding_id;
  a.scale = d->scale;
  return a;
}
struct EmbeddingLayout {
  size_t list, hist, part;  // bytes
  size_t all() const { return 4 * list + hist + part; }
};
EmbeddingLayout embedding_layout(const vc_embedding_desc* d) {
  const vcja::EmbeddingPlan p = vcja::embedding_plan(d->tokens, d->vocab, d->cols);
  EmbeddingLayout l;
  l.list = align256((size_t)d->tokens * sizeof(uint32_t));
  l.hist = p.blocks > 1 ? align256((size_t)p.blocks * 512 * sizeof(uint32_t)) : 0;
  l.part = align256((size_t)p.chunks * 2 * d->cols * sizeof(float));
  return l;
}

}  // namespace

extern "C" {

vc_status vc_embedding_fwd(const vc_embedding_desc* desc, const void* ids, const void* table, void* out, void* stream) {
  vc_status st = check_embedding(desc, false);
  if (st != VC_OK) return st;
  if (!ids || !table || !out) return VC_ERR_NULL;
  if (!aligned_ids(ids, desc->ids64) || !aligned_elem(table, desc->table_type) || !aligned_elem(out, desc->out_type))
    return VC_ERR_ALIGN;
  if ((st = vcja::check_device()) != VC_OK) return st;
  vcja::EmbeddingArgs a = embedding_args(desc, ids);
  a.table = table;
  a.out = out;
  a.table_stride = desc->row_stride ? desc->row_stride : desc->cols;
  a.table_f32 = desc->table_type == VC_FP32;
  a.out_f32 = desc->out_type == VC_FP32;
  return vcja::launch_embedding_fwd(a, as_stream(stream)) == hipSuccess ? VC_OK : VC_ERR_HIP;
}

size_t vc_embedding_bwd_workspace_bytes(const vc_embedding_desc* desc) {
  return check_embedding(desc, true) == VC_OK ? embedding_layout(desc).all() : 0;
}

vc_status vc_embedding_bwd(const vc_embedding_desc* desc, const void* ids, const void* dout, void* dtable, void* workspace,
                           size_t workspace_bytes, void* stream) {
  vc_status st = check_embedding(desc, true);
  if (st != VC_OK) return st;
  if (!ids || !dout || !dtable) return VC_ERR_NULL;
  if (!aligned_ids(ids, desc->ids64) || !aligned_elem(dout, desc->out_type) || !aligned_elem(dtable, desc->table_type))
    return VC_ERR_ALIGN;
  const EmbeddingLayout l = embedding_layout(desc);
  if ((st = check_ws(workspace, workspace_bytes, l.all())) != VC_OK) return st;
  if ((st = vcja::check_device()) != VC_OK) return st;
  vcja::EmbeddingArgs a = embedding_args(desc, ids);
  a.dout = dout;
  a.dout_stride = desc->row_stride ? desc->row_stride : desc->cols;
  a.grad = dtable;
  a.out_f32 = desc->out_type == VC_FP32;
  a.grad_f32 = desc->table_type == VC_FP32;
  a.add = desc->accumulate;
  char* ws = static_cast<char*>(workspace);
  a.keys[0] = reinterpret_cast<uint32_t*>(ws);
  a.keys[1] = reinterpret_cast<uint32_t*>(ws + l.list);
  a.pos[0] = reinterpret_cast<uint32_t*>(ws + 2 * l.list);
  a.pos[1] = reinterpret_cast<uint32_t*>(ws + 3 * l.list);
  a.hist = reinterpret_cast<uint32_t*>(ws + 4 * l.list);
  a.part = reinterpret_cast<float*>(ws + 4 * l.list + l.hist);
  return vcja::launch_embedding_bwd(a, as_stream(stream)) == hipSuccess ? VC_OK : VC_ERR_HIP;
}

}  // extern "C"
