"""The operators around a block's attention: the gated residual with the norms before and after a block, activation
checkpoints in 8 bits, and the embedding of tokens.

As everywhere in this package, the tensor-level helpers check and marshal arguments and allocate outputs;
every step of the computation runs in the library's HIP kernels (include/vc_jointattn.h).
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple

from paper_2501_08453_amd import (JointAttnError, _call, _lib, _ptr, _save_whole, _stream, _workspace,
                                  vc_checkpoint_desc, vc_embedding_desc, vc_residualnorm_desc)
from paper_2501_08453_amd.tower import _check_all, _row_stride, _ws_bytes

NORMS = {None: 0, "layer": 1, "rms": 2}  # VC_NORM_*
SHARED = -1                              # VC_SHARED
BLOCK = 128                              # columns of a row that share a checkpoint's scale


# --------------------------------------------------------------------------
# Raw entry points with the C names (pointers are ints or torch tensors).
# --------------------------------------------------------------------------

def vc_residualnorm_fwd(desc, x, a, gate, scale, shift, post_weight, cu, lens, h, y, mean, rstd, post_mean, post_rstd,
                        h8, h8_scales, a8, a8_scales, stream=None):
    _call("vc_residualnorm_fwd", ctypes.byref(desc), _ptr(x), _ptr(a), _ptr(gate), _ptr(scale), _ptr(shift),
          _ptr(post_weight), _ptr(cu), _ptr(lens), _ptr(h), _ptr(y), _ptr(mean), _ptr(rstd), _ptr(post_mean),
          _ptr(post_rstd), _ptr(h8), _ptr(h8_scales), _ptr(a8), _ptr(a8_scales), _stream(stream))


def vc_residualnorm_bwd_workspace_bytes(desc) -> int:
    return _lib().vc_residualnorm_bwd_workspace_bytes(ctypes.byref(desc))


def vc_residualnorm_bwd(desc, dh, dy, h, a, h8_scales, a8_scales, gate, scale, post_weight, cu, lens, mean, rstd,
                        post_mean, post_rstd, dx, da, dgate, dscale, dshift, dpost_weight, workspace, workspace_bytes,
                        stream=None):
    _call("vc_residualnorm_bwd", ctypes.byref(desc), _ptr(dh), _ptr(dy), _ptr(h), _ptr(a), _ptr(h8_scales),
          _ptr(a8_scales), _ptr(gate), _ptr(scale), _ptr(post_weight), _ptr(cu), _ptr(lens), _ptr(mean), _ptr(rstd),
          _ptr(post_mean), _ptr(post_rstd), _ptr(dx), _ptr(da), _ptr(dgate), _ptr(dscale), _ptr(dshift),
          _ptr(dpost_weight), _ptr(workspace), int(workspace_bytes), _stream(stream))


def vc_checkpoint_pack(desc, x, q, scales, stream=None):
    _call("vc_checkpoint_pack", ctypes.byref(desc), _ptr(x), _ptr(q), _ptr(scales), _stream(stream))


def vc_checkpoint_unpack(desc, q, scales, y, stream=None):
    _call("vc_checkpoint_unpack", ctypes.byref(desc), _ptr(q), _ptr(scales), _ptr(y), _stream(stream))


def vc_embedding_fwd(desc, ids, table, out, stream=None):
    _call("vc_embedding_fwd", ctypes.byref(desc), _ptr(ids), _ptr(table), _ptr(out), _stream(stream))


def vc_embedding_bwd_workspace_bytes(desc) -> int:
    return _lib().vc_embedding_bwd_workspace_bytes(ctypes.byref(desc))


def vc_embedding_bwd(desc, ids, dout, dtable, workspace, workspace_bytes, stream=None):
    _call("vc_embedding_bwd", ctypes.byref(desc), _ptr(ids), _ptr(dout), _ptr(dtable), _ptr(workspace),
          int(workspace_bytes), _stream(stream))


# --------------------------------------------------------------------------
# Gated residual with the norms before and after a block
# --------------------------------------------------------------------------

def make_residual_desc(rows, cols, samples=1, norm="layer", post_norm=None, residual_scale=1.0, eps=1e-5, plus_one=True,
                       checkpoint=False):
    """Descriptor of a gated residual over rows x cols of `samples` samples: h = residual_scale * x + gate * P(a),
    y = N(h) * (1 + scale) + shift (plus_one False: N(h) * scale + shift). norm (N) and post_norm (P): "layer", "rms" or None.
    checkpoint: what the backward needs of h and a is kept in 8 bits (see checkpoint_pack)."""
    for k in (norm, post_norm):
        if k not in NORMS:
            raise ValueError('a norm is "layer", "rms" or None, got %r' % (k,))
    return vc_residualnorm_desc(int(rows), int(cols), int(samples), 0, 0, 0, NORMS[norm], NORMS[post_norm], 0,
                                1 if plus_one else 0, 1 if checkpoint else 0, 1, float(residual_scale), float(eps))


class Packed8(NamedTuple):
    """A tensor in 8 bits: q int8 of its shape, scales fp32 [..., ceil(columns / 128)], and the type it had."""
    q: object
    scales: object
    dtype: object


class ResidualSaved(NamedTuple):
    """What a residual_norm_bwd takes of its forward. h and a: tensors, or with a checkpoint Packed8. stats: fp32 [4, rows],
    means and reciprocal deviations of h, then of a; those of rows that take no part, of norms that there are not, and the
    means of RMS norms are not defined."""
    desc: object
    h: object
    a: object
    gate: object
    scale: object
    shift: object
    post_weight: object
    cu: object
    lens: object
    stats: object
    y_dtype: object


_CURRENT = []  # the current device's number, and a device's current stream


def _call_on(device, name, desc, *args):
    """The library's `name` with `device` current and its current stream; args: tensors, addresses or None. Small calls spend
    more time here than on the GPU, hence no wrapper for each argument."""
    import torch
    if not _CURRENT:
        _CURRENT[:] = (getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device),  # both at once: threads share it
                       getattr(torch._C, "_cuda_getCurrentRawStream", lambda i: torch.cuda.current_stream(i).cuda_stream))
    number, stream = _CURRENT
    f = getattr(_lib(), name)
    p = [t if t is None or type(t) is int else t.data_ptr() for t in args]
    i = device.index
    if i == number():
        st = f(ctypes.byref(desc), *p, stream(i))
    else:
        with torch.cuda.device(device):
            st = f(ctypes.byref(desc), *p, stream(i))
    if st:
        raise JointAttnError(st, name)


_TYPES = {}
_COLS = 0x7fffffff  # more columns than any descriptor takes: what a call with more of them says, not the number's low 32 bits


def _type(name, t):
    """VC_BF16 or VC_FP32"""
    if not _TYPES:
        import torch
        _TYPES.update({torch.bfloat16: 0, torch.float32: 1})
    k = _TYPES.get(t.dtype)
    if k is None:
        raise ValueError("%s must be torch.bfloat16 or torch.float32, got %s" % (name, t.dtype))
    return k


def _new(t, shape, dtype, device):
    """A contiguous tensor; of one that is just so and at hand it takes less time."""
    import torch
    if t is not None and t.dtype is dtype and t.is_contiguous():
        return torch.empty_like(t, memory_format=torch.contiguous_format)
    return torch.empty(shape, dtype=dtype, device=device)


def _vector(name, p, cols, S, every, dtype):
    """Appends a parameter to the checks; its stride between samples."""
    if p.dim() == 1:
        every.append((name, p, (cols,), dtype, False))
        return SHARED
    every.append((name, p, (S, cols), dtype, True))
    if p.is_contiguous():
        return 0
    strides = p.stride()
    if S == 1 and strides[-1] == 1:
        return 0
    if len(strides) != 2 or strides[1] != 1 or strides[0] < cols:
        raise ValueError("%s must be [columns], or [samples, columns] with contiguous rows" % name)
    return strides[0]


def _vectors(d, every, gate, scale, shift, post_weight):
    """Appends the parameters of a call to its checks, and sets the descriptor's type and strides of them."""
    cols, dtype = d.cols, None
    for name, p in (("gate", gate), ("scale", scale), ("shift", shift), ("post_weight", post_weight)):
        if p is None:
            continue
        if dtype is None:
            dtype = p.dtype
            d.param_type = _type("gate, scale, shift and post_weight", p)
        if name == "post_weight":
            every.append((name, p, (cols,), dtype, False))
        else:
            setattr(d, name + "_stride", _vector(name, p, cols, d.samples, every, dtype))


def _residual_desc(desc, x, a, gate, scale, shift, post_weight, cu, lens, y_type):
    """A copy of the descriptor with the types and strides of the tensors of one call, checked."""
    import torch
    d = vc_residualnorm_desc.from_buffer_copy(desc)
    cols, S = d.cols, d.samples
    shape = (d.rows, cols)
    d.x_type = _type("x", x)
    d.x_stride = _row_stride("x", x)
    every = [("x", x, shape, x.dtype, True)]
    d.y_type = y_type
    if a is not None:
        every.append(("a", a, shape, a.dtype, True))
        d.a_stride = _row_stride("a", a)
    _vectors(d, every, gate, scale, shift, post_weight)
    if cu is not None:
        d.packed = 1
        every.append(("cu", cu, (S + 1,), torch.int32, False))
    if lens is not None:
        every.append(("lens", lens, (S,), torch.int32, False))
    _check_all(every)
    return d


def _kept(rows, cols, device, dtype):
    import torch
    return Packed8(torch.empty((rows, cols), dtype=torch.int8, device=device),
                   torch.empty((rows, (cols + BLOCK - 1) // BLOCK), dtype=torch.float32, device=device), dtype)


def _stat_ptrs(stats, rows):
    """Addresses of the four rows of the statistics."""
    if stats is None:
        return None, None, None, None
    p = stats.data_ptr()
    return p, p + 4 * rows, p + 8 * rows, p + 12 * rows


def residual_norm_fwd(x, a, desc, gate=None, scale=None, shift=None, post_weight=None, cu=None, lens=None, y_dtype=None):
    """(h, y, saved): the residual stream x [rows, columns] with a block's output a taken in, and its norm for the next
    block; `saved` is what residual_norm_bwd takes. a None: the norm alone (h is x). gate, scale, shift: [columns],
    shared by all samples, or [samples, columns], of which consecutive samples may lie further apart, as in slices of one
    projection. Rows are in equal slots, or with cu (int32 [samples + 1]) in those; the first lens[s] (int32 [samples]) of a
    slot take part. All other rows of h and y are 0. x and a: bf16 or fp32 (a not fp32 with x bf16), rows may lie further apart; h has x's
    type, y a's (without a: y_dtype, or x's)."""
    import torch
    if y_dtype is None:
        y_dtype = x.dtype if a is None else a.dtype
        y_type = _type("x" if a is None else "a", x if a is None else a)
    elif a is not None and y_dtype is not a.dtype:
        raise ValueError("y has a's type, %s" % a.dtype)
    elif y_dtype is not torch.bfloat16 and y_dtype is not torch.float32:
        raise ValueError("y_dtype must be torch.bfloat16 or torch.float32, got %s" % y_dtype)
    else:
        y_type = 1 if y_dtype is torch.float32 else 0
    d = _residual_desc(desc, x, a, gate, scale, shift, post_weight, cu, lens, y_type)
    rows, cols, dev = d.rows, d.cols, x.device
    shape = (rows, cols)
    h = None if a is None else _new(x, shape, x.dtype, dev)
    y = stats = h8 = a8 = None
    if d.norm:
        y = _new(x if a is None else a, shape, y_dtype, dev)
    if d.norm or d.post_norm:
        stats = torch.empty((4, rows), dtype=torch.float32, device=dev)
    if d.checkpoint:
        h8 = _kept(rows, cols, dev, x.dtype) if d.norm else None
        a8 = None if a is None else _kept(rows, cols, dev, a.dtype)
    _call_on(dev, "vc_residualnorm_fwd", d, x, a, gate, scale, shift, post_weight, cu, lens, h, y, *_stat_ptrs(stats, rows),
             h8 and h8.q, h8 and h8.scales, a8 and a8.q, a8 and a8.scales)
    if h is None:
        h = x
    if not d.checkpoint:
        h8, a8 = (h if d.norm else None), a
    return h, y, ResidualSaved(d, h8, a8, gate, scale, shift, post_weight, cu, lens, stats, y_dtype)


def residual_norm_bwd(dh, dy, saved, ws=None, want=(True,) * 6):
    """(dx, da, dgate, dscale, dshift, dpost_weight) from the gradients of h and y (either may be None: 0) and what the
    forward saved; None where there was no such input, or where `want` has it as not wanted. Vectors' gradients have their
    vectors' shape. Rows that take no part are 0."""
    import torch
    s = saved
    h, a, hs, as_ = s.h, s.a, None, None
    d = vc_residualnorm_desc.from_buffer_copy(s.desc)
    if d.checkpoint:
        h, hs = (None, None) if h is None else (h.q, h.scales)
        a, as_ = (None, None) if a is None else (a.q, a.scales)
    if dh is None and dy is None:
        raise ValueError("dh and dy are both None")
    if not d.norm and (dh is None or dy is not None):
        raise ValueError("there is no y without a norm")
    shape, every = (d.rows, d.cols), []
    types = (torch.bfloat16, torch.float32)
    if dh is not None:
        every.append(("dh", dh, shape, types[d.x_type], True))
        d.dh_stride = _row_stride("dh", dh)
    if dy is not None:
        every.append(("dy", dy, shape, types[d.y_type], True))
        d.dy_stride = _row_stride("dy", dy)
    if s.stats is not None:
        every.append(("saved.stats", s.stats, (4, d.rows), torch.float32, False))
    # What was saved may lie otherwise than it did (a hook of the saved tensors packs strided ones close, say).
    blocks = (d.rows, (d.cols + BLOCK - 1) // BLOCK)
    for name, t, scales, of in (("h", h, hs, d.x_type), ("a", a, as_, d.y_type)):
        if t is None:
            continue
        every.append(("saved." + name, t, shape, torch.int8 if d.checkpoint else types[of], not d.checkpoint))
        if d.checkpoint:
            every.append(("saved.%s.scales" % name, scales, blocks, torch.float32, False))
    if not d.checkpoint:
        if a is not None:
            d.a_stride = _row_stride("saved.a", a)
        elif h is not None:
            d.x_stride = _row_stride("saved.h", h)
        if a is not None and h is not None and not h.is_contiguous():
            raise ValueError("saved.h must be contiguous")
    _vectors(d, every, s.gate, s.scale, s.shift, s.post_weight)
    if s.cu is not None:
        every.append(("saved.cu", s.cu, (d.samples + 1,), torch.int32, False))
    if s.lens is not None:
        every.append(("saved.lens", s.lens, (d.samples,), torch.int32, False))
    _check_all(every)
    dev = every[0][1].device
    dx = _new(dh, shape, types[d.x_type], dev) if want[0] else None
    da = _new(dy, shape, types[d.y_type], dev) if a is not None and want[1] else None
    vectors, sums = [], False
    for p, w in zip((s.gate, s.scale, s.shift, s.post_weight), want[2:]):
        g = None
        if p is not None and w:
            g, sums = _new(p, p.shape, p.dtype, dev), True
        vectors.append(g)
    if dx is None and da is None and not sums:
        return (None,) * 6
    if ws is None and sums:
        ws = _workspace(_lib().vc_residualnorm_bwd_workspace_bytes(ctypes.byref(d)), dev)
    _call_on(dev, "vc_residualnorm_bwd", d, dh, dy, h, a, hs, as_, s.gate, s.scale, s.post_weight, s.cu, s.lens,
             *_stat_ptrs(s.stats, d.rows), dx, da, *vectors, ws, 0 if ws is None else _ws_bytes(ws, dev))
    return (dx, da, *vectors)


# --------------------------------------------------------------------------
# Activation checkpoints in 8 bits
# --------------------------------------------------------------------------

def _rows_of(x):
    """(rows, columns, stride) of x as rows of its last dimension."""
    if x.dim() == 0:
        raise ValueError("x has shape (), expected [..., columns]")
    if x.numel() == 0:
        return 0, x.shape[-1], 0
    return x.numel() // x.shape[-1], x.shape[-1], _row_stride("x", x)


def checkpoint_pack(x, out=None):
    """x (bf16 or fp32; contiguous, or [rows, columns] with rows further apart) in 8 bits, a scale for each 128
    columns: a Packed8 of 1 + 1/32 bytes an element. Off by at most half a step, the largest |x| of the 128 over 254; a block
    that holds an infinity or a NaN unpacks to NaN. out: a Packed8 of x's shape and type to write to."""
    import torch
    f32 = _type("x", x)
    rows, cols, stride = _rows_of(x)
    shape = x.shape
    kept, blocks = out, (*shape[:-1], (cols + BLOCK - 1) // BLOCK)
    if out is None:
        _check_all([("x", x, shape, x.dtype, True)])
        kept = Packed8(torch.empty_like(x, dtype=torch.int8, memory_format=torch.contiguous_format),
                       torch.empty(blocks, dtype=torch.float32, device=x.device), x.dtype)
    elif out.dtype is not x.dtype:
        raise ValueError("out is of %s, x of %s" % (out.dtype, x.dtype))
    else:
        _check_all([("x", x, shape, x.dtype, True), ("out.q", out.q, shape, torch.int8, False),
                    ("out.scales", out.scales, blocks, torch.float32, False)])
    if rows:
        _call_on(x.device, "vc_checkpoint_pack", vc_checkpoint_desc(rows, min(cols, _COLS), f32, stride), x, kept.q, kept.scales)
    return kept


def checkpoint_unpack(kept, dtype=None, out=None):
    """The values that checkpoint_pack kept, in the type they had or `dtype`; into `out` where that is given."""
    import torch
    q, scales = kept.q, kept.scales
    rows, cols, _ = _rows_of(q)
    if out is None:
        out = torch.empty_like(q, dtype=kept.dtype if dtype is None else dtype, memory_format=torch.contiguous_format)
    elif dtype is not None and out.dtype is not dtype:
        raise ValueError("out must be %s, got %s" % (dtype, out.dtype))
    f32 = _type("out", out)
    shape = q.shape
    _check_all([("q", q, shape, torch.int8, False),
                ("scales", scales, (*shape[:-1], (cols + BLOCK - 1) // BLOCK), torch.float32, False),
                ("out", out, shape, out.dtype, False)])
    if rows:
        _call_on(q.device, "vc_checkpoint_unpack", vc_checkpoint_desc(rows, min(cols, _COLS), f32, 0), q, scales, out)
    return out


class _Whole(NamedTuple):
    """A saved tensor as it is, and how often it had been changed in place."""
    tensor: object
    version: int


# Operations whose results are values of their operands: casts, copies, views, joined tensors.
_MOVES = frozenset("%sBackward" % n for n in (
    "ToCopy", "Clone", "Alias", "View", "UnsafeView", "ReshapeAlias", "T", "Transpose", "Permute", "Select", "Slice", "Split",
    "SplitWithSizes", "Unbind", "Squeeze", "Unsqueeze", "Expand", "AsStrided", "Cat", "Stack"))


def _of_leaves(t):
    """Whether t is a leaf or holds the values of leaves in another type, order or place."""
    t = t if t._base is None else t._base
    open_, seen = [] if t.is_leaf else [t.grad_fn], set()
    while open_:
        f = open_.pop()
        if f is None or f in seen or f.name() == "torch::autograd::AccumulateGrad":  # a constant, or a leaf's end of the graph
            continue
        seen.add(f)
        if f.name().rstrip("0123456789") not in _MOVES:
            return False
        open_ += [g for g, _ in f.next_functions]
    return True


def saved_in_8bit(min_elements=1 << 16):
    """A context in which autograd keeps activations in 8 bits: contiguous tensors of bf16, of at least min_elements elements, two
    dimensions and 64 columns, that an operation saves for its backward are packed, and unpacked where the backward asks for
    them. Leaves (parameters, inputs) stay as they are, and so do casts, copies, views and joined forms of them (weights in bf16 of
    parameters in 32 bits): an input's gradient is that of the weight itself. Weights that are computed otherwise are taken for activations. Tensors of 32 bits stay too
    (log-sum-exps, statistics). A tensor that several operations save is packed for each of them. Of an attention of this package v
    and o are packed; q, k and a bias stay, since the backward computes the probabilities again from them with the exact log-sum-exps.
    The vectors of a residual_norm stay, which are few and weigh every row.
    Results of log_softmax (cross_entropy) stay, of which the backward takes exponentials. Other operations whose backward takes exponentials
    of what they saved (a fused attention of another origin, logsumexp) cannot be told from the rest here and do not belong in the context."""
    import torch

    def pack(t):
        if (t.device.type != "cuda" or t.dtype is not torch.bfloat16 or t.dim() < 2 or
                t.numel() < min_elements or t.shape[-1] < 64 or not t.is_contiguous() or
                hasattr(t, "_vc_save_whole") or _of_leaves(t) or "LogSoftmax" in (t.grad_fn.name() if t.grad_fn else "")):
            return _Whole(t.detach(), t._version)  # a result that its operation saves would hold that operation, and itself through it
        return checkpoint_pack(t.detach())

    def unpack(kept):
        if isinstance(kept, Packed8):
            return checkpoint_unpack(kept)
        if kept.tensor._version != kept.version:  # autograd itself does not look where there are hooks
            raise RuntimeError("a tensor %s that an operation saved for its backward was changed in place since" % (tuple(kept.tensor.shape),))
        return kept.tensor

    return torch.autograd.graph.saved_tensors_hooks(pack, unpack)


# --------------------------------------------------------------------------
# Embedding of tokens
# --------------------------------------------------------------------------

def _ids(ids):
    import torch
    if ids.dtype is not torch.int64 and ids.dtype is not torch.int32:
        raise ValueError("ids must be torch.int32 or torch.int64, got %s" % ids.dtype)
    return 1 if ids.dtype is torch.int64 else 0


def embedding_fwd(ids, table, scale=1.0, padding_id=None, dtype=None, out=None):
    """scale * table[ids] of the table's type or `dtype`: ids int32 or int64 of any shape, table [vocab, columns] in bf16 or
    fp32 (rows may lie further apart). Tokens of the padding id, or of none of the table's, get zeros."""
    import torch
    i64, tf = _ids(ids), _type("table", table)
    if table.dim() != 2:
        raise ValueError("table has shape %s, expected [vocab, columns]" % (tuple(table.shape),))
    V, cols = table.shape
    shape = (*ids.shape, cols)
    if out is None:
        out = torch.empty(shape, dtype=table.dtype if dtype is None else dtype, device=table.device)
    elif dtype is not None and out.dtype is not dtype:
        raise ValueError("out must be %s, got %s" % (dtype, out.dtype))
    of = _type("out", out)
    _check_all([("ids", ids, ids.shape, ids.dtype, False), ("table", table, (V, cols), table.dtype, True),
                ("out", out, shape, out.dtype, False)])
    desc = vc_embedding_desc(ids.numel(), V, -1 if padding_id is None else padding_id, _row_stride("table", table), min(cols, _COLS), i64, tf,
                             of, scale, 0)
    if desc.tokens:
        _call_on(table.device, "vc_embedding_fwd", desc, ids, table, out)
    return out


def embedding_bwd(dout, ids, vocab, scale=1.0, padding_id=None, dtype=None, into=None, ws=None):
    """The table's gradient [vocab, columns], of dout's type or `dtype` (bf16 or fp32): scale times the sum of the rows of
    dout whose tokens have the id, zeros for ids that no token has. into: a gradient that is there, to which the sums are added
    instead (and which is returned). dout: ids' shape and columns, contiguous or [tokens, columns] with rows further apart."""
    import torch
    i64, of = _ids(ids), _type("dout", dout)
    cols = dout.shape[-1] if dout.dim() else 0
    if into is None:
        grad = torch.empty((vocab, cols), dtype=dout.dtype if dtype is None else dtype, device=dout.device)
    elif dtype is not None and into.dtype is not dtype:
        raise ValueError("into must be %s, got %s" % (dtype, into.dtype))
    else:
        grad = into
    gf = _type("dtable", grad)
    _check_all([("dout", dout, (*ids.shape, cols), dout.dtype, True), ("ids", ids, ids.shape, ids.dtype, False),
                ("into", grad, (vocab, cols), grad.dtype, False)])
    desc = vc_embedding_desc(ids.numel(), vocab, -1 if padding_id is None else padding_id, _row_stride("dout", dout), min(cols, _COLS), i64,
                             gf, of, scale, 0 if into is None else 1)
    if not desc.tokens:
        return grad.zero_() if into is None else grad
    if ws is None:
        ws = _workspace(_lib().vc_embedding_bwd_workspace_bytes(ctypes.byref(desc)), dout.device)
    _call_on(dout.device, "vc_embedding_bwd", desc, ids, dout, grad, ws, _ws_bytes(ws, dout.device))
    return grad


# --------------------------------------------------------------------------
# Differentiable forms
# --------------------------------------------------------------------------

_AUTOGRAD = {}


def _autograd_functions():
    if _AUTOGRAD:
        return _AUTOGRAD
    import torch
    from torch.autograd.function import once_differentiable

    class ResidualNorm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, a, gate, scale, shift, post_weight, desc, cu, lens, y_dtype):
            ctx.set_materialize_grads(False)
            h, y, s = residual_norm_fwd(x, a, desc, gate, scale, shift, post_weight, cu, lens, y_dtype)
            kept = (s.h, s.a)
            if s.desc.checkpoint:
                kept = tuple(t for k in kept for t in ((None, None) if k is None else (k.q, k.scales)))
            _save_whole(gate, scale, shift, post_weight)
            ctx.save_for_backward(*kept, gate, scale, shift, post_weight, cu, lens, s.stats)
            ctx.desc, ctx.types = s.desc, (x.dtype, s.y_dtype)
            if a is None:  # h is x: the caller has it
                return y
            return (h, y) if y is not None else h

        @staticmethod
        @once_differentiable
        def backward(ctx, *grads):
            t, d = ctx.saved_tensors, ctx.desc
            if d.checkpoint:
                kept = tuple(None if q is None else Packed8(q, s, dt) for q, s, dt in zip(t[0:4:2], t[1:4:2], ctx.types))
                t = t[4:]
            else:
                kept, t = t[:2], t[2:]
            dh, dy = grads if len(grads) == 2 else (None, *grads) if kept[1] is None else (*grads, None)
            if dh is None and dy is None:
                return (None,) * 10
            cont = lambda g: None if g is None else g.contiguous()  # noqa: E731
            saved = ResidualSaved(d, *kept, *t, ctx.types[1])
            return residual_norm_bwd(cont(dh), cont(dy), saved, want=ctx.needs_input_grad[:6]) + (None,) * 4

    class Embedding(torch.autograd.Function):
        @staticmethod
        def forward(ctx, ids, table, scale, padding_id, dtype):
            ctx.save_for_backward(ids)
            ctx.how = (table.shape[0], scale, padding_id, table.dtype)
            return embedding_fwd(ids, table, scale, padding_id, dtype)

        @staticmethod
        @once_differentiable
        def backward(ctx, dout):
            return (None, embedding_bwd(dout.contiguous(), ctx.saved_tensors[0], *ctx.how), None, None, None)

    _AUTOGRAD.update(residual=ResidualNorm, embedding=Embedding)
    return _AUTOGRAD


def residual_norm(x, a, desc, gate=None, scale=None, shift=None, post_weight=None, cu=None, lens=None, y_dtype=None):
    """Differentiable gated residual (see residual_norm_fwd): (h, y) with gradients of x, a, gate, scale, shift and
    post_weight; y alone without a, h alone where the descriptor has no norm. For a captured graph take residual_norm_fwd and
    residual_norm_bwd: autograd itself waits, across streams, for other graphs of the same leaves."""
    return _autograd_functions()["residual"].apply(x, a, gate, scale, shift, post_weight, desc, cu, lens, y_dtype)


def embedding(ids, table, scale=1.0, padding_id=None, dtype=None):
    """Differentiable embedding (see embedding_fwd): the table's gradient has the table's type. For a captured graph take
    embedding_fwd and embedding_bwd (see residual_norm)."""
    return _autograd_functions()["embedding"].apply(ids, table, scale, padding_id, dtype)
