"""The text tower's operators: packed attention (sequences of different lengths, grouped heads, causal or
not, with a learned bias per bucket of the relative position) and layer norm.

As everywhere in this package, the tensor-level helpers check and marshal arguments and allocate outputs;
every step of the computation runs in the library's HIP kernels (include/vc_jointattn.h).
"""
from __future__ import annotations

import ctypes

from paper_2501_08453_amd import (_call, _check_placed, _check_shape, _lib, _ptr, _save_whole, _stream, _workspace,
                                  vc_layernorm_desc, vc_packedattn_desc)

MAX_DISTANCE = 512   # largest max_distance of a bias (VC_ERR_SHAPE beyond)
MAX_BUCKETS = 1024


# --------------------------------------------------------------------------
# Raw entry points with the C names (pointers are ints or torch tensors).
# --------------------------------------------------------------------------

def vc_packedattn_fwd_workspace_bytes(desc) -> int:
    return _lib().vc_packedattn_fwd_workspace_bytes(ctypes.byref(desc))


def vc_packedattn_bwd_workspace_bytes(desc) -> int:
    return _lib().vc_packedattn_bwd_workspace_bytes(ctypes.byref(desc))


def vc_packedattn_fwd(desc, q, k, v, cu_q, cu_k, len_q, len_k, bias, buckets, o, lse, workspace, workspace_bytes,
                      stream=None):
    _call("vc_packedattn_fwd", ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(cu_q), _ptr(cu_k), _ptr(len_q),
          _ptr(len_k), _ptr(bias), _ptr(buckets), _ptr(o), _ptr(lse), _ptr(workspace), int(workspace_bytes),
          _stream(stream))


def vc_packedattn_bwd(desc, q, k, v, o, lse, dout, cu_q, cu_k, len_q, len_k, bias, buckets, dq, dk, dv, dbias,
                      workspace, workspace_bytes, stream=None):
    _call("vc_packedattn_bwd", ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(dout), _ptr(cu_q),
          _ptr(cu_k), _ptr(len_q), _ptr(len_k), _ptr(bias), _ptr(buckets), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dbias),
          _ptr(workspace), int(workspace_bytes), _stream(stream))


def vc_layernorm_fwd(desc, x, weight, bias, y, mean, rstd, stream=None):
    _call("vc_layernorm_fwd", ctypes.byref(desc), _ptr(x), _ptr(weight), _ptr(bias), _ptr(y), _ptr(mean), _ptr(rstd),
          _stream(stream))


def vc_layernorm_bwd_workspace_bytes(desc) -> int:
    return _lib().vc_layernorm_bwd_workspace_bytes(ctypes.byref(desc))


def vc_layernorm_bwd(desc, dout, x, weight, mean, rstd, dx, dweight, dbias, workspace, workspace_bytes, stream=None):
    _call("vc_layernorm_bwd", ctypes.byref(desc), _ptr(dout), _ptr(x), _ptr(weight), _ptr(mean), _ptr(rstd), _ptr(dx),
          _ptr(dweight), _ptr(dbias), _ptr(workspace), int(workspace_bytes), _stream(stream))


# --------------------------------------------------------------------------
# Packed attention
# --------------------------------------------------------------------------

def make_packed_desc(sequences, heads, kv_heads, head_dim, total_q, total_k, max_q, max_k, causal=False, scale=None,
                     num_buckets=0, max_distance=0):
    """Descriptor of a packed call: `sequences` slots in total_q query rows and total_k key rows, none of more than
    max_q and max_k rows (upper bounds are enough, exact ones give the best division of the work). With num_buckets, every call takes a
    bias [heads, num_buckets] and the buckets of the distances -max_distance .. max_distance."""
    return vc_packedattn_desc(int(sequences), int(heads), int(kv_heads), int(head_dim), int(total_q), int(total_k),
                              min(int(max_q), int(total_q)), min(int(max_k), int(total_k)), 0, 0, 0, 1 if causal else 0,
                              float(scale) if scale else 0.0, int(num_buckets),
                              int(max_distance), 0)


def packed_fwd_workspace(desc, device):
    return _workspace(vc_packedattn_fwd_workspace_bytes(desc), device)


def packed_bwd_workspace(desc, device):
    return _workspace(vc_packedattn_bwd_workspace_bytes(desc), device)


def relative_buckets(num_buckets, max_distance, bidirectional=True, device="cuda"):
    """Buckets of the relative positions d = key - query, -max_distance <= d <= max_distance (int32
    [2 max_distance + 1]): with n = |d| (bidirectional, where the keys behind the query have the upper half of the
    buckets) or max(-d, 0), of the h buckets of a direction the first h // 2 hold one n each, the others
    ranges that widen with the logarithm of n up to max_distance. The borders are found in whole numbers."""
    import torch
    num_buckets, max_distance = int(num_buckets), int(max_distance)
    half = num_buckets // 2 if bidirectional else num_buckets
    exact = half // 2
    if exact < 1 or num_buckets > MAX_BUCKETS or not exact < max_distance <= MAX_DISTANCE:
        raise ValueError("relative_buckets: %d buckets over distances up to %d" % (num_buckets, max_distance))
    wide = half - exact
    side, k = [], 0
    for n in range(max_distance + 1):
        # bucket exact + k from (n / exact)^wide >= (max_distance / exact)^k on
        while k < wide - 1 and n ** wide >= max_distance ** (k + 1) * exact ** (wide - k - 1):
            k += 1
        side.append(n if n < exact else exact + k)
    ahead = [half + b for b in side[1:]] if bidirectional else [0] * max_distance
    return torch.tensor(side[:0:-1] + [0] + ahead, dtype=torch.int32, device=device)


def _launch(device, f, *args):
    """f(*args) with `device` current (the library launches on the current device)."""
    import torch
    if device.index == torch.cuda.current_device():
        return f(*args)
    with torch.cuda.device(device):
        return f(*args)


def _ws_bytes(ws, device):
    """Bytes of a workspace given by the caller: contiguous, on the device of the call's tensors (the kernels write to it)."""
    if ws.device != device:
        raise ValueError("ws is on %s, the call's tensors on %s" % (ws.device, device))
    if not ws.is_contiguous():
        raise ValueError("ws must be contiguous")
    return ws.numel() * ws.element_size()


def _token_stride(name, t):
    """Elements between the rows of consecutive tokens of a [tokens, heads, D] tensor whose heads are contiguous; 0
    where the whole tensor is."""
    if t.is_contiguous():
        return 0
    n, h, d = t.shape
    if t.stride(2) != 1 or (h > 1 and t.stride(1) != d):
        raise ValueError("the heads of %s must be contiguous" % name)
    if n == 1:
        return 0
    if t.stride(0) < h * d or t.stride(0) % 8:
        raise ValueError("%s: tokens %d elements apart (at least %d, a multiple of 8)" % (name, t.stride(0), h * d))
    return t.stride(0)


def _fits(t, shape, dtype, index, strided=False):
    return t.shape == shape and t.dtype is dtype and t.get_device() == index and (strided or t.is_contiguous())


def _check_all(every):
    """every: (name, tensor, shape, dtype, strided) of one call; all on one GPU, contiguous unless strided. The plain
    comparisons first, as they cost a small call as much as its launch; what is wrong is then found out in the
    order of the package's checks: shapes and dtypes of all, then where they lie."""
    index = every[0][1].get_device()
    if index >= 0:
        for _, t, shape, dtype, strided in every:
            if not _fits(t, shape, dtype, index, strided):
                break
        else:
            return
    for name, t, shape, dtype, _ in every:
        _check_shape(name, t, shape, dtype)
    for name, t, _, _, strided in every:
        if t.device.type != "cuda":
            raise ValueError("%s must be on a GPU" % name)
        if t.device != every[0][1].device:
            raise ValueError("%s is on %s, %s on %s" % (name, t.device, every[0][0], every[0][1].device))
        if not strided:
            _check_placed(name, t)


def _check_packed(desc, q, k, v, cu_q, cu_k, len_q, len_k, bias, buckets, like_q, like_k, lse):
    """Checks the tensors of one call against each other and the descriptor; returns a copy of the descriptor with
    the tensors' strides. like_q, like_k: further (name, tensor) with the shape of q (of k)."""
    import torch
    bf16, i32 = torch.bfloat16, torch.int32
    d = vc_packedattn_desc.from_buffer_copy(desc)
    S, H, D = d.sequences, d.heads, d.head_dim
    if (d.num_buckets > 0) != (bias is not None) or (bias is None) != (buckets is None):
        raise ValueError("a bias and its buckets go with a descriptor of num_buckets > 0, and only with that")
    sq, sk = (d.total_q, H, D), (d.total_k, d.kv_heads, D)
    every = [("q", q, sq, bf16, True), ("k", k, sk, bf16, True), ("v", v, sk, bf16, True), ("cu_q", cu_q, (S + 1,), i32, False),
             ("cu_k", cu_k, (S + 1,), i32, False)]
    if len_q is not None:
        every.append(("len_q", len_q, (S,), i32, False))
    if len_k is not None:
        every.append(("len_k", len_k, (S,), i32, False))
    if bias is not None:
        every.append(("bias", bias, (H, d.num_buckets), bf16, False))
        every.append(("buckets", buckets, (2 * d.max_distance + 1,), i32, False))
    for name, t in like_q:
        every.append((name, t, sq, bf16, False))
    for name, t in like_k:
        every.append((name, t, sk, bf16, False))
    every.append(("lse", lse, (H, d.total_q), torch.float32, False))
    _check_all(every)
    d.q_stride, d.k_stride, d.v_stride = _token_stride("q", q), _token_stride("k", k), _token_stride("v", v)
    return d


def packed_fwd(q, k, v, desc, cu_q, cu_k, len_q=None, len_k=None, bias=None, buckets=None, out=None, lse=None, ws=None):
    """(o, lse) of packed attention: q [total_q, heads, D], k and v [total_k, kv_heads, D] in bf16 (tokens may be any
    multiple of 8 elements apart, as in slices of one projection), lse [heads, total_q]. Sequence s has the rows
    [cu_q[s], cu_q[s+1]) and [cu_k[s], cu_k[s+1]) or, of these, the first len_q[s] and len_k[s]. Rows outside every
    slot are 0 (lse: -inf) in each tensor made here, and left as they were in `out` or `lse` where that is given."""
    import torch
    clear = (1 if lse is None else 2) if out is None else 3 if lse is None else 0  # both, out, lse, none
    if out is None:
        out = torch.empty((desc.total_q, desc.heads, desc.head_dim), dtype=torch.bfloat16, device=q.device)
    if lse is None:
        lse = torch.empty((desc.heads, desc.total_q), dtype=torch.float32, device=q.device)
    d = _check_packed(desc, q, k, v, cu_q, cu_k, len_q, len_k, bias, buckets, (("out", out),), (), lse)
    d.clear_outside = clear
    ws = packed_fwd_workspace(d, q.device) if ws is None else ws
    _launch(q.device, vc_packedattn_fwd, d, q, k, v, cu_q, cu_k, len_q, len_k, bias, buckets, out, lse, ws,
            _ws_bytes(ws, q.device))
    return out, lse


def packed_bwd(q, k, v, o, lse, dout, desc, cu_q, cu_k, len_q=None, len_k=None, bias=None, buckets=None, ws=None, dq=None,
               dk=None, dv=None, want_dbias=True):
    """(dq, dk, dv, dbias) of packed attention; dbias (bf16 [heads, num_buckets]) is None without a bias or where it
    is not wanted. Rows outside every slot are 0 in tensors made here, and left as they were where dq, dk
    and dv are given (all three or none)."""
    import torch
    made = dq is None and dk is None and dv is None
    if not made and (dq is None or dk is None or dv is None):
        raise ValueError("dq, dk and dv are given together or not at all")
    if made:
        new = lambda n, h: torch.empty((n, h, desc.head_dim), dtype=torch.bfloat16, device=q.device)  # noqa: E731
        dq, dk, dv = new(desc.total_q, desc.heads), new(desc.total_k, desc.kv_heads), new(desc.total_k, desc.kv_heads)
    d = _check_packed(desc, q, k, v, cu_q, cu_k, len_q, len_k, bias, buckets,
                      (("o", o), ("dout", dout), ("dq", dq)), (("dk", dk), ("dv", dv)), lse)
    d.clear_outside = 1 if made else 0
    dbias = torch.empty_like(bias) if bias is not None and want_dbias else None
    ws = packed_bwd_workspace(d, q.device) if ws is None else ws
    _launch(q.device, vc_packedattn_bwd, d, q, k, v, o, lse, dout, cu_q, cu_k, len_q, len_k, bias, buckets, dq, dk, dv, dbias,
            ws, _ws_bytes(ws, q.device))
    return dq, dk, dv, dbias


# --------------------------------------------------------------------------
# Layer norm
# --------------------------------------------------------------------------

def _row_stride(name, t):
    """Elements between the rows of x, seen as [rows, columns]: 0 if contiguous."""
    if t.is_contiguous():
        return 0
    if t.dim() == 2 and t.stride(1) == 1 and t.stride(0) >= t.shape[1]:
        return t.stride(0)
    raise ValueError("%s must be contiguous, or two-dimensional with contiguous rows" % name)


def _norm_desc(x, weight, bias, eps, dout=None, mean=None, rstd=None, out=None):
    import torch
    if x.dtype is not torch.bfloat16 and x.dtype is not torch.float32:
        raise ValueError("x must be torch.bfloat16 or torch.float32, got %s" % x.dtype)
    shape = x.shape
    if not shape or shape[-1] < 1:
        raise ValueError("x has shape %s, expected [..., columns]" % (tuple(shape),))
    cols = shape[-1]
    first = weight if weight is not None else bias
    if first is not None and first.dtype is not torch.bfloat16 and first.dtype is not torch.float32:
        raise ValueError("weight and bias must be torch.bfloat16 or torch.float32, got %s" % first.dtype)
    if weight is not None and bias is not None and bias.dtype is not weight.dtype:
        raise ValueError("weight and bias must be of one dtype, got %s and %s" % (weight.dtype, bias.dtype))
    every = [("x", x, shape, x.dtype, True)]
    if weight is not None:
        every.append(("weight", weight, (cols,), first.dtype, False))
    if bias is not None:
        every.append(("bias", bias, (cols,), first.dtype, False))
    if dout is not None:
        every.append(("dout", dout, shape, x.dtype, True))
        every.append(("mean", mean, shape[:-1], torch.float32, False))
        every.append(("rstd", rstd, shape[:-1], torch.float32, False))
    if out is not None:
        every.append(("out", out, shape, x.dtype, False))
    _check_all(every)
    return vc_layernorm_desc(x.numel() // cols, cols, 1 if x.dtype is torch.float32 else 0,
                             1 if first is not None and first.dtype is torch.float32 else 0, eps, _row_stride("x", x),
                             0 if dout is None else _row_stride("dout", dout))


def layer_norm_fwd(x, weight=None, bias=None, eps=1e-5, out=None):
    """(y, mean, rstd): layer norm over the last dimension of x (bf16 or fp32; contiguous, or [rows, columns] with
    rows further apart). weight and bias: [columns] in bf16 or fp32. mean and rstd are fp32, for the backward."""
    import torch
    desc = _norm_desc(x, weight, bias, eps, out=out)
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device) if out is None else out
    mean = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    rstd = torch.empty_like(mean)
    if desc.rows:
        _launch(x.device, vc_layernorm_fwd, desc, x, weight, bias, y, mean, rstd)
    return y, mean, rstd


def layer_norm_bwd(dout, x, weight, bias, mean, rstd, ws=None):
    """(dx, dweight, dbias) from the forward's inputs, mean and rstd; dweight (dbias) is None where weight (bias) is."""
    import torch
    desc = _norm_desc(x, weight, bias, 0.0, dout, mean, rstd)
    dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    new = torch.empty_like if desc.rows else torch.zeros_like
    dw, db = (None if t is None else new(t) for t in (weight, bias))
    if desc.rows:
        if ws is None and (dw is not None or db is not None):
            ws = _workspace(vc_layernorm_bwd_workspace_bytes(desc), x.device)
        _launch(x.device, vc_layernorm_bwd, desc, dout, x, weight, mean, rstd, dx, dw, db, ws,
                0 if ws is None else _ws_bytes(ws, x.device))
    return dx, dw, db


# --------------------------------------------------------------------------
# Differentiable forms
# --------------------------------------------------------------------------

_AUTOGRAD = {}


def _autograd_functions():
    if _AUTOGRAD:
        return _AUTOGRAD
    import torch
    from torch.autograd.function import once_differentiable

    class PackedAttention(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v, bias, desc, cu_q, cu_k, len_q, len_k, buckets):
            o, lse = packed_fwd(q, k, v, desc, cu_q, cu_k, len_q, len_k, bias, buckets)
            _save_whole(q, k, bias)
            ctx.save_for_backward(q, k, v, bias, o, lse, cu_q, cu_k, len_q, len_k, buckets)
            ctx.desc = vc_packedattn_desc.from_buffer_copy(desc)  # the caller may change theirs before the backward
            return o

        @staticmethod
        @once_differentiable
        def backward(ctx, do):
            q, k, v, bias, o, lse, cu_q, cu_k, len_q, len_k, buckets = ctx.saved_tensors
            g = packed_bwd(q, k, v, o, lse, do.contiguous(), ctx.desc, cu_q, cu_k, len_q, len_k, bias, buckets,
                           want_dbias=ctx.needs_input_grad[3])
            return g + (None,) * 6

    class LayerNorm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight, bias, eps):
            y, mean, rstd = layer_norm_fwd(x, weight, bias, eps)
            ctx.save_for_backward(x, weight, bias, mean, rstd)
            return y

        @staticmethod
        @once_differentiable
        def backward(ctx, dy):
            x, weight, bias, mean, rstd = ctx.saved_tensors
            return layer_norm_bwd(dy.contiguous(), x, weight, bias, mean, rstd) + (None,)

    _AUTOGRAD.update(packed=PackedAttention, norm=LayerNorm)
    return _AUTOGRAD


def packed_attention(q, k, v, desc, cu_q, cu_k, len_q=None, len_k=None, bias=None, buckets=None):
    """Differentiable packed attention (see packed_fwd): gradients of q, k, v and the bias. For a captured graph take
    packed_fwd and packed_bwd: autograd itself waits, across streams, for other graphs of the same leaves."""
    return _autograd_functions()["packed"].apply(q, k, v, bias, desc, cu_q, cu_k, len_q, len_k, buckets)


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """Differentiable layer norm over the last dimension of x: gradients of x, weight and bias. For a captured graph take
    layer_norm_fwd and layer_norm_bwd (see packed_attention)."""
    return _autograd_functions()["norm"].apply(x, weight, bias, eps)
