"""Training operators of language models on the GPU: layer norm, attention and the loss over a vocabulary, forward and
backward.  Thin ctypes binding of the C boundary in include/ff_ops.h (same names, argument marshalling only) and, on
top of it, functions that take torch tensors: torch is used for device memory and streams, nothing else, and there is
no CPU fallback.

The functions check what they are given (ValueError), allocate their outputs and workspace with torch on the tensors'
device and put the kernels on its current stream; they do not wait.  Captured into a HIP graph, they use the graph's
memory.  What a call refuses on the library's side raises binding.FFSimError.
"""
from __future__ import annotations

import ctypes as C
import math

from . import binding

FF_F32, FF_F16, FF_BF16 = 0, 1, 2

EXPORTS = ["ff_op_layernorm_fwd", "ff_op_layernorm_bwd_workspace_bytes", "ff_op_layernorm_bwd",
           "ff_op_attention_fwd_workspace_bytes", "ff_op_attention_fwd", "ff_op_attention_bwd_workspace_bytes", "ff_op_attention_bwd",
           "ff_op_vocab_loss_fwd_workspace_bytes", "ff_op_vocab_loss_fwd", "ff_op_vocab_loss_bwd_workspace_bytes", "ff_op_vocab_loss_bwd"]


class ff_rows_t(C.Structure):
    _fields_ = [("p", C.c_void_p), ("stride", C.c_int64)]


class ff_heads_t(C.Structure):
    _fields_ = [("p", C.c_void_p), ("batch", C.c_int64), ("head", C.c_int64), ("pos", C.c_int64)]


_WS = [("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]
_u32, _vp = C.c_uint32, C.c_void_p


class ff_layernorm_fwd_t(C.Structure):
    _fields_ = [("dtype", _u32), ("cols", _u32), ("rows", C.c_uint64), ("eps", C.c_float)] + [(n, ff_rows_t) for n in ("x", "res", "h", "y")] + \
        [(n, _vp) for n in ("weight", "bias", "mean", "rstd")]


class ff_layernorm_bwd_t(C.Structure):
    _fields_ = [("dtype", _u32), ("cols", _u32), ("rows", C.c_uint64)] + [(n, ff_rows_t) for n in ("dy", "h", "dh", "dx")] + \
        [(n, _vp) for n in ("weight", "mean", "rstd", "dweight", "dbias")] + _WS


_ATTN = [(n, _u32) for n in ("dtype", "batch", "heads", "kv_heads", "q_len", "kv_len", "head_dim", "causal")] + [("scale", C.c_float)]


class ff_attention_fwd_t(C.Structure):
    _fields_ = _ATTN + [(n, ff_heads_t) for n in ("q", "k", "v", "o")] + [(n, _vp) for n in ("lse", "q_lengths", "kv_lengths")] + _WS


class ff_attention_bwd_t(C.Structure):
    _fields_ = _ATTN + [(n, ff_heads_t) for n in ("dout", "q", "k", "v", "o", "dq", "dk", "dv")] + \
        [(n, _vp) for n in ("lse", "q_lengths", "kv_lengths")] + _WS


_VOCAB = [(n, _u32) for n in ("dtype", "rows", "vocab", "dim")] + [("ignore_index", C.c_int32), ("first_word", C.c_int32)]


class ff_vocab_loss_fwd_t(C.Structure):
    _fields_ = _VOCAB + [(n, ff_rows_t) for n in ("x", "w")] + [(n, _vp) for n in ("targets", "loss", "lse", "target_logit")] + _WS


class ff_vocab_loss_bwd_t(C.Structure):
    _fields_ = _VOCAB + [(n, ff_rows_t) for n in ("x", "w", "dx", "dw")] + [(n, _vp) for n in ("targets", "dloss", "lse")] + _WS


_RECORDS = {"ff_op_layernorm_fwd": ff_layernorm_fwd_t, "ff_op_layernorm_bwd": ff_layernorm_bwd_t, "ff_op_attention_fwd": ff_attention_fwd_t,
            "ff_op_attention_bwd": ff_attention_bwd_t, "ff_op_vocab_loss_fwd": ff_vocab_loss_fwd_t, "ff_op_vocab_loss_bwd": ff_vocab_loss_bwd_t}
_declared = None


def lib():
    """the library with the operators' calls declared"""
    global _declared
    L = binding.lib()
    if _declared is not L:
        for name in EXPORTS:
            f = getattr(L, name)
            record = C.POINTER(_RECORDS[name.replace("_workspace_bytes", "")])
            if name.endswith("_workspace_bytes"):
                f.restype, f.argtypes = C.c_size_t, [record]
            else:
                f.restype, f.argtypes = C.c_int, [record, _vp]
        _declared = L
    return L


def call(name, record, stream=None):
    """name(record, stream) of include/ff_ops.h; raises FFSimError"""
    code = getattr(lib(), name)(C.byref(record), stream)
    if code != binding.FF_OK:
        raise binding.FFSimError(code, name)


def workspace_bytes(name, record):
    return getattr(lib(), name + "_workspace_bytes")(C.byref(record))


# ---- torch tensors ---------------------------------------------------------------------

def _torch():
    import torch
    return torch


def _dtype(t, what, allowed=("float16", "bfloat16")):
    torch = _torch()
    for name, code in (("float32", FF_F32), ("float16", FF_F16), ("bfloat16", FF_BF16)):
        if t.dtype == getattr(torch, name) and name in allowed:
            return code
    raise ValueError(f"{what} is {t.dtype}; one of {', '.join(allowed)} is wanted")


def _check(t, what, shape, dtype, device):
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what} has shape {tuple(t.shape)}, {tuple(shape)} is wanted")
    if t.dtype != dtype:
        raise ValueError(f"{what} is {t.dtype}, {dtype} is wanted")
    if t.device != device:
        raise ValueError(f"{what} is on {t.device}, {device} is wanted")


def _on_gpu(t, what):
    if t.device.type != "cuda":
        raise ValueError(f"{what} is on {t.device}: the operators have no CPU path")


def _rows(t):
    """a matrix whose rows' elements lie side by side, as a record; `t` must outlive the launch"""
    return ff_rows_t(t.data_ptr(), t.stride(0))


def _dense_rows(t):
    return t if t is None or t.stride(1) == 1 or t.shape[1] <= 1 else t.contiguous()


def _vector(t):
    return None if t is None else t.contiguous()


def _ptr(t):
    return None if t is None else t.data_ptr()


def _launch(name, record, device):
    torch = _torch()
    with torch.cuda.device(device):
        ws = None
        if name + "_workspace_bytes" in EXPORTS:
            n = workspace_bytes(name, record)
            if n:
                ws = torch.empty(n, dtype=torch.uint8, device=device)
                record.workspace, record.workspace_bytes = ws.data_ptr(), n
        call(name, record, torch.cuda.current_stream(device).cuda_stream)


def layernorm_fwd(x, weight, bias=None, *, residual=None, eps=1e-5):
    """(y, h, mean, rstd) of rows x [rows, cols] (float32, float16 or bfloat16): h = x + residual (x itself without one),
    y = (h - mean) * rstd * weight + bias.  mean and rstd [rows] are float32."""
    torch = _torch()
    if x.dim() != 2:
        raise ValueError("x is a matrix [rows, cols]")
    dtype = _dtype(x, "x", ("float32", "float16", "bfloat16"))
    _on_gpu(x, "x")
    R, Cn = x.shape
    _check(weight, "weight", (Cn,), x.dtype, x.device)
    if bias is not None:
        _check(bias, "bias", (Cn,), x.dtype, x.device)
    if residual is not None:
        _check(residual, "residual", (R, Cn), x.dtype, x.device)
    xs, res, weight, bias = _dense_rows(x), _dense_rows(residual), _vector(weight), _vector(bias)
    y = torch.empty(R, Cn, dtype=x.dtype, device=x.device)
    h = x if residual is None else torch.empty_like(y)
    mean, rstd = (torch.empty(R, dtype=torch.float32, device=x.device) for _ in range(2))
    none = ff_rows_t(None, 0)
    rec = ff_layernorm_fwd_t(dtype, Cn, R, eps, _rows(xs), none if res is None else _rows(res), none if res is None else _rows(h), _rows(y),
                             _ptr(weight), _ptr(bias), _ptr(mean), _ptr(rstd))
    _launch("ff_op_layernorm_fwd", rec, x.device)
    return y, h, mean, rstd


def layernorm_bwd(dy, h, weight, mean, rstd, *, dh=None):
    """(dx, dweight, dbias) from what layernorm_fwd returned; dh: the gradient that reaches h past the norm.  dx is the
    gradient of x and of residual alike."""
    torch = _torch()
    if h.dim() != 2:
        raise ValueError("h is a matrix [rows, cols]")
    dtype = _dtype(h, "h", ("float32", "float16", "bfloat16"))
    _on_gpu(h, "h")
    R, Cn = h.shape
    _check(dy, "dy", (R, Cn), h.dtype, h.device)
    _check(weight, "weight", (Cn,), h.dtype, h.device)
    _check(mean, "mean", (R,), torch.float32, h.device)
    _check(rstd, "rstd", (R,), torch.float32, h.device)
    if dh is not None:
        _check(dh, "dh", (R, Cn), h.dtype, h.device)
    dy, hs, dh, weight, mean, rstd = _dense_rows(dy), _dense_rows(h), _dense_rows(dh), _vector(weight), _vector(mean), _vector(rstd)
    dx = torch.empty(R, Cn, dtype=h.dtype, device=h.device)
    dw, db = (torch.empty(Cn, dtype=h.dtype, device=h.device) for _ in range(2))
    rec = ff_layernorm_bwd_t(dtype, Cn, R, _rows(dy), _rows(hs), ff_rows_t(None, 0) if dh is None else _rows(dh), _rows(dx),
                             _ptr(weight), _ptr(mean), _ptr(rstd), _ptr(dw), _ptr(db))
    _launch("ff_op_layernorm_bwd", rec, h.device)
    return dx, dw, db


def _heads(t):
    return ff_heads_t(t.data_ptr(), t.stride(0), t.stride(1), t.stride(2))


def _dense_heads(t):
    """the tensor itself where the kernels can read it (elements of a head side by side, 16-byte steps), else a copy"""
    fits = t.stride(3) == 1 and all(s % 8 == 0 for s in t.stride()[:3]) and t.data_ptr() % 16 == 0
    return t if fits or t.numel() == 0 else t.clone(memory_format=_torch().contiguous_format)


def _attention_args(q, k, v, causal, q_lengths, kv_lengths, scale):
    torch = _torch()
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q and k are [batch, heads, positions, elements]")
    dtype = _dtype(q, "q")
    _on_gpu(q, "q")
    B, H, Sq, D = q.shape
    K, Sk = k.shape[1], k.shape[2]
    _check(k, "k", (B, K, Sk, D), q.dtype, q.device)
    _check(v, "v", (B, K, Sk, D), q.dtype, q.device)
    if K == 0 or H == 0 or H % K:
        raise ValueError(f"{H} query heads do not share {K} key heads evenly")
    if D == 0 or D % 8 or D > 128:
        raise ValueError(f"a head has {D} elements; a multiple of 8 up to 128 is wanted")
    for t, what in ((q_lengths, "q_lengths"), (kv_lengths, "kv_lengths")):
        if t is not None:
            _check(t, what, (B,), torch.int32, q.device)
    scale = 1 / math.sqrt(D) if scale is None else float(scale)
    if not (scale > 0 and math.isfinite(scale)):
        raise ValueError("scale is a positive number")
    return (dtype, B, H, K, Sq, Sk, D, 1 if causal else 0, scale), _vector(q_lengths), _vector(kv_lengths)


def _like_heads(t):
    """an output in the memory order of `t`, heads or positions outside"""
    torch = _torch()
    B, H, S, D = t.shape
    if t.stride(1) < t.stride(2):
        return torch.empty(B, S, H, D, dtype=t.dtype, device=t.device).transpose(1, 2)
    return torch.empty(B, H, S, D, dtype=t.dtype, device=t.device)


def attention_fwd(q, k, v, *, causal=False, q_lengths=None, kv_lengths=None, scale=None):
    """(o, lse): o [batch, heads, q_len, dim] = softmax(scale q k^T) v over the keys that a query sees, lse [batch, heads, q_len]
    float32.  q [batch, heads, q_len, dim], k and v [batch, kv_heads, kv_len, dim], float16 or bfloat16, any strides
    (a copy is made where elements of a head do not lie side by side or strides are no multiples of 8).  q_lengths, kv_lengths:
    int32 [batch].  With causal the last query sees all keys and those before it one fewer each.  A query that sees no key has
    o = 0 and lse = -inf.  scale: 1 / sqrt(dim) if not given."""
    torch = _torch()
    sizes, q_lengths, kv_lengths = _attention_args(q, k, v, causal, q_lengths, kv_lengths, scale)
    o = _like_heads(q)
    lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device)
    q, k, v = _dense_heads(q), _dense_heads(k), _dense_heads(v)
    rec = ff_attention_fwd_t(*sizes, _heads(q), _heads(k), _heads(v), _heads(o), _ptr(lse), _ptr(q_lengths), _ptr(kv_lengths))
    _launch("ff_op_attention_fwd", rec, q.device)
    return o, lse


def attention_bwd(dout, q, k, v, o, lse, *, causal=False, q_lengths=None, kv_lengths=None, scale=None):
    """(dq, dk, dv) from the gradient of o and what attention_fwd returned for the same arguments"""
    torch = _torch()
    sizes, q_lengths, kv_lengths = _attention_args(q, k, v, causal, q_lengths, kv_lengths, scale)
    _check(dout, "dout", q.shape, q.dtype, q.device)
    _check(o, "o", q.shape, q.dtype, q.device)
    _check(lse, "lse", q.shape[:3], torch.float32, q.device)
    dq, dk, dv = _like_heads(q), _like_heads(k), _like_heads(v)
    dout, q, k, v, o, lse = _dense_heads(dout), _dense_heads(q), _dense_heads(k), _dense_heads(v), _dense_heads(o), lse.contiguous()
    rec = ff_attention_bwd_t(*sizes, *(_heads(t) for t in (dout, q, k, v, o, dq, dk, dv)), _ptr(lse), _ptr(q_lengths), _ptr(kv_lengths))
    _launch("ff_op_attention_bwd", rec, q.device)
    return dq, dk, dv


def _vocab_args(x, weight, targets, ignore_index, first_word):
    torch = _torch()
    if x.dim() != 2 or weight.dim() != 2:
        raise ValueError("x is a matrix [rows, dim], weight [vocab, dim]")
    dtype = _dtype(x, "x")
    _on_gpu(x, "x")
    N, D = x.shape
    _check(weight, "weight", (weight.shape[0], D), x.dtype, x.device)
    _check(targets, "targets", (N,), torch.int32, x.device)
    if weight.shape[0] == 0 or D == 0:
        raise ValueError("an empty vocabulary or vectors without elements")
    for n, what in ((ignore_index, "ignore_index"), (first_word, "first_word")):
        if not -2 ** 31 <= n < 2 ** 31:
            raise ValueError(f"{what} does not fit 32 bits")
    return (dtype, N, weight.shape[0], D, ignore_index, first_word), _dense_rows(x), _dense_rows(weight), _vector(targets)


def vocab_loss_fwd(x, weight, targets, *, ignore_index=-100, first_word=None):
    """(loss, lse, target_logit), float32 [rows], of rows x [rows, dim] against the vocabulary weight [vocab, dim] (float16 or
    bfloat16): lse = log sum_v exp(<x, w_v>), target_logit = <x, w_target>, loss = lse - target_logit.  targets: int32 [rows];
    a row with ignore_index has loss 0, a target that is no word a NaN.  The logits are not kept.

    With first_word, weight is a shard: words first_word .. first_word + vocab - 1 of a larger vocabulary that targets count in.
    loss is then None; target_logit is 0 where the target is another shard's.  log sum exp of the shards' lse, and the sum of
    their target_logit, make the loss, and vocab_loss_bwd of a shard takes the joined lse."""
    torch = _torch()
    sizes, x, weight, targets = _vocab_args(x, weight, targets, ignore_index, first_word or 0)
    loss = torch.empty(x.shape[0], dtype=torch.float32, device=x.device) if first_word is None else None
    lse, logit = (torch.empty(x.shape[0], dtype=torch.float32, device=x.device) for _ in range(2))
    rec = ff_vocab_loss_fwd_t(*sizes, _rows(x), _rows(weight), _ptr(targets), _ptr(loss), _ptr(lse), _ptr(logit))
    _launch("ff_op_vocab_loss_fwd", rec, x.device)
    return loss, lse, logit


def vocab_loss_bwd(dloss, x, weight, targets, lse, *, ignore_index=-100, first_word=None):
    """(dx, dweight) from the gradient of each row's loss (float32 [rows]) and the forward pass' lse; for a shard of the vocabulary, dx is its share of the sum"""
    torch = _torch()
    sizes, xs, ws, targets = _vocab_args(x, weight, targets, ignore_index, first_word or 0)
    _check(dloss, "dloss", targets.shape, torch.float32, x.device)
    _check(lse, "lse", targets.shape, torch.float32, x.device)
    dloss, lse = dloss.contiguous(), lse.contiguous()
    dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    dw = torch.empty(weight.shape, dtype=x.dtype, device=x.device)
    rec = ff_vocab_loss_bwd_t(*sizes, _rows(xs), _rows(ws), _rows(dx), _rows(dw), _ptr(targets), _ptr(dloss), _ptr(lse))
    _launch("ff_op_vocab_loss_bwd", rec, x.device)
    return dx, dw
