"""Training operators of language models on the GPU: layer norm, attention and the loss over a vocabulary, forward and
backward.  Thin ctypes binding of the C boundary in include/ff_ops.h (same names, argument marshalling only) and, on
top of it, functions that take torch tensors: torch is used for device memory and streams, nothing else, and there is
no CPU fallback.

The functions check what they are given (ValueError), allocate their outputs and workspace with torch on the tensors'
device and put the kernels on its current stream; they do not wait.  Captured into a HIP graph, they use the graph's
memory.  What a call refuses on the library's side raises binding.FFSimError.

autograd does not see them: gradients are the ..._bwd functions' outputs.  So tensors that require gradients are refused
where they would be recorded; under torch.no_grad() they are taken.
"""
from __future__ import annotations

import ctypes as C
import functools
import math
import struct

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
    """the library with the operators' calls declared: a record by its address, or as the bytes that it consists of"""
    global _declared
    L = binding.lib()
    if _declared is not L:
        for name in EXPORTS:
            f = getattr(L, name)
            if name.endswith("_workspace_bytes"):
                f.restype, f.argtypes = C.c_size_t, [_vp]
            else:
                f.restype, f.argtypes = C.c_int, [_vp, _vp]
        _declared = L
    return L


def call(name, record, stream=None):
    """name(record, stream) of include/ff_ops.h; raises FFSimError"""
    code = getattr(lib(), name)(C.byref(record), stream)
    if code != binding.FF_OK:
        raise binding.FFSimError(code, name)


def workspace_bytes(name, record):
    return getattr(lib(), name + "_workspace_bytes")(C.byref(record))


_CODES = {C.c_uint32: "I", C.c_int32: "i", C.c_uint64: "Q", C.c_int64: "q", C.c_float: "f", C.c_void_p: "P", C.c_size_t: "N"}


def _format(record):
    """the record as a format of struct.pack: its fields in order, records in it field by field"""
    fmt, at = "", 0
    for name, kind in record._fields_:
        place = getattr(record, name).offset
        fmt += "%dx" % (place - at) if place > at else ""
        fmt += _format(kind)[1:] if issubclass(kind, C.Structure) else _CODES[kind]
        at = place + C.sizeof(kind)
    return "@" + fmt + ("%dx" % (C.sizeof(record) - at) if C.sizeof(record) > at else "")


@functools.lru_cache(maxsize=None)
def _call_of(name, L):
    """(pack, function, workspace function or None) of a call; packing a record's values takes a tenth of the time that filling a Structure does"""
    packer = struct.Struct(_format(_RECORDS[name]))
    if packer.size != C.sizeof(_RECORDS[name]):
        raise RuntimeError(f"{name}: the packed record has {packer.size} bytes")
    more = name + "_workspace_bytes"
    return packer.pack, getattr(L, name), getattr(L, more) if more in EXPORTS else None


# ---- torch tensors ---------------------------------------------------------------------

_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


_DTYPES = {}


def _dtype(t, what, f32=False):
    if not _DTYPES:
        torch = _torch()
        _DTYPES.update({torch.float32: FF_F32, torch.float16: FF_F16, torch.bfloat16: FF_BF16})
    code = _DTYPES.get(t.dtype, -1)
    if code < (0 if f32 else 1):
        raise ValueError(f"{what} is {t.dtype}; float16, bfloat16{' or float32' if f32 else ''} is wanted")
    if not t.is_cuda:
        raise ValueError(f"{what} is on {t.device}: the operators have no CPU path")
    return code


def _check(t, what, shape, dtype, device):
    if t.shape != shape:
        raise ValueError(f"{what} has shape {tuple(t.shape)}, {tuple(shape)} is wanted")
    if t.dtype is not dtype:
        raise ValueError(f"{what} is {t.dtype}, {dtype} is wanted")
    if t.device != device:
        raise ValueError(f"{what} is on {t.device}, {device} is wanted")


def _not_recorded(*ts):
    for t in ts:
        if t is not None and t.requires_grad and _torch().is_grad_enabled():
            raise ValueError("a tensor requires gradients, which autograd would lose here: call this under torch.no_grad(), and the _bwd function for the gradients")


def _dense_rows(t):
    """the matrix itself where its rows' elements lie side by side, else a copy"""
    return t if t is None or t.stride(1) == 1 or t.shape[1] <= 1 else t.contiguous()


def _vector(t):
    return t if t is None or t.is_contiguous() else t.contiguous()


def _ptr(t):
    return 0 if t is None else t.data_ptr()


def _launch(name, device, *values):
    """packs the record, with a workspace if there is to be one, and calls `name` on the device's current stream"""
    torch = _torch()
    if device.index != torch.cuda.current_device():
        with torch.cuda.device(device):
            return _launch(name, device, *values)
    pack, function, workspace = _call_of(name, lib())
    if workspace is None:
        record = pack(*values)
    else:
        record = pack(*values, 0, 0)
        n = workspace(record)
        if n:
            ws = torch.empty(n, dtype=torch.uint8, device=device)      # its memory is reused in the order of the stream
            record = pack(*values, ws.data_ptr(), n)
    code = function(record, _stream(torch, device))
    if code != binding.FF_OK:
        raise binding.FFSimError(code, name)


def _stream(torch, device):
    """the device's current stream; the object that torch.cuda.current_stream makes of it takes longer than all else here"""
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(device.index) if raw else torch.cuda.current_stream(device).cuda_stream


def layernorm_fwd(x, weight, bias=None, *, residual=None, eps=1e-5):
    """(y, h, mean, rstd) of rows x [rows, cols] (float32, float16 or bfloat16): h = x + residual (x itself without one),
    y = (h - mean) * rstd * weight + bias.  mean and rstd [rows] are float32."""
    torch = _torch()
    _not_recorded(x, weight, bias, residual)
    if x.dim() != 2:
        raise ValueError("x is a matrix [rows, cols]")
    dtype, device = _dtype(x, "x", True), x.device
    R, Cn = x.shape
    _check(weight, "weight", (Cn,), x.dtype, device)
    if bias is not None:
        _check(bias, "bias", (Cn,), x.dtype, device)
    if residual is not None:
        _check(residual, "residual", (R, Cn), x.dtype, device)
    xs, res, weight, bias = _dense_rows(x), _dense_rows(residual), _vector(weight), _vector(bias)
    y = torch.empty((R, Cn), dtype=x.dtype, device=device)
    h = x if residual is None else torch.empty_like(y)
    mean, rstd = torch.empty((2, R), dtype=torch.float32, device=device).unbind()
    _launch("ff_op_layernorm_fwd", device, dtype, Cn, R, eps, xs.data_ptr(), xs.stride(0), _ptr(res), 0 if res is None else res.stride(0),
            0 if res is None else h.data_ptr(), Cn, y.data_ptr(), Cn, weight.data_ptr(), _ptr(bias), mean.data_ptr(), rstd.data_ptr())
    return y, h, mean, rstd


def layernorm_bwd(dy, h, weight, mean, rstd, *, dh=None):
    """(dx, dweight, dbias) from what layernorm_fwd returned; dh: the gradient that reaches h past the norm.  dx is the
    gradient of x and of residual alike."""
    torch = _torch()
    _not_recorded(dy, h, weight, mean, rstd, dh)
    if h.dim() != 2:
        raise ValueError("h is a matrix [rows, cols]")
    dtype, device = _dtype(h, "h", True), h.device
    R, Cn = h.shape
    _check(dy, "dy", (R, Cn), h.dtype, device)
    _check(weight, "weight", (Cn,), h.dtype, device)
    _check(mean, "mean", (R,), torch.float32, device)
    _check(rstd, "rstd", (R,), torch.float32, device)
    if dh is not None:
        _check(dh, "dh", (R, Cn), h.dtype, device)
    dy, hs, dh, weight, mean, rstd = _dense_rows(dy), _dense_rows(h), _dense_rows(dh), _vector(weight), _vector(mean), _vector(rstd)
    dx = torch.empty((R, Cn), dtype=h.dtype, device=device)
    dw, db = torch.empty((2, Cn), dtype=h.dtype, device=device).unbind()
    _launch("ff_op_layernorm_bwd", device, dtype, Cn, R, dy.data_ptr(), dy.stride(0), hs.data_ptr(), hs.stride(0), _ptr(dh), 0 if dh is None else dh.stride(0),
            dx.data_ptr(), Cn, weight.data_ptr(), mean.data_ptr(), rstd.data_ptr(), dw.data_ptr(), db.data_ptr())
    return dx, dw, db


def _heads(*ts):
    """addresses and strides of batch, head and position, one tensor after another"""
    return [x for t in ts for x in (t.data_ptr(), *t.stride()[:3])]


def _dense_heads(t):
    """the tensor itself where the kernels can read it (elements of a head side by side, 16-byte steps), else a copy"""
    b, h, p, e = t.stride()
    fits = e == 1 and not (b | h | p) & 7 and t.data_ptr() % 16 == 0
    return t if fits or t.numel() == 0 else t.clone(memory_format=_torch().contiguous_format)


def _attention_args(q, k, v, causal, q_lengths, kv_lengths, scale):
    torch = _torch()
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q and k are [batch, heads, positions, elements]")
    dtype = _dtype(q, "q")
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
    _not_recorded(q, k, v)
    sizes, q_lengths, kv_lengths = _attention_args(q, k, v, causal, q_lengths, kv_lengths, scale)
    o = _like_heads(q)
    lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device)
    q, k, v = _dense_heads(q), _dense_heads(k), _dense_heads(v)
    _launch("ff_op_attention_fwd", q.device, *sizes, *_heads(q, k, v, o), lse.data_ptr(), _ptr(q_lengths), _ptr(kv_lengths))
    return o, lse


def attention_bwd(dout, q, k, v, o, lse, *, causal=False, q_lengths=None, kv_lengths=None, scale=None):
    """(dq, dk, dv) from the gradient of o and what attention_fwd returned for the same arguments.  Where k and v are a piece of the
    keys, o and lse those of all pieces: this piece's dk and dv, and its part of dq."""
    torch = _torch()
    _not_recorded(dout, q, k, v, o, lse)
    sizes, q_lengths, kv_lengths = _attention_args(q, k, v, causal, q_lengths, kv_lengths, scale)
    _check(dout, "dout", q.shape, q.dtype, q.device)
    _check(o, "o", q.shape, q.dtype, q.device)
    _check(lse, "lse", q.shape[:3], torch.float32, q.device)
    dq, dk, dv = _like_heads(q), _like_heads(k), _like_heads(v)
    dout, q, k, v, o, lse = _dense_heads(dout), _dense_heads(q), _dense_heads(k), _dense_heads(v), _dense_heads(o), lse.contiguous()
    _launch("ff_op_attention_bwd", q.device, *sizes, *_heads(dout, q, k, v, o, dq, dk, dv), lse.data_ptr(), _ptr(q_lengths), _ptr(kv_lengths))
    return dq, dk, dv


def _vocab_args(x, weight, targets, ignore_index, first_word):
    torch = _torch()
    if x.dim() != 2 or weight.dim() != 2:
        raise ValueError("x is a matrix [rows, dim], weight [vocab, dim]")
    dtype = _dtype(x, "x")
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
    _not_recorded(x, weight)
    sizes, x, weight, targets = _vocab_args(x, weight, targets, ignore_index, first_word or 0)
    loss, lse, logit = torch.empty((3, x.shape[0]), dtype=torch.float32, device=x.device).unbind()
    if first_word is not None:
        loss = None
    _launch("ff_op_vocab_loss_fwd", x.device, *sizes, x.data_ptr(), x.stride(0), weight.data_ptr(), weight.stride(0), targets.data_ptr(), _ptr(loss), lse.data_ptr(), logit.data_ptr())
    return loss, lse, logit


def vocab_loss_bwd(dloss, x, weight, targets, lse, *, ignore_index=-100, first_word=None):
    """(dx, dweight) from the gradient of each row's loss (float32 [rows]) and the forward pass' lse; for a shard of the vocabulary, dx is its share of the sum.
    Rows with ignore_index cost no products: their dx is 0, and what x, dloss and lse hold there is not used."""
    torch = _torch()
    _not_recorded(dloss, x, weight, lse)
    sizes, xs, ws, targets = _vocab_args(x, weight, targets, ignore_index, first_word or 0)
    _check(dloss, "dloss", targets.shape, torch.float32, x.device)
    _check(lse, "lse", targets.shape, torch.float32, x.device)
    dloss, lse = _vector(dloss), _vector(lse)
    D = x.shape[1]
    dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    dw = torch.empty(weight.shape, dtype=x.dtype, device=x.device)
    _launch("ff_op_vocab_loss_bwd", x.device, *sizes, xs.data_ptr(), xs.stride(0), ws.data_ptr(), ws.stride(0), dx.data_ptr(), D, dw.data_ptr(), D,
            targets.data_ptr(), dloss.data_ptr(), lse.data_ptr())
    return dx, dw
