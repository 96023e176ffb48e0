"""Operators of language models on the GPU: for training, layer norm, attention and the loss over a vocabulary, forward and
backward; for answering, a paged cache of keys and values, attention over it and the choice of the next token.  Thin ctypes binding of the C boundary in include/ff_ops.h (same names, argument marshalling only) and, on
top of it, functions that take torch tensors: torch is used for device memory and streams, nothing else, and there is
no CPU fallback.

The functions check what they are given (ValueError), allocate their outputs and workspace with torch on the tensors'
device and put the kernels on its current stream; they do not wait.  Captured into a HIP graph, they use the graph's
memory.  What a call refuses on the library's side raises binding.FFSimError.

autograd does not see them: gradients are the ..._bwd functions' outputs.  So tensors that require gradients are refused
where they would be recorded; under torch.no_grad() they are taken.  Dual tensors of forward mode are refused.
"""
from __future__ import annotations

import ctypes as C
import functools
import math
import struct

from . import binding

FF_F32, FF_F16, FF_BF16 = 0, 1, 2
FF_HELD_SAME, FF_HELD_E4M3, FF_HELD_E2M1 = 0, 1, 2

EXPORTS = ["ff_op_layernorm_fwd", "ff_op_layernorm_bwd_workspace_bytes", "ff_op_layernorm_bwd",
           "ff_op_attention_fwd_workspace_bytes", "ff_op_attention_fwd", "ff_op_attention_bwd_workspace_bytes", "ff_op_attention_bwd",
           "ff_op_vocab_loss_fwd_workspace_bytes", "ff_op_vocab_loss_fwd", "ff_op_vocab_loss_bwd_workspace_bytes", "ff_op_vocab_loss_bwd",
           "ff_op_cache_write", "ff_op_cache_read", "ff_op_attention_paged_fwd_workspace_bytes", "ff_op_attention_paged_fwd", "ff_op_sample"]


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


class ff_cache_t(C.Structure):
    _fields_ = [(n, _vp) for n in ("k", "v", "k_scale", "v_scale", "table")] + \
        [(n, C.c_int64) for n in ("k_stride", "v_stride", "k_scale_stride", "v_scale_stride", "table_stride")] + [(n, _u32) for n in ("pages", "page", "table_pages", "held")]


class ff_cache_write_t(C.Structure):
    _fields_ = [(n, _u32) for n in ("dtype", "batch", "kv_heads", "head_dim", "new_len")] + [("k", ff_heads_t), ("v", ff_heads_t), ("cache", ff_cache_t), ("start", _vp), ("lengths", _vp)]


class ff_cache_read_t(C.Structure):
    _fields_ = [(n, _u32) for n in ("dtype", "batch", "kv_heads", "head_dim", "kv_len")] + [("k", ff_heads_t), ("v", ff_heads_t), ("cache", ff_cache_t), ("lengths", _vp)]


class ff_attention_paged_fwd_t(C.Structure):
    _fields_ = [(n, _u32) for n in ("dtype", "batch", "heads", "kv_heads", "q_len", "head_dim", "causal")] + [("scale", C.c_float), ("q", ff_heads_t), ("o", ff_heads_t), ("cache", ff_cache_t)] + \
        [(n, _vp) for n in ("lse", "q_lengths", "kv_lengths")] + _WS


class ff_sample_t(C.Structure):
    _fields_ = [(n, _u32) for n in ("dtype", "rows", "vocab")] + [("logits", ff_rows_t)] + [(n, _vp) for n in ("u", "temperatures", "top_ps", "min_ps", "top_ks")] + \
        [(n, C.c_float) for n in ("temperature", "top_p", "min_p")] + [("top_k", C.c_int32), ("words", _vp), ("logprob", _vp)]


_RECORDS = {"ff_op_layernorm_fwd": ff_layernorm_fwd_t, "ff_op_layernorm_bwd": ff_layernorm_bwd_t, "ff_op_attention_fwd": ff_attention_fwd_t,
            "ff_op_attention_bwd": ff_attention_bwd_t, "ff_op_vocab_loss_fwd": ff_vocab_loss_fwd_t, "ff_op_vocab_loss_bwd": ff_vocab_loss_bwd_t,
            "ff_op_cache_write": ff_cache_write_t, "ff_op_cache_read": ff_cache_read_t, "ff_op_attention_paged_fwd": ff_attention_paged_fwd_t, "ff_op_sample": ff_sample_t}
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
    torch = _torch()
    for t in ts:
        if t is not None and t.requires_grad and torch.is_grad_enabled():
            raise ValueError("a tensor requires gradients, which autograd would lose here: call this under torch.no_grad(), and the _bwd function for the gradients")
    forward = torch.autograd.forward_ad
    if getattr(forward, "_current_level", 0) >= 0:      # (outside of all levels no tensor has a tangent)
        for t in ts:
            if t is not None and forward.unpack_dual(t).tangent is not None:
                raise ValueError("a tensor has a tangent, which would be lost here: the operators have no forward mode")


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


def _page_stride(shape, stride, size, what):
    """bytes from page to page; the rest of a page lies side by side"""
    n, h, p, e = shape
    _, sh, sp, se = stride
    if not (e == 1 or se == 1) or not (p == 1 or sp == e) or not (h == 1 or sh == p * e):
        raise ValueError(f"{what}: the elements of a page lie side by side; only pages may have room between them")
    n = stride[0] * size if n > 1 else h * p * e * size
    if n % 16:
        raise ValueError(f"{what}: pages begin at multiples of 16 bytes")
    return n


@functools.lru_cache(maxsize=256)
def _cache_layout(dtype, k, v, table, k_scales, v_scales):
    """(kv_heads, head_dim, strides of the cache's record, its other sizes) for tensors of `dtype`, from (shape, stride, type) of each"""
    torch = _torch()
    shape, stride, kind = k
    if len(shape) != 4 or len(table[0]) != 2:
        raise ValueError("k_pages are [pages, kv_heads, page, elements], the table [batch, entries]")
    N, K, P, E = shape
    for t, what, want, to in ((v, "v_pages", shape, kind), (table, "table", table[0], torch.int32)):
        if t[0] != want or t[2] is not to:
            raise ValueError(f"{what} has shape {tuple(t[0])} and is {t[2]}, {tuple(want)} and {to} are wanted")
    if table[0][1] > 1 and table[1][1] != 1:
        raise ValueError("a row of the table lies side by side")
    if kind is dtype:
        held, D, blocks, unit, size = FF_HELD_SAME, E, 0, 8, 2
    elif kind is torch.float8_e4m3fn:
        held, D, blocks, unit, size = FF_HELD_E4M3, E, 1, 16, 1
    elif kind is torch.uint8:
        held, D, blocks, unit, size = FF_HELD_E2M1, 2 * E, E // 16, 32, 1
    else:
        raise ValueError(f"k_pages is {kind}; {dtype}, float8_e4m3fn or uint8 (two 4-bit floats) is wanted")
    if N == 0 or K == 0:
        raise ValueError("a cache without pages or heads")
    if D == 0 or D % unit or D > 128:
        raise ValueError(f"a head has {D} elements; a multiple of {unit} up to 128 is wanted for {kind}")
    if P < 16 or P & (P - 1) or P > 32768:
        raise ValueError(f"a page has {P} positions; a power of two from 16 to 32768 is wanted")
    scales = [0, 0]
    for i, (t, what) in enumerate(((k_scales, "k_scales"), (v_scales, "v_scales"))):
        if held == FF_HELD_SAME:
            if t is not None:
                raise ValueError(f"{dtype} is held without scales")
            continue
        if t is None:
            raise ValueError(f"{what} are missing: {kind} is held with scales")
        if t[0] != (N, K, blocks, P) or t[2] is not torch.uint8:
            raise ValueError(f"{what} has shape {tuple(t[0])} and is {t[2]}, {(N, K, blocks, P)} and uint8 are wanted")
        sn, sh, sb, sp = t[1]
        if sp != 1 or not (blocks == 1 or sb == P) or not (K == 1 or sh == blocks * P) or (N > 1 and sn % 4):
            raise ValueError(f"{what}: the scales of a page lie side by side; only pages may have room between them, in steps of 4")
        scales[i] = sn if N > 1 else K * blocks * P
    return K, D, (_page_stride(shape, stride, size, "k_pages"), _page_stride(v[0], v[1], size, "v_pages"), *scales, table[1][0]), (N, P, table[0][1], held)


def _cache_args(k_pages, v_pages, table, k_scales, v_scales, dtype):
    """(kv_heads, head_dim, values of the cache's record) of a cache for tensors of `dtype`"""
    if not k_pages.is_cuda:
        raise ValueError(f"k_pages is on {k_pages.device}: the operators have no CPU path")
    few = (k_scales.shape, k_scales.stride(), k_scales.dtype) if k_scales is not None else None, (v_scales.shape, v_scales.stride(), v_scales.dtype) if v_scales is not None else None
    K, D, strides, sizes = _cache_layout(dtype, (k_pages.shape, k_pages.stride(), k_pages.dtype), (v_pages.shape, v_pages.stride(), v_pages.dtype), (table.shape, table.stride(), table.dtype), *few)
    device, at = k_pages.device, (k_pages.data_ptr(), v_pages.data_ptr(), _ptr(k_scales), _ptr(v_scales), table.data_ptr())
    if v_pages.device != device or table.device != device or (k_scales is not None and (k_scales.device != device or v_scales.device != device)):
        raise ValueError(f"the parts of a cache are on one device, {device}")
    if (at[0] | at[1]) % 16 or (at[2] | at[3]) % 4:
        raise ValueError("pages begin at multiples of 16 bytes, their scales of 4")
    return K, D, (*at, *strides, *sizes)


def cache_write(k, v, k_pages, v_pages, table, start, *, lengths=None, k_scales=None, v_scales=None):
    """Writes new keys and values k, v [batch, kv_heads, new, dim] (float16 or bfloat16) into a paged cache: position i of sequence b becomes its
    position start[b] + i, for the first lengths[b] of them (int32 [batch] both; all of them without lengths).

    The cache: k_pages, v_pages [pages, kv_heads, page, dim]; position i of sequence b is in page table[b, i // page] (int32 [batch, entries]) at place
    i % page.  Pages hold the tensors' type, or float8_e4m3fn with k_scales, v_scales (uint8 [pages, kv_heads, 1, page]: a power of two for
    each row of dim), or uint8 [pages, kv_heads, page, dim / 2], 4-bit floats, two a byte, with scales [pages, kv_heads, dim / 32, page] for each 32 elements.
    A scale s stands for 2^(s - 127); 255: the block held a value that was not finite and is read as NaN.  Positions outside the table, and entries that are no page, are not
    written.  Sequences may share pages, but no two positions of a call the same place."""
    torch = _torch()
    _not_recorded(k, v, k_pages, v_pages)
    if k.dim() != 4:
        raise ValueError("k is [batch, kv_heads, positions, elements]")
    dtype, device = _dtype(k, "k"), k.device
    K, D, cache = _cache_args(k_pages, v_pages, table, k_scales, v_scales, k.dtype)
    _check(k, "k", (table.shape[0], K, k.shape[2], D), k.dtype, k_pages.device)
    _check(v, "v", k.shape, k.dtype, device)
    B = k.shape[0]
    _check(start, "start", (B,), torch.int32, device)
    if lengths is not None:
        _check(lengths, "lengths", (B,), torch.int32, device)
    n, start, lengths = k.shape[2], _vector(start), _vector(lengths)
    k, v = _dense_heads(k), _dense_heads(v)
    _launch("ff_op_cache_write", device, dtype, B, K, D, n, *_heads(k, v), *cache, start.data_ptr(), _ptr(lengths))


def cache_read(k_pages, v_pages, table, lengths, *, kv_len=None, dtype=None, k_scales=None, v_scales=None):
    """(k, v) [batch, kv_heads, kv_len, dim] of the first lengths[b] positions (int32 [batch]) of each sequence of a paged cache (see cache_write), zeros behind them.
    kv_len: the positions of the table if not given; dtype: float16 or bfloat16, the pages' own if they hold one of these.  A position whose entry is no page gives NaN."""
    torch = _torch()
    _not_recorded(k_pages, v_pages)
    if dtype is None and k_pages.dtype in (torch.float16, torch.bfloat16):
        dtype = k_pages.dtype
    if dtype not in (torch.float16, torch.bfloat16):
        raise ValueError("dtype is float16 or bfloat16")
    K, D, cache = _cache_args(k_pages, v_pages, table, k_scales, v_scales, dtype)
    B, device = table.shape[0], k_pages.device
    _check(lengths, "lengths", (B,), torch.int32, device)
    kv_len = table.shape[1] * k_pages.shape[2] if kv_len is None else kv_len
    if kv_len < 0:
        raise ValueError("kv_len is a number of positions")
    lengths = _vector(lengths)
    k, v = k_pages.new_empty((2, B, K, kv_len, D), dtype=dtype).unbind()
    code, most = FF_F16 if dtype is torch.float16 else FF_BF16, max(1, 65535 // K)             # most: sequences of a launch
    if B <= most:
        _launch("ff_op_cache_read", device, code, B, K, D, kv_len, *_heads(k, v), *cache, lengths.data_ptr())
    else:
        for i in range(0, B, most):
            some = slice(i, min(B, i + most))
            cache = _cache_args(k_pages, v_pages, table[some], k_scales, v_scales, dtype)[2]
            _launch("ff_op_cache_read", device, code, some.stop - i, K, D, kv_len, *_heads(k[some], v[some]), *cache, lengths[some].data_ptr())
    return k, v


def attention_paged_fwd(q, k_pages, v_pages, table, kv_lengths, *, causal=False, q_lengths=None, scale=None, k_scales=None, v_scales=None):
    """(o, lse) of new queries q [batch, heads, q_len, dim] (float16 or bfloat16) over the first kv_lengths[b] positions (int32 [batch]) of a paged cache (see cache_write), their own among
    them; otherwise as attention_fwd: with causal the last query sees all positions and those before it one fewer each, q_lengths are int32 [batch], a query that sees nothing has o = 0 and
    lse = -inf.  A query that sees a position whose entry is no page gets NaN.  Value rows that some queries of a sequence see and others do not have to be finite (a block
    held in fewer bits that was not reads back as NaN).  Keys and values are read once for a few queries of each head (16 queries times heads of a key head are worked together, 32 where there are more), so
    long prompts, of more than about 128 queries times heads of a key head, are better read back with cache_read for attention_fwd."""
    torch = _torch()
    _not_recorded(q, k_pages, v_pages)
    if q.dim() != 4:
        raise ValueError("q is [batch, heads, positions, elements]")
    dtype, device = _dtype(q, "q"), q.device
    K, D, cache = _cache_args(k_pages, v_pages, table, k_scales, v_scales, q.dtype)
    B, H, n, _ = q.shape
    _check(q, "q", (table.shape[0], H, n, D), q.dtype, k_pages.device)
    if H == 0 or H % K:
        raise ValueError(f"{H} query heads do not share {K} key heads evenly")
    _check(kv_lengths, "kv_lengths", (B,), torch.int32, device)
    if q_lengths is not None:
        _check(q_lengths, "q_lengths", (B,), torch.int32, device)
    scale = 1 / math.sqrt(D) if scale is None else float(scale)
    if not (scale > 0 and math.isfinite(scale)):
        raise ValueError("scale is a positive number")
    o, lse = torch.empty_like(q), q.new_empty((B, H, n), dtype=torch.float32)
    if o.stride(3) != 1 or o.stride(0) % 8 or o.stride(1) % 8 or o.stride(2) % 8:
        o = _like_heads(q)
    q, q_lengths, kv_lengths = _dense_heads(q), _vector(q_lengths), _vector(kv_lengths)
    _launch("ff_op_attention_paged_fwd", device, dtype, B, H, K, n, D, 1 if causal else 0, scale, *_heads(q, o), *cache, lse.data_ptr(), _ptr(q_lengths), kv_lengths.data_ptr())
    return o, lse


def checked_choice(u, rows, device, *, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(vectors, numbers) of temperature, top_p, min_p and top_k: what sample would be given beside logits of so many rows, refused as there.  For those who have work to do before there are logits."""
    torch = _torch()
    _check(u, "u", (rows,), torch.float32, device)
    numbers, vectors = [], []
    for x, what, to, kind in ((temperature, "temperature", torch.float32, float), (top_p, "top_p", torch.float32, float), (min_p, "min_p", torch.float32, float), (top_k, "top_k", torch.int32, int)):
        if isinstance(x, torch.Tensor):
            _not_recorded(x)
            _check(x, what, (rows,), to, device)
            vectors.append(_vector(x))
            numbers.append(kind())
        else:
            vectors.append(None)
            numbers.append(kind(x))
    if not -2 ** 31 <= numbers[3] < 2 ** 31:
        raise ValueError("top_k does not fit 32 bits")
    for n, what, least in zip(numbers, ("temperature", "top_p", "min_p"), (0.0, -math.inf, -math.inf)):
        if not n >= least or not abs(n) <= 3e38:
            raise ValueError(f"{what} is {n}")
    return vectors, numbers


def sample(logits, u, *, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(words, logprob), int32 and float32 [rows]: a word for each row of logits [rows, vocab] (float32, float16 or bfloat16), chosen by the given random number u[row] in [0, 1) (float32 [rows]).

    Words are taken in the order of their logits, equal ones in the order of their numbers, and weigh exp((z - max z) / temperature), in 64 bits.  The first top_k are
    kept (0: all), of these the shortest beginning that has top_p of their weight, of these the words that weigh at least min_p (the first weighs 1); the word is the first at which the running
    sum exceeds u times the weight of all that are kept.  logprob: the logarithm of its share of that.  At temperature 0 it is the first word, with
    logprob 0.  Each parameter is a number, or a tensor with one for each row (float32, top_k int32).  Rows that hold a NaN or only -inf, or
    whose temperature is below 0 or another parameter no number, give word -1 and logprob NaN."""
    torch = _torch()
    _not_recorded(logits)
    if logits.dim() != 2:
        raise ValueError("logits are a matrix [rows, vocab]")
    dtype, device = _dtype(logits, "logits", True), logits.device
    R, V = logits.shape
    if V == 0:
        raise ValueError("an empty vocabulary")
    vectors, numbers = checked_choice(u, R, device, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)
    logits, u = _dense_rows(logits), _vector(u)
    words, logprob = u.new_empty(R, dtype=torch.int32), u.new_empty(R)
    _launch("ff_op_sample", device, dtype, R, V, logits.data_ptr(), logits.stride(0), u.data_ptr(), *(_ptr(t) for t in vectors), *numbers, words.data_ptr(), logprob.data_ptr())
    return words, logprob
