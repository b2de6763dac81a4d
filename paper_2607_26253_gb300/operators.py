"""Operators on torch CUDA tensors over an 8-bit paged KV cache and over the logits of sampled tokens (include/sara.h).

Calls are a decode step's: their checks are written for speed (attributes compared in place, messages made only for a refusal).
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass

from .sara import SARA_EINVAL, Kv8Cache, SaraError, _check, load

KV8_PAGE, KV8_SCALE = 128, 32   # positions of a cache block, and of a scale

torch = None   # imported by the first call, as the rest of the package does
_types = {}    # torch dtype -> SARA_BF16, SARA_FP16, SARA_FP32
_formats = {}  # torch dtype -> SARA_KV8_*
_int32 = _fp32 = None


def _import_torch():
    global torch, _int32, _fp32
    import torch as t
    _types.update({t.bfloat16: 0, t.float16: 1, t.float32: 2})
    _formats.update({t.float8_e4m3fn: 0, t.int8: 1})
    _int32, _fp32 = t.int32, t.float32
    torch = t


def _refuse(msg):
    raise SaraError(SARA_EINVAL, msg)


def _vector(x, dtype, n, dev, what):
    """Address of a contiguous vector (or None -> NULL) of n elements on GPU dev."""
    if x is None:
        return None
    if x.dtype is not dtype or x.dim() != 1 or x.numel() != n or x.get_device() != dev or (n > 1 and x.stride(0) != 1):
        _refuse(f"{what} must be a contiguous {dtype} tensor of {n} elements on the operands' device")
    return x.data_ptr()


def _matrix(x, dtype, shape, dev, what):
    """Address of a contiguous tensor of a shape (or None -> NULL) on GPU dev."""
    if x is None:
        return None
    if x.dtype is not dtype or x.shape != shape or x.get_device() != dev or not x.is_contiguous():
        _refuse(f"{what} must be a contiguous {dtype} tensor of shape {tuple(shape)} on the operands' device")
    return x.data_ptr()


def _launch(dev, fn, *args):
    """fn(*args, stream) on the current stream of GPU dev."""
    if dev < 0:
        _refuse("operands must be CUDA tensors")
    if dev == torch._C._cuda_getDevice():
        rc = fn(*args, torch._C._cuda_getCurrentRawStream(dev))
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, torch._C._cuda_getCurrentRawStream(dev))
    if rc:
        _check(rc)


def _kv8(codes, scales, table):
    """The Kv8Cache of a cache's tensors, checked, and their GPU."""
    if torch is None:
        _import_torch()
    fmt, dev, shape = _formats.get(codes.dtype), codes.get_device(), codes.shape
    if fmt is None:
        _refuse(f"codes must be float8_e4m3fn or int8, not {codes.dtype}")
    if len(shape) != 5 or shape[1] != 2 or shape[3] != KV8_PAGE or not codes.is_contiguous():
        _refuse("codes must be contiguous, [n_blocks, 2, n_kv_heads, 128, head_dim]")
    nb, _, kvh, _, hd = shape
    at = _matrix(scales, _fp32, (nb, 2, kvh, KV8_PAGE // KV8_SCALE), dev, "scales")
    if table.dtype != _int32 or table.dim() != 2 or table.get_device() != dev:
        _refuse("table must be an int32 tensor [n_seq, max_blocks] on the cache's device")
    n, blocks = table.shape
    stride, step = table.stride()
    if not (step == 1 or blocks == 1) or (n > 1 and stride < blocks):
        _refuse("table must have rows of consecutive elements")
    return Kv8Cache(codes.data_ptr(), at, table.data_ptr(), max(stride, blocks), nb, blocks, kvh, hd, fmt), n, dev


def _kv8_tokens(x, c, total, dev, what):
    """Row stride of a tensor of tokens [total, n_kv_heads, head_dim] whose heads lie side by side."""
    kvh, hd = c.n_kv_heads, c.head_dim
    if x.shape != (total, kvh, hd) or x.get_device() != dev:
        _refuse(f"{what} must be [{total}, {kvh}, {hd}] on the cache's device")
    row, head, step = x.stride()
    if step != 1 or not (kvh == 1 or head == hd):
        _refuse(f"{what} must have each token's heads side by side")
    return row


def kv8_cache(n_blocks: int, n_kv_heads: int, head_dim: int, dtype=None, device="cuda"):
    """An empty 8-bit paged KV cache: codes [n_blocks, 2, n_kv_heads, 128, head_dim] (torch.float8_e4m3fn, the default, or
    torch.int8) and scales [n_blocks, 2, n_kv_heads, 4]."""
    if torch is None:
        _import_torch()
    codes = torch.zeros((n_blocks, 2, n_kv_heads, KV8_PAGE, head_dim), dtype=torch.uint8, device=device)
    scales = torch.ones((n_blocks, 2, n_kv_heads, KV8_PAGE // KV8_SCALE), dtype=torch.float32, device=device)
    return codes.view(dtype or torch.float8_e4m3fn), scales


def kv8_write(codes, scales, table, k, v, pos0, seq_start, status=None):
    """Quantise new tokens into the cache (see sara_kv8_write): rows seq_start[i] .. seq_start[i + 1] of k and v
    [T, n_kv_heads, head_dim] (bf16 or fp16) become positions pos0[i], pos0[i] + 1, ... of sequence i, whose blocks stand
    in table[i].  pos0 [n_seq] and seq_start [n_seq + 1] int32; status: int32 [1], set to SARA_EINVAL by a wrong range or
    block id.  Everything on one GPU."""
    c, n, dev = _kv8(codes, scales, table)
    total, typ = k.shape[0], _types.get(k.dtype, 2)
    if typ == 2 or v.dtype != k.dtype:
        _refuse("k and v must both be bf16 or fp16")
    _launch(dev, load().sara_kv8_write, ctypes.byref(c), n, _vector(pos0, _int32, n, dev, "pos0"),
            _vector(seq_start, _int32, n + 1, dev, "seq_start"), total, k.data_ptr(), _kv8_tokens(k, c, total, dev, "k"),
            v.data_ptr(), _kv8_tokens(v, c, total, dev, "v"), typ, _vector(status, _int32, 1, dev, "status"))


def kv8_read(codes, scales, table, pos0, seq_start, total: int, dtype=None, status=None, out=None):
    """Read positions back (see sara_kv8_read): (k, v), each [total, n_kv_heads, head_dim] of `dtype` (bf16, the default, fp16 or
    fp32), row seq_start[i] + j holding position pos0[i] + j of sequence i.  `out`: (k, v) to write into instead; rows
    of no sequence are left as they are there, and are not defined otherwise."""
    c, n, dev = _kv8(codes, scales, table)
    if out is None:
        shape, dtype = (total, c.n_kv_heads, c.head_dim), dtype or torch.bfloat16
        k, v = scales.new_empty(shape, dtype=dtype), scales.new_empty(shape, dtype=dtype)
        ks = vs = c.n_kv_heads * c.head_dim
    else:
        k, v = out
        ks, vs = _kv8_tokens(k, c, total, dev, "out[0]"), _kv8_tokens(v, c, total, dev, "out[1]")
    typ = _types.get(k.dtype)
    if typ is None or v.dtype != k.dtype:
        _refuse("what is read must be bf16, fp16 or fp32")
    _launch(dev, load().sara_kv8_read, ctypes.byref(c), n, _vector(pos0, _int32, n, dev, "pos0"),
            _vector(seq_start, _int32, n + 1, dev, "seq_start"), total, k.data_ptr(), ks, v.data_ptr(), vs, typ,
            _vector(status, _int32, 1, dev, "status"))
    return k, v


def attention_kv8_workspace(n_seq: int, n_heads: int, n_kv_heads: int, head_dim: int, device="cuda"):
    """The scratch of attention_decode_kv8 for up to these sizes, to be kept from call to call (zeroed; calls that
    share it must not overlap)."""
    if torch is None:
        _import_torch()
    return torch.zeros(load().sara_attention_kv8_workspace_bytes(n_seq, n_heads, n_kv_heads, head_dim), dtype=torch.uint8,
                       device=device)


def attention_decode_kv8(q, codes, scales, table, ctx, first=None, workspace=None, out=None, lse=None, status=None):
    """Decode attention over the 8-bit cache (see sara_attention_decode_kv8): q [n_seq, n_heads, head_dim] bf16 or fp16, row i over
    positions first[i] (None: 0) <= p < ctx[i] of sequence i; returns `out`, like q.  lse: fp32 [n_seq, n_heads] that receives the
    logarithm of each row's sum."""
    c, n, dev = _kv8(codes, scales, table)
    typ, shape, hd = _types.get(q.dtype, 2), q.shape, c.head_dim
    if typ == 2 or len(shape) != 3 or shape[0] != n or shape[2] != hd or q.get_device() != dev:
        _refuse(f"q must be bf16 or fp16, [{n}, heads, {hd}] on the cache's device")
    H = shape[1]
    row, head, step = q.stride()
    if step != 1 or not (H == 1 or head == hd):
        _refuse("q must have each row's heads side by side")
    if out is None:
        out = q.new_empty(shape)
        at = out.data_ptr()
    else:
        at = _matrix(out, q.dtype, shape, dev, "out")
    if workspace is None:
        workspace = attention_kv8_workspace(n, H, c.n_kv_heads, hd, q.device)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        _refuse("workspace must be contiguous, on the cache's device")
    _launch(dev, load().sara_attention_decode_kv8, ctypes.byref(c), n, H, q.data_ptr(), row, _vector(ctx, _int32, n, dev, "ctx"),
            _vector(first, _int32, n, dev, "first"), at, _matrix(lse, _fp32, (n, H), dev, "lse"), typ,
            _vector(status, _int32, 1, dev, "status"), workspace.data_ptr(), workspace.nbytes)
    return out


@dataclass
class LogProbs:
    logprob: object            # [R] fp32, of the given tokens (None without tokens)
    entropy: object            # [R] fp32
    stats: object              # [R, 2] fp32: each row's maximum and the logarithm of its sum, for logprobs_backward
    top_token: object = None   # [R, top] int32, -1 behind the last alternative
    top_logprob: object = None  # [R, top] fp32


def _logits(z, what="logits"):
    """Type, row stride and GPU of a matrix of logits."""
    if torch is None:
        _import_torch()
    typ = _types.get(z.dtype)
    if typ is None or z.dim() != 2:
        _refuse(f"{what} must be bf16, fp16 or fp32, [rows, vocabulary]")
    row, step = z.stride()
    if step != 1 and z.shape[1] != 1:
        _refuse(f"{what} must have rows of consecutive elements")
    return typ, row, z.get_device()


def logprobs(logits, tokens, top: int = 0) -> LogProbs:
    """Log-probabilities of one token per row of logits [R, V] (bf16, fp16 or fp32; rows may be strided), each row's
    entropy and its `top` (at most 32) most probable tokens (see sara_logprobs).  tokens [R] int32, negative for rows
    of padding; None: entropy and alternatives alone."""
    typ, row, dev = _logits(logits)
    R, V = logits.shape
    if not 0 <= top <= 32:
        _refuse("top must be 0 .. 32")
    tok = _vector(tokens, _int32, R, dev, "tokens")
    # (an allocation each: views of one cost more host time)
    lp = logits.new_empty(R, dtype=_fp32) if tok is not None else None
    ent, stats = logits.new_empty(R, dtype=_fp32), logits.new_empty((R, 2), dtype=_fp32)
    tt = tl = None
    if top:
        tt, tl = logits.new_empty((R, top), dtype=_int32), logits.new_empty((R, top), dtype=_fp32)
    _launch(dev, load().sara_logprobs, logits.data_ptr(), row, typ, R, V, tok, top, None if lp is None else lp.data_ptr(),
            ent.data_ptr(), stats.data_ptr(), None if tt is None else tt.data_ptr(), None if tl is None else tl.data_ptr())
    return LogProbs(lp, ent, stats, tt, tl)


def logprobs_backward(logits, tokens, stats, entropy, grad_logprob=None, grad_entropy=None, out=None):
    """Gradient of logprobs with respect to the logits (see sara_logprobs_backward), in the logits' type: grad_logprob and
    grad_entropy [R] fp32 weigh the rows' log-probabilities and entropies.  `out` may be `logits` itself."""
    typ, row, dev = _logits(logits)
    shape = logits.shape
    R, V = shape
    if out is None:
        out, orow = logits.new_empty(shape), V
    else:
        otyp, orow, odev = _logits(out, "out")
        if otyp != typ or odev != dev or out.shape != shape:
            _refuse("out must be like logits")
    _launch(dev, load().sara_logprobs_backward, logits.data_ptr(), row, typ, R, V, _vector(tokens, _int32, R, dev, "tokens"),
            _matrix(stats, _fp32, (R, 2), dev, "stats"), _vector(entropy, _fp32, R, dev, "entropy"),
            _vector(grad_logprob, _fp32, R, dev, "grad_logprob"), _vector(grad_entropy, _fp32, R, dev, "grad_entropy"),
            out.data_ptr(), orow)
    return out
