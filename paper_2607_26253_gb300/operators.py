"""Operators on torch CUDA tensors over an 8-bit paged KV cache and over the logits of sampled tokens (include/sara.h).

Results are not recorded by autograd: logprobs has its gradient as a call of its own.  These are a decode step's calls, and
most of them cost more on the host than on the GPU: checks are written out where they are made, messages put together only for a
refusal, and the cache's description is packed as bytes instead of a ctypes structure (~2 us of 14 a call).
"""
from __future__ import annotations

import struct
from dataclasses import dataclass

from .sara import SARA_EINVAL, SaraError, _check, load

KV8_PAGE, KV8_SCALE = 128, 32   # positions of a cache block, and of a scale
_MOST = 2 ** 31 - 1             # of anything that is counted (the C calls' int32)

torch = None   # imported by the first call, as the rest of the package does
_lib = None
_types = {}    # torch dtype -> SARA_BF16, SARA_FP16, SARA_FP32
_formats = {}  # torch dtype -> SARA_KV8_*
_int32 = _fp32 = _device = _stream = None
_pack_cache = struct.Struct("@QQQqiiiii4x").pack  # sara_kv8_cache


def _start():
    global torch, _lib, _int32, _fp32, _device, _stream
    import torch as t
    _types.update({t.bfloat16: 0, t.float16: 1, t.float32: 2})
    _formats.update({t.float8_e4m3fn: 0, t.int8: 1})
    _int32, _fp32 = t.int32, t.float32
    _device, _stream = t._C._cuda_getDevice, t._C._cuda_getCurrentRawStream  # the current GPU; a GPU's current stream
    _lib = load()
    torch = t


def _refuse(msg):
    raise SaraError(SARA_EINVAL, msg)


def _elsewhere(dev, fn, *args):
    """fn(*args) with GPU dev, which is not the current one, made so."""
    if dev < 0:
        _refuse("operands must be CUDA tensors")
    with torch.cuda.device(dev):
        return fn(*args)


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


def _kv8(codes, scales, table):
    """A cache's tensors, checked: the packed sara_kv8_cache, sequences, KV heads, head dim, GPU."""
    if torch is None:
        _start()
    fmt, dev, shape = _formats.get(codes.dtype), codes.get_device(), codes.shape
    if fmt is None or len(shape) != 5 or shape[1] != 2 or shape[3] != KV8_PAGE or not codes.is_contiguous():
        _refuse("codes must be contiguous, float8_e4m3fn or int8, [n_blocks, 2, n_kv_heads, 128, head_dim]")
    nb, _, kvh, _, hd = shape
    if scales.dtype is not _fp32 or scales.shape != (nb, 2, kvh, 4) or scales.get_device() != dev or not scales.is_contiguous():
        _refuse(f"scales must be contiguous, fp32, {(nb, 2, kvh, 4)}, on the cache's device")
    if table.dtype is not _int32 or table.dim() != 2 or table.get_device() != dev:
        _refuse("table must be an int32 tensor [n_seq, max_blocks] on the cache's device")
    n, blocks = table.shape
    stride, step = table.stride()
    if (step != 1 and blocks != 1) or (n > 1 and stride < blocks):
        _refuse("table must have rows of consecutive elements")
    if n > _MOST or blocks > _MOST:
        _refuse("table must have at most 2^31 - 1 rows and columns")
    if stride < blocks:
        stride = blocks
    return _pack_cache(codes.data_ptr(), scales.data_ptr(), table.data_ptr(), stride, nb, blocks, kvh, hd, fmt), n, kvh, hd, dev


def _tokens(x, total, kvh, hd, dev, what):
    """Row stride of a tensor of tokens [total, kvh, hd] whose heads lie side by side."""
    if x.shape != (total, kvh, hd) or x.get_device() != dev:
        _refuse(f"{what} must be [{total}, {kvh}, {hd}] on the cache's device")
    row, head, step = x.stride()
    if step != 1 or (head != hd and kvh != 1):
        _refuse(f"{what} must have each token's heads side by side")
    return row


def kv8_cache(n_blocks: int, n_kv_heads: int, head_dim: int, dtype=None, device="cuda"):
    """An empty 8-bit paged KV cache: codes [n_blocks, 2, n_kv_heads, 128, head_dim] (torch.float8_e4m3fn, the default, or
    torch.int8) and scales [n_blocks, 2, n_kv_heads, 4].  Blocks that go from one sequence to another which does not write them from their
    first position on want their scales set to 2^-100 again, as they are here."""
    if torch is None:
        _start()
    codes = torch.zeros((n_blocks, 2, n_kv_heads, KV8_PAGE, head_dim), dtype=torch.uint8, device=device)
    # (the lowest scale: a block's first tokens set their own, wherever in it they stand)
    scales = torch.full((n_blocks, 2, n_kv_heads, KV8_PAGE // KV8_SCALE), 2.0 ** -100, dtype=torch.float32, device=device)
    return codes.view(dtype or torch.float8_e4m3fn), scales


def kv8_write(codes, scales, table, k, v, pos0, seq_start, status=None):
    """Quantise new tokens into the cache (see sara_kv8_write): rows seq_start[i] .. seq_start[i + 1] of k and v
    [T, n_kv_heads, head_dim] (bf16 or fp16) become positions pos0[i], pos0[i] + 1, ... of sequence i, whose blocks stand
    in table[i].  pos0 [n_seq] and seq_start [n_seq + 1] int32; status: int32 [1], set to SARA_EINVAL by a wrong range or
    block id.  Everything on one GPU."""
    cache, n, kvh, hd, dev = _kv8(codes, scales, table)
    total, typ = k.shape[0], _types.get(k.dtype, 2)
    if typ == 2 or v.dtype is not k.dtype:
        _refuse("k and v must both be bf16 or fp16")
    if total > _MOST:
        _refuse("k and v must have at most 2^31 - 1 rows")
    ks, vs = _tokens(k, total, kvh, hd, dev, "k"), _tokens(v, total, kvh, hd, dev, "v")
    at_pos, at_start = _vector(pos0, _int32, n, dev, "pos0"), _vector(seq_start, _int32, n + 1, dev, "seq_start")
    at_status = None if status is None else _vector(status, _int32, 1, dev, "status")
    if dev < 0 or dev != _device():
        return _elsewhere(dev, kv8_write, codes, scales, table, k, v, pos0, seq_start, status)
    rc = _lib.sara_kv8_write(cache, n, at_pos, at_start, total, k.data_ptr(), ks, v.data_ptr(), vs, typ, at_status, _stream(dev))
    if rc:
        _check(rc)


def kv8_read(codes, scales, table, pos0, seq_start, total: int, dtype=None, status=None, out=None):
    """Read positions back (see sara_kv8_read): (k, v), each [total, n_kv_heads, head_dim] of `dtype` (bf16, the default, fp16 or
    fp32), row seq_start[i] + j holding position pos0[i] + j of sequence i.  `out`: (k, v) to write into instead; rows
    of no sequence are left as they are there, and are not defined otherwise."""
    cache, n, kvh, hd, dev = _kv8(codes, scales, table)
    if not 0 <= total <= _MOST:
        _refuse("total must be 0 .. 2^31 - 1")
    at_pos, at_start = _vector(pos0, _int32, n, dev, "pos0"), _vector(seq_start, _int32, n + 1, dev, "seq_start")
    at_status = None if status is None else _vector(status, _int32, 1, dev, "status")
    if dev < 0 or dev != _device():
        return _elsewhere(dev, kv8_read, codes, scales, table, pos0, seq_start, total, dtype, status, out)
    if out is None:
        shape, dtype = (total, kvh, hd), dtype or torch.bfloat16
        k, v = scales.new_empty(shape, dtype=dtype), scales.new_empty(shape, dtype=dtype)
        ks = vs = kvh * hd
    else:
        k, v = out
        ks, vs = _tokens(k, total, kvh, hd, dev, "out[0]"), _tokens(v, total, kvh, hd, dev, "out[1]")
    typ = _types.get(k.dtype)
    if typ is None or v.dtype is not k.dtype:
        _refuse("what is read must be bf16, fp16 or fp32")
    rc = _lib.sara_kv8_read(cache, n, at_pos, at_start, total, k.data_ptr(), ks, v.data_ptr(), vs, typ, at_status, _stream(dev))
    if rc:
        _check(rc)
    return k, v


def attention_kv8_workspace(n_seq: int, n_heads: int, n_kv_heads: int, head_dim: int, device="cuda"):
    """The scratch of attention_decode_kv8 for up to these sizes, to be kept from call to call (zeroed; calls that
    share it must not overlap)."""
    if torch is None:
        _start()
    return torch.zeros(_lib.sara_attention_kv8_workspace_bytes(n_seq, n_heads, n_kv_heads, head_dim), dtype=torch.uint8, device=device)


def attention_decode_kv8(q, codes, scales, table, ctx, first=None, workspace=None, out=None, lse=None, status=None):
    """Decode attention over the 8-bit cache (see sara_attention_decode_kv8): q [n_seq, n_heads, head_dim] bf16 or fp16, row i over
    positions first[i] (None: 0) <= p < ctx[i] of sequence i; returns `out`, like q.  lse: fp32 [n_seq, n_heads] that receives the
    logarithm of each row's sum."""
    cache, n, kvh, hd, dev = _kv8(codes, scales, table)
    typ, shape = _types.get(q.dtype, 2), q.shape
    if typ == 2 or len(shape) != 3 or shape[0] != n or shape[2] != hd or q.get_device() != dev:
        _refuse(f"q must be bf16 or fp16, [{n}, heads, {hd}] on the cache's device")
    H = shape[1]
    row, head, step = q.stride()
    if step != 1 or (head != hd and H != 1):
        _refuse("q must have each row's heads side by side")
    at_ctx = _vector(ctx, _int32, n, dev, "ctx")
    at_first = None if first is None else _vector(first, _int32, n, dev, "first")
    at_lse = None if lse is None else _matrix(lse, _fp32, (n, H), dev, "lse")
    at_status = None if status is None else _vector(status, _int32, 1, dev, "status")
    at_out = None if out is None else _matrix(out, q.dtype, shape, dev, "out")
    if workspace is not None and (workspace.get_device() != dev or not workspace.is_contiguous()):
        _refuse("workspace must be contiguous, on the cache's device")
    if dev < 0 or dev != _device():
        return _elsewhere(dev, attention_decode_kv8, q, codes, scales, table, ctx, first, workspace, out, lse, status)
    if out is None:
        out = q.new_empty(shape)
        at_out = out.data_ptr()
    if workspace is None:
        workspace = attention_kv8_workspace(n, H, kvh, hd, q.device)
    rc = _lib.sara_attention_decode_kv8(cache, n, H, q.data_ptr(), row, at_ctx, at_first, at_out, at_lse, typ, at_status,
                                        workspace.data_ptr(), workspace.nbytes, _stream(dev))
    if rc:
        _check(rc)
    return out


@dataclass
class LogProbs:
    logprob: object            # [R] fp32, of the given tokens (None without tokens)
    entropy: object            # [R] fp32
    stats: object              # [R, 2] fp32: each row's maximum and the logarithm of its sum, for logprobs_backward
    top_token: object = None   # [R, top] int32, -1 behind the last alternative
    top_logprob: object = None  # [R, top] fp32


def _logits(z, what="logits"):
    """Type, rows, vocabulary, row stride and GPU of a matrix of logits."""
    if torch is None:
        _start()
    typ = _types.get(z.dtype)
    if typ is None or z.dim() != 2:
        _refuse(f"{what} must be bf16, fp16 or fp32, [rows, vocabulary]")
    R, V = z.shape
    row, step = z.stride()
    if step != 1 and V != 1:
        _refuse(f"{what} must have rows of consecutive elements")
    if R > _MOST or V > _MOST:
        _refuse(f"{what} must have at most 2^31 - 1 rows and columns")
    return typ, R, V, row, z.get_device()


def logprobs(logits, tokens, top: int = 0) -> LogProbs:
    """Log-probabilities of one token per row of logits [R, V] (bf16, fp16 or fp32; rows may be strided), each row's
    entropy and its `top` (at most 32) most probable tokens (see sara_logprobs).  tokens [R] int32, negative for rows
    of padding; None: entropy and alternatives alone."""
    typ, R, V, row, dev = _logits(logits)
    if not 0 <= top <= 32:
        _refuse("top must be 0 .. 32")
    tok = None if tokens is None else _vector(tokens, _int32, R, dev, "tokens")
    if dev < 0 or dev != _device():
        return _elsewhere(dev, logprobs, logits, tokens, top)
    # (an allocation each: views of one cost more host time)
    new = logits.new_empty
    ent, stats = new(R, dtype=_fp32), new((R, 2), dtype=_fp32)
    lp = at_lp = tt = tl = at_tt = at_tl = None
    if tokens is not None:
        lp = new(R, dtype=_fp32)
        at_lp = lp.data_ptr()
    if top:
        tt, tl = new((R, top), dtype=_int32), new((R, top), dtype=_fp32)
        at_tt, at_tl = tt.data_ptr(), tl.data_ptr()
    rc = _lib.sara_logprobs(logits.data_ptr(), row, typ, R, V, tok, top, at_lp, ent.data_ptr(), stats.data_ptr(), at_tt, at_tl,
                            _stream(dev))
    if rc:
        _check(rc)
    return LogProbs(lp, ent, stats, tt, tl)


def logprobs_backward(logits, tokens, stats, entropy, grad_logprob=None, grad_entropy=None, out=None):
    """Gradient of logprobs with respect to the logits (see sara_logprobs_backward), in the logits' type: grad_logprob and
    grad_entropy [R] fp32 weigh the rows' log-probabilities and entropies.  `out` may be `logits` itself."""
    typ, R, V, row, dev = _logits(logits)
    at_tok, at_stats = _vector(tokens, _int32, R, dev, "tokens"), _matrix(stats, _fp32, (R, 2), dev, "stats")
    at_ent, at_g = _vector(entropy, _fp32, R, dev, "entropy"), _vector(grad_logprob, _fp32, R, dev, "grad_logprob")
    at_gh = _vector(grad_entropy, _fp32, R, dev, "grad_entropy")
    if out is not None:
        otyp, oR, oV, orow, odev = _logits(out, "out")
        if otyp != typ or odev != dev or oR != R or oV != V:
            _refuse("out must be like logits")
    if dev < 0 or dev != _device():
        return _elsewhere(dev, logprobs_backward, logits, tokens, stats, entropy, grad_logprob, grad_entropy, out)
    if out is None:
        out, orow = logits.new_empty((R, V)), V
    rc = _lib.sara_logprobs_backward(logits.data_ptr(), row, typ, R, V, at_tok, at_stats, at_ent, at_g, at_gh, out.data_ptr(), orow,
                                     _stream(dev))
    if rc:
        _check(rc)
    return out
