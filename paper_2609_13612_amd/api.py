"""Python binding of the C ABI in include/attnfuse.h and attnfuse_llm.h -- argument marshalling only.

Each function takes torch tensors that already live on the GPU, checks their
shape/dtype/contiguity against the call, passes raw device pointers and the
current torch stream to the library, and raises AttnFuseError on a non-zero
return code.  Every step of the computation runs in the HIP kernels.

Plain calls are marshalled by native/binding.cpp, which does the same checks;
it declines (returns None) whatever it does not recognise, and the Python code
after it then marshals the call or raises.
"""
import ctypes
import functools
import math

import numpy as np
import torch

from . import _lib

try:   # the native half of this module: the same calls with their marshalling in C++
    from . import _native
except ImportError:   # not built for this interpreter: every call is marshalled below
    _native = None

DTYPE = {torch.bfloat16: 0, torch.float32: 1}
ROPE = {"none": 0, "neox": 1, "interleaved": 2}
MASK = {"none": 0, "causal": 1, "sliding_window": 2}
SECTION_ORDER = {"blocks": 0, "turns": 1}
FREQUENCIES = {"shared": 0, "own": 1}


class AttnFuseError(RuntimeError):
    def __init__(self, code, where):
        msg = _lib.load().attnfuse_strerror(code).decode()
        super().__init__(f"{where}: {msg} (code {code})")
        self.code = code


def _check(code, where):
    if code != 0:
        raise AttnFuseError(code, where)


def _result(r, where):
    """The outputs of a native call, which returns the library's code when that is not 0."""
    if type(r) is int:
        raise AttnFuseError(r, where)
    return r


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _shape(q, k):
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q must be [B, H, S, D] and k/v [B, H_kv, S, D]")
    B, H, S, D = q.shape
    if k.shape[0] != B or k.shape[2] != S or k.shape[3] != D:
        raise ValueError("k/v must be [B, H_kv, S, D] matching q")
    return B, H, k.shape[1], S, D


def _device(q):
    """The GPU that q lives on (every other tensor of the call must be there too)."""
    if not isinstance(q, torch.Tensor) or not q.is_cuda:
        raise ValueError("q must be a tensor on a GPU")
    if q.dtype not in DTYPE:
        raise ValueError(f"dtype must be one of {sorted(str(d) for d in DTYPE)}")
    return q.device


def _need(t, name, shape, dtype, device):
    """Raise unless t is a contiguous tensor of exactly that shape and dtype on device."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.device != device:
        raise ValueError(f"{name} must be on {device} (it is on {t.device})")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype} (it is {t.dtype})")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)} (it has {tuple(t.shape)})")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _opt(t, name, shape, dtype, device):
    """A caller-provided output: checked like an input, or allocated."""
    if t is None:
        return torch.empty(shape, device=device, dtype=dtype)
    _need(t, name, shape, dtype, device)
    return t


def _inputs(q, k, v, device):
    """q [B, H, S, D]; k and v [B, H_kv, S, D] of q's dtype, all on q's device."""
    _need(q, "q", q.shape, q.dtype, device)
    _need(k, "k", k.shape, q.dtype, device)
    _need(v, "v", k.shape, q.dtype, device)


def _bwd_inputs(q, k, v, o, do, lse, device, lse_needed):
    _inputs(q, k, v, device)
    _need(o, "o", q.shape, q.dtype, device)
    _need(do, "do", q.shape, q.dtype, device)
    if lse is not None or lse_needed:
        _need(lse, "lse", q.shape[:3], torch.float32, device)


def _grads(q, k, dq, dk, dv, device):
    return (_opt(dq, "dq", q.shape, q.dtype, device), _opt(dk, "dk", k.shape, q.dtype, device),
            _opt(dv, "dv", k.shape, q.dtype, device))


def _workspace(ws, nbytes, device):
    """(tensor, size in bytes) of the workspace: the caller's, checked, or a new one."""
    if ws is None:
        return torch.empty(nbytes, device=device, dtype=torch.uint8), nbytes
    if not isinstance(ws, torch.Tensor) or ws.device != device or not ws.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on q's device")
    return ws, ws.numel() * ws.element_size()


# RoPE cos/sin tables this binding built, per (device index, D, theta): a list
# of tables (each a [rows, D/2, 2] fp32 tensor), never freed, since a kernel
# on any stream may still read one.  The library itself keeps nothing.
_TABLES = {}
_TABLE_MIN_ROWS = 4096


def rope_table(D, theta, rows, device=None, out=None, *, sections=None, section_order="blocks", frequencies="shared"):
    """A RoPE cos/sin table for positions 0..rows-1: T[n][i] = (cos, sin) of
    n * theta^(-2i/D), filled by attnfuse_rope_table_fill on the current stream
    (see include/attnfuse.h).  Pass it as ``rope_table=`` to any call with the
    same D and theta and S <= rows.  With ``sections`` and frequencies="own" it is
    that of positions of several axes, each with its own ladder of frequencies
    (attnfuse_axes_table_fill), for calls with the same sections in the same order."""
    if sections is not None:
        sections, section_order = _sections(sections, section_order, frequencies, D)
    device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    shape = (rows, D // 2, 2)
    if out is None:
        out = torch.empty(shape, device=device, dtype=torch.float32)
    else:
        _need(out, "out", shape, torch.float32, device)
    with torch.cuda.device(device):
        if sections is None:
            code = _lib.load().attnfuse_rope_table_fill(out.data_ptr(), rows, D, float(theta), _stream())
        else:
            code = _lib.load().attnfuse_axes_table_fill(out.data_ptr(), rows, D, float(theta), len(sections),
                                                        (ctypes.c_int * len(sections))(*sections),
                                                        SECTION_ORDER[section_order], FREQUENCIES[frequencies], _stream())
    _check(code, "attnfuse_rope_table_fill" if sections is None else "attnfuse_axes_table_fill")
    return out


def _table(rope, theta, D, S, device, given, own=None):
    """The cos/sin table a call reads, as a tensor: the caller's (checked), or
    one this binding keeps for (device, D, theta).  Under HIP graph capture a
    table not yet built is filled inside the capture (stream-ordered before the
    call that reads it) and not kept; the caller holds the returned tensor
    until its launch is enqueued.  own: (sections, section_order) where every axis
    has its own frequencies.  None without RoPE."""
    if ROPE[rope] == ROPE["none"]:
        return None
    if given is not None:
        if (not isinstance(given, torch.Tensor) or given.device != device or given.dtype != torch.float32
                or given.dim() != 3 or tuple(given.shape[1:]) != (D // 2, 2) or not given.is_contiguous()):
            raise ValueError(f"rope_table must be a contiguous fp32 [rows, {D // 2}, 2] tensor on {device}")
        if given.shape[0] < S:
            raise ValueError(f"rope_table has {given.shape[0]} rows, the call needs {S}")
        return given
    key = (device.index, D, float(np.float32(theta))) + (own or ())
    axes = dict(sections=own[0], section_order=own[1], frequencies="own") if own else {}
    for t in _TABLES.get(key, ()):
        if t.shape[0] >= S:
            return t
    rows = _TABLE_MIN_ROWS
    while rows < S:
        rows *= 2
    with torch.cuda.device(device):
        if torch.cuda.is_current_stream_capturing():
            return rope_table(D, theta, S, device, **axes)
        t = rope_table(D, theta, rows, device, **axes)
        # ready for any stream before it is shared: one wait, once per table
        torch.cuda.current_stream().synchronize()
    _TABLES.setdefault(key, []).append(t)
    return t


def _tab(t):
    """(pointer, rows) of a table from _table."""
    return (None, 0) if t is None else (t.data_ptr(), t.shape[0])


def _count(n):
    """A window, or a number of sinks, in the library's 32 bits (ctypes would drop the others): from there on a larger one
    shows no more keys, and a negative one is refused as -1 is."""
    return max(-1, min(int(n or 0), 2 ** 31 - 1))


def _variant(rope, theta, mask, window, alibi_slopes, scale, D, H=None, device=None):
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    if alibi_slopes is not None:
        _need(alibi_slopes, "alibi_slopes", (H,), torch.float32, device)
    return ROPE[rope], float(theta), MASK[mask], _count(window), scale


@functools.lru_cache(maxsize=4096)
def _fwd_scratch_bytes(*sizes):
    """af_fwd_workspace_bytes, a pure function of the sizes (a dictionary lookup costs the smallest calls less)."""
    return _lib.load().af_fwd_workspace_bytes(*sizes)


def _fwd_scratch(q, B, H, Hkv, S, D, r, m, w, blocks=0, norm=0, extra=0):
    """Scratch for keys rotated once ahead of a forward, where that is faster
    (af_fwd_workspace_bytes), else None.  Without memory for it the keys are
    rotated in the loop: the same result."""
    n = _fwd_scratch_bytes(B, H, Hkv, S, D, DTYPE[q.dtype], r, m, w, norm, extra, blocks) if r else 0
    if n == 0:
        return None
    try:
        return torch.empty(n, device=q.device, dtype=torch.uint8)
    except torch.OutOfMemoryError:
        return None


def attnfuse_fwd(q, k, v, *, rope="none", theta=10000.0, mask="causal", window=None,
                 alibi_slopes=None, scale=None, out=None, lse=None, rope_table=None, sinks=0):
    """O, LSE = attention(q, k, v); see attnfuse_fwd in include/attnfuse.h, and for
    ``sinks`` > 0 (first keys that stay visible under a sliding window)
    attnfuse_fwd_sinks in include/attnfuse_llm.h."""
    if sinks:
        return _fwd_sinks(q, k, v, rope, theta, mask, window, alibi_slopes, scale, out, lse, rope_table, sinks)
    if _native is not None:
        r = _native.fwd(q, k, v, out, lse, alibi_slopes, rope_table, _TABLES, ROPE.get(rope, -1), theta,
                        MASK.get(mask, -1), window, scale, 0, 0, 0, 0, 0, 0, 0, 0)
        if r is not None:
            return _result(r, "attnfuse_fwd")
    dev = _device(q)
    B, H, Hkv, S, D = _shape(q, k)
    _inputs(q, k, v, dev)
    out = _opt(out, "out", q.shape, q.dtype, dev)
    lse = _opt(lse, "lse", (B, H, S), torch.float32, dev)
    r, th, m, w, sc = _variant(rope, theta, mask, window, alibi_slopes, scale, D, H, dev)
    tab = _table(rope, theta, D, S, dev, rope_table)
    tp, tr = _tab(tab)
    ws = _fwd_scratch(q, B, H, Hkv, S, D, r, m, w, extra=int(alibi_slopes is not None))
    with torch.cuda.device(dev):
        if ws is not None:
            code = _lib.load().af_fwd_ws(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), None, None, None, 0, 0, 0, 0,
                                         ws.data_ptr(), ws.numel(), B, H, Hkv, S, D, DTYPE[q.dtype], r, th, tp, tr, m,
                                         w, _ptr(alibi_slopes), sc, _stream())
            _check(code, "attnfuse_fwd")
            return out, lse
        code = _lib.load().attnfuse_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), B, H, Hkv, S, D,
                                        DTYPE[q.dtype], r, th, tp, tr, m, w, _ptr(alibi_slopes), sc, _stream())
    _check(code, "attnfuse_fwd")
    return out, lse


def attnfuse_bwd_workspace_bytes(B, H, H_kv, S, D, rope="none"):
    return _lib.load().attnfuse_bwd_workspace_bytes(B, H, H_kv, S, D, ROPE[rope])


def attnfuse_bwd(q, k, v, o, do, lse, *, rope="none", theta=10000.0, mask="causal", window=None,
                 alibi_slopes=None, scale=None, dq=None, dk=None, dv=None, workspace=None, rope_table=None, sinks=0):
    """dQ, dK, dV of attnfuse_fwd; see attnfuse_bwd in include/attnfuse.h (with
    ``sinks`` attnfuse_bwd_sinks in include/attnfuse_llm.h)."""
    if sinks:
        return _bwd_sinks(q, k, v, o, do, lse, rope, theta, mask, window, alibi_slopes, scale, dq, dk, dv, workspace,
                          rope_table, sinks)
    if _native is not None:
        r = _native.bwd(q, k, v, o, do, lse, dq, dk, dv, workspace, alibi_slopes, rope_table, _TABLES,
                        ROPE.get(rope, -1), theta, MASK.get(mask, -1), window, scale, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0)
        if r is not None:
            return _result(r, "attnfuse_bwd")
    dev = _device(q)
    B, H, Hkv, S, D = _shape(q, k)
    _bwd_inputs(q, k, v, o, do, lse, dev, lse_needed=True)
    dq, dk, dv = _grads(q, k, dq, dk, dv, dev)
    workspace, wbytes = _workspace(workspace, attnfuse_bwd_workspace_bytes(B, H, Hkv, S, D, rope), dev)
    r, th, m, w, sc = _variant(rope, theta, mask, window, alibi_slopes, scale, D, H, dev)
    tab = _table(rope, theta, D, S, dev, rope_table)
    tp, tr = _tab(tab)
    with torch.cuda.device(dev):
        code = _lib.load().attnfuse_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(do), _ptr(lse),
                                        _ptr(dq), _ptr(dk), _ptr(dv), _ptr(workspace), wbytes,
                                        B, H, Hkv, S, D, DTYPE[q.dtype], r, th, tp, tr, m, w,
                                        _ptr(alibi_slopes), sc, _stream())
    _check(code, "attnfuse_bwd")
    return dq, dk, dv


def _mask_ptrs(block_mask, q, S):
    if block_mask.S != S:
        raise ValueError(f"block mask built for S={block_mask.S}, tensors have S={S}")
    ts = (block_mask.q_ptr, block_mask.k_idx, block_mask.k_ptr, block_mask.q_idx)
    for t in ts:
        if t.device != q.device or t.dtype != torch.int32 or not t.is_contiguous():
            raise ValueError("block mask lists must be contiguous int32 tensors on q's device")
    # the offset arrays are read up to entry nb; their values are those the
    # blockmask constructors built and checked
    nb = (S + 63) // 64
    if block_mask.q_ptr.numel() != nb + 1 or block_mask.k_ptr.numel() != nb + 1:
        raise ValueError(f"block mask offset lists must have nb + 1 = {nb + 1} entries")
    # an empty index list has no storage; any valid aligned address serves
    return [t.data_ptr() if t.numel() else block_mask.q_ptr.data_ptr() for t in ts]


def attnfuse_fwd_blocksparse(q, k, v, block_mask, *, rope="none", theta=10000.0, mask="none", window=None,
                             alibi_slopes=None, scale=None, out=None, lse=None, rope_table=None):
    """O, LSE of attention restricted to the active blocks of ``block_mask``
    (a blockmask.BlockMask); see attnfuse_fwd_blocksparse."""
    dev = _device(q)
    B, H, Hkv, S, D = _shape(q, k)
    _inputs(q, k, v, dev)
    qp, ki, _, _ = _mask_ptrs(block_mask, q, S)
    blocks = max(1, block_mask.k_idx.numel())
    if _native is not None:
        r = _native.fwd(q, k, v, out, lse, alibi_slopes, rope_table, _TABLES, ROPE.get(rope, -1), theta,
                        MASK.get(mask, -1), window, scale, 0, 0, 0, 0, 0, qp, ki, blocks)
        if r is not None:
            return _result(r, "attnfuse_fwd_blocksparse")
    out = _opt(out, "out", q.shape, q.dtype, dev)
    lse = _opt(lse, "lse", (B, H, S), torch.float32, dev)
    r, th, m, w, sc = _variant(rope, theta, mask, window, alibi_slopes, scale, D, H, dev)
    tab = _table(rope, theta, D, S, dev, rope_table)
    tp, tr = _tab(tab)
    ws = _fwd_scratch(q, B, H, Hkv, S, D, r, m, w, blocks, extra=int(alibi_slopes is not None))
    with torch.cuda.device(dev):
        if ws is not None:
            code = _lib.load().af_fwd_ws(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), qp, ki, None, 0, 0, 0, 0,
                                         ws.data_ptr(), ws.numel(), B, H, Hkv, S, D, DTYPE[q.dtype], r, th, tp, tr, m,
                                         w, _ptr(alibi_slopes), sc, _stream())
            _check(code, "attnfuse_fwd_blocksparse")
            return out, lse
        code = _lib.load().attnfuse_fwd_blocksparse(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), qp, ki,
                                                    B, H, Hkv, S, D, DTYPE[q.dtype], r, th, tp, tr, m, w,
                                                    _ptr(alibi_slopes), sc, _stream())
    _check(code, "attnfuse_fwd_blocksparse")
    return out, lse


def attnfuse_bwd_blocksparse(q, k, v, o, do, lse, block_mask, *, rope="none", theta=10000.0, mask="none",
                             window=None, alibi_slopes=None, scale=None, dq=None, dk=None, dv=None,
                             workspace=None, rope_table=None):
    """dQ, dK, dV of attnfuse_fwd_blocksparse; see attnfuse_bwd_blocksparse."""
    dev = _device(q)
    B, H, Hkv, S, D = _shape(q, k)
    _bwd_inputs(q, k, v, o, do, lse, dev, lse_needed=True)
    qp, ki, kp, qi = _mask_ptrs(block_mask, q, S)
    longest, tiles = (block_mask.col_tiles or ((0, 0), (0, 0)))[mask != "none"]
    if _native is not None:
        r = _native.bwd(q, k, v, o, do, lse, dq, dk, dv, workspace, alibi_slopes, rope_table, _TABLES,
                        ROPE.get(rope, -1), theta, MASK.get(mask, -1), window, scale, 0, 0, 0, 0, 0, qp, ki, kp, qi,
                        longest, tiles)
        if r is not None:
            return _result(r, "attnfuse_bwd_blocksparse")
    dq, dk, dv = _grads(q, k, dq, dk, dv, dev)
    workspace, wbytes = _workspace(workspace, attnfuse_bwd_workspace_bytes(B, H, Hkv, S, D, rope), dev)
    r, th, m, w, sc = _variant(rope, theta, mask, window, alibi_slopes, scale, D, H, dev)
    tab = _table(rope, theta, D, S, dev, rope_table)
    tp, tr = _tab(tab)
    with torch.cuda.device(dev):
        code = _lib.load().af_bwd_blocksparse(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(do), _ptr(lse), _ptr(dq),
                                              _ptr(dk), _ptr(dv), qp, ki, kp, qi, longest, tiles, _ptr(workspace),
                                              wbytes, B, H, Hkv, S, D, DTYPE[q.dtype], r, th, tp, tr, m, w,
                                              _ptr(alibi_slopes), sc, _stream())
    _check(code, "attnfuse_bwd_blocksparse")
    return dq, dk, dv


NORM = {"softmax": 0, "relu": 1}


def _bias_args(bias, q, B, H, S):
    """(pointer, stride_b, stride_h, stride_q) of an fp32 GPU bias broadcastable
    to [B, H, S, S] with keys contiguous (broadcast dimensions get stride 0)."""
    if bias is None:
        return None, 0, 0, 0
    if bias.dtype != torch.float32 or bias.device != q.device:
        raise ValueError("bias must be an fp32 tensor on q's device")
    while bias.dim() < 4:
        bias = bias.unsqueeze(0)
    e = bias.expand(B, H, S, S)
    if e.stride(3) != 1:
        raise ValueError("bias must be contiguous along the key dimension")
    return e.data_ptr(), e.stride(0), e.stride(1), e.stride(2)


def attnfuse_fwd_bias_norm(q, k, v, *, bias=None, norm="softmax", rope="none", theta=10000.0, mask="causal",
                           window=None, scale=None, out=None, lse=None, rope_table=None):
    """O (and LSE, None under relu attention) with a dense additive bias and/or
    relu attention; see attnfuse_fwd_bias_norm in include/attnfuse.h."""
    dev = _device(q)
    B, H, Hkv, S, D = _shape(q, k)
    if _native is not None:
        r = _native.fwd(q, k, v, out, lse, None, rope_table, _TABLES, ROPE.get(rope, -1), theta, MASK.get(mask, -1),
                        window, scale, *_bias_args(bias, q, B, H, S), NORM.get(norm, -1),
                        0, 0, 0)
        if r is not None:
            return _result(r, "attnfuse_fwd_bias_norm")
    _inputs(q, k, v, dev)
    out = _opt(out, "out", q.shape, q.dtype, dev)
    if NORM[norm] == NORM["softmax"] or lse is not None:
        lse = _opt(lse, "lse", (B, H, S), torch.float32, dev)
    bp, sb, sh, sq = _bias_args(bias, q, B, H, S)
    r, th, m, w, sc = _variant(rope, theta, mask, window, None, scale, D)
    tab = _table(rope, theta, D, S, dev, rope_table)
    tp, tr = _tab(tab)
    ws = _fwd_scratch(q, B, H, Hkv, S, D, r, m, w, norm=NORM[norm], extra=int(bias is not None))
    with torch.cuda.device(dev):
        if ws is not None:
            code = _lib.load().af_fwd_ws(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), None, None, bp, sb, sh, sq,
                                         NORM[norm], ws.data_ptr(), ws.numel(), B, H, Hkv, S, D, DTYPE[q.dtype], r,
                                         th, tp, tr, m, w, None, sc, _stream())
            _check(code, "attnfuse_fwd_bias_norm")
            return out, lse
        code = _lib.load().attnfuse_fwd_bias_norm(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), bp, sb, sh,
                                                  sq, NORM[norm], B, H, Hkv, S, D, DTYPE[q.dtype], r, th, tp, tr, m, w,
                                                  None, sc, _stream())
    _check(code, "attnfuse_fwd_bias_norm")
    return out, lse


def attnfuse_bwd_bias_norm(q, k, v, o, do, lse, *, bias=None, norm="softmax", rope="none", theta=10000.0,
                           mask="causal", window=None, scale=None, dq=None, dk=None, dv=None, workspace=None,
                           rope_table=None):
    """dQ, dK, dV of attnfuse_fwd_bias_norm (lse may be None under relu
    attention); see attnfuse_bwd_bias_norm."""
    dev = _device(q)
    B, H, Hkv, S, D = _shape(q, k)
    if _native is not None:
        r = _native.bwd(q, k, v, o, do, lse, dq, dk, dv, workspace, None, rope_table, _TABLES, ROPE.get(rope, -1),
                        theta, MASK.get(mask, -1), window, scale, *_bias_args(bias, q, B, H, S), NORM.get(norm, -1),
                        0, 0, 0, 0, 0, 0)
        if r is not None:
            return _result(r, "attnfuse_bwd_bias_norm")
    _bwd_inputs(q, k, v, o, do, lse, dev, lse_needed=NORM[norm] == NORM["softmax"])
    dq, dk, dv = _grads(q, k, dq, dk, dv, dev)
    workspace, wbytes = _workspace(workspace, attnfuse_bwd_workspace_bytes(B, H, Hkv, S, D, rope), dev)
    bp, sb, sh, sq = _bias_args(bias, q, B, H, S)
    r, th, m, w, sc = _variant(rope, theta, mask, window, None, scale, D)
    tab = _table(rope, theta, D, S, dev, rope_table)
    tp, tr = _tab(tab)
    with torch.cuda.device(dev):
        code = _lib.load().attnfuse_bwd_bias_norm(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(do), _ptr(lse),
                                                  _ptr(dq), _ptr(dk), _ptr(dv), bp, sb, sh, sq, NORM[norm],
                                                  _ptr(workspace), wbytes, B, H, Hkv, S, D, DTYPE[q.dtype],
                                                  r, th, tp, tr, m, w, None, sc, _stream())
    _check(code, "attnfuse_bwd_bias_norm")
    return dq, dk, dv


def attnfuse_decode_workspace_bytes(B, H, H_kv, S_kv, D):
    return _lib.load().attnfuse_decode_workspace_bytes(B, H, H_kv, S_kv, D)


def _decode_args(q, k_cache, v_cache, cache_lens, out, lse):
    dev = _device(q)
    if q.dim() != 3 or k_cache.dim() != 4 or v_cache.shape != k_cache.shape:
        raise ValueError("q must be [B, H, D] and the caches [B, H_kv, S_kv, D]")
    B, H, D = q.shape
    Hkv, S_kv = k_cache.shape[1], k_cache.shape[2]
    if k_cache.shape[0] != B or k_cache.shape[3] != D:
        raise ValueError("cache shape does not match q")
    _need(q, "q", q.shape, q.dtype, dev)
    _need(k_cache, "k_cache", k_cache.shape, q.dtype, dev)
    _need(v_cache, "v_cache", k_cache.shape, q.dtype, dev)
    if cache_lens is not None:
        _need(cache_lens, "cache_lens", (B,), torch.int32, dev)
    out = _opt(out, "out", q.shape, q.dtype, dev)
    lse = _opt(lse, "lse", (B, H), torch.float32, dev)
    return dev, (B, H, Hkv, S_kv, D), out, lse


def attnfuse_decode(q, k_cache, v_cache, cache_lens=None, *, rope="none", theta=10000.0, mask="causal",
                    window=None, alibi_slopes=None, scale=None, out=None, lse=None, workspace=None,
                    rope_table=None, sinks=0):
    """O [B,H,D], LSE [B,H] of one query per sequence against a KV cache of
    already-rotated keys; see attnfuse_decode in include/attnfuse.h, and for
    ``sinks`` > 0 (first keys that stay visible under a sliding window)
    attnfuse_decode_sinks in include/attnfuse_llm.h."""
    if sinks:
        return _decode_sinks(q, k_cache, v_cache, cache_lens, rope, theta, mask, window, alibi_slopes, scale, out, lse,
                             workspace, rope_table, sinks)
    if _native is not None:
        r = _native.decode(q, k_cache, v_cache, cache_lens, out, lse, workspace, alibi_slopes, rope_table, _TABLES,
                           ROPE.get(rope, -1), theta, MASK.get(mask, -1), window, scale, 0)
        if r is not None:
            return _result(r, "attnfuse_decode")
    dev, (B, H, Hkv, S_kv, D), out, lse = _decode_args(q, k_cache, v_cache, cache_lens, out, lse)
    workspace, wbytes = _workspace(workspace, attnfuse_decode_workspace_bytes(B, H, Hkv, S_kv, D), dev)
    r, th, m, w, sc = _variant(rope, theta, mask, window, alibi_slopes, scale, D, H, dev)
    tab = _table(rope, theta, D, S_kv, dev, rope_table)
    tp, tr = _tab(tab)
    with torch.cuda.device(dev):
        code = _lib.load().attnfuse_decode(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(cache_lens), _ptr(out),
                                           _ptr(lse), _ptr(workspace), wbytes, B, H, Hkv, S_kv, D,
                                           DTYPE[q.dtype], r, th, tp, tr, m, w, _ptr(alibi_slopes), sc, _stream())
    _check(code, "attnfuse_decode")
    return out, lse


def attnfuse_decode_noalloc(q, k_cache, v_cache, cache_lens=None, *, rope="none", theta=10000.0, mask="causal",
                            window=None, alibi_slopes=None, scale=None, out=None, lse=None, rope_table=None):
    """attnfuse_decode with the library's static scratch in place of a
    workspace; see attnfuse_decode_noalloc in include/attnfuse.h.  Pass
    ``out``, ``lse`` (and, with RoPE, ``rope_table``) for a call that
    allocates nothing at all."""
    if _native is not None:
        r = _native.decode(q, k_cache, v_cache, cache_lens, out, lse, None, alibi_slopes, rope_table, _TABLES,
                           ROPE.get(rope, -1), theta, MASK.get(mask, -1), window, scale, 1)
        if r is not None:
            return _result(r, "attnfuse_decode_noalloc")
    dev, (B, H, Hkv, S_kv, D), out, lse = _decode_args(q, k_cache, v_cache, cache_lens, out, lse)
    r, th, m, w, sc = _variant(rope, theta, mask, window, alibi_slopes, scale, D, H, dev)
    tab = _table(rope, theta, D, S_kv, dev, rope_table)
    tp, tr = _tab(tab)
    with torch.cuda.device(dev):
        code = _lib.load().attnfuse_decode_noalloc(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(cache_lens),
                                                   _ptr(out), _ptr(lse), B, H, Hkv, S_kv, D, DTYPE[q.dtype], r, th,
                                                   tp, tr, m, w, _ptr(alibi_slopes), sc, _stream())
    _check(code, "attnfuse_decode_noalloc")
    return out, lse


def _rope_call(name, x0, x1, y0, y1, rope, theta, rope_table):
    if _native is not None:
        r = _native.rope(x0, x1, y0, y1, rope_table, _TABLES, ROPE.get(rope, -1), theta,
                         int(name == "attnfuse_rope_bwd"))
        if r is not None:
            return _result(r, name)
    dev = _device(x0)
    if x1 is not None:
        B, H, Hkv, S, D = _shape(x0, x1)
        _need(x1, "k", x1.shape, x0.dtype, dev)
    else:
        if x0.dim() != 4:
            raise ValueError("q must be [B, H, S, D]")
        B, H, S, D = x0.shape
        Hkv = 1
    _need(x0, "q", x0.shape, x0.dtype, dev)
    y0 = _opt(y0, "out_q", x0.shape, x0.dtype, dev)
    if x1 is not None:
        y1 = _opt(y1, "out_k", x1.shape, x0.dtype, dev)
    elif y1 is not None:
        raise ValueError("out_k needs k")
    tab = _table(rope, theta, D, S, dev, rope_table)
    tp, tr = _tab(tab)
    with torch.cuda.device(dev):
        code = getattr(_lib.load(), name)(_ptr(x0), _ptr(x1), _ptr(y0), _ptr(y1), B, H, Hkv, S, D,
                                          DTYPE[x0.dtype], ROPE[rope], float(theta), tp, tr, _stream())
    _check(code, name)
    return y0, y1


def attnfuse_rope(q, k=None, *, rope="neox", theta=10000.0, out_q=None, out_k=None, rope_table=None):
    """Qr, Kr = R q, R k (separate pre-rotation); see attnfuse_rope."""
    return _rope_call("attnfuse_rope", q, k, out_q, out_k, rope, theta, rope_table)


def attnfuse_rope_bwd(dqr, dkr=None, *, rope="neox", theta=10000.0, out_q=None, out_k=None, rope_table=None):
    """dQ, dK = R^T dQr, R^T dKr; see attnfuse_rope_bwd."""
    return _rope_call("attnfuse_rope_bwd", dqr, dkr, out_q, out_k, rope, theta, rope_table)


def attnfuse_rope_table_bytes(rows, D):
    return _lib.load().attnfuse_rope_table_bytes(rows, D)


# ---------------------------------------------------------------- include/attnfuse_llm.h
def _rows(t, name, shape, dtype, device):
    """The strides, in elements, of a tensor of rows that may lie apart: exactly that shape, type and device, each row
    contiguous and 16-byte aligned.  A dimension of one row has stride 0."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.device != device:
        raise ValueError(f"{name} must be on {device} (it is on {t.device})")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype} (it is {t.dtype})")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)} (it has {tuple(t.shape)})")
    st = [s if n > 1 else 0 for s, n in zip(t.stride()[:-1], t.shape[:-1])]
    if (t.stride(-1) != 1 and t.shape[-1] > 1) or t.data_ptr() % 16 or any(s * t.element_size() % 16 for s in st):
        raise ValueError(f"{name} must have contiguous rows, each 16-byte aligned")
    return st


def _norm_weights(qw, kw, D, dtype, device):
    """The library's code for the type of the norm weights: fp32 or the rows' own, the same for both."""
    given = [w for w in (qw, kw) if w is not None]
    if not given:
        return DTYPE[torch.float32]
    for w, name in ((qw, "q_weight"), (kw, "k_weight")):
        if w is not None:
            if isinstance(w, torch.Tensor) and w.dtype not in (torch.float32, dtype):
                raise ValueError(f"{name} must be {torch.float32} or {dtype} (it is {w.dtype})")
            _need(w, name, (D,), w.dtype if isinstance(w, torch.Tensor) else dtype, device)
            if w.data_ptr() % 16:
                raise ValueError(f"{name} must be 16-byte aligned")
    if given[0].dtype != given[-1].dtype:
        raise ValueError("q_weight and k_weight must have the same dtype")
    return DTYPE[given[0].dtype]


def _position_table(rope, theta, D, n, device, positions, shape, max_positions, rope_table):
    """The table of a call whose rows are at `positions`, or at 0..n-1 without any: its first max_positions rows, where
    that is given, however many more it has."""
    if positions is None or ROPE[rope] == ROPE["none"]:
        return _table(rope, theta, D, n, device, rope_table)
    _need(positions, "positions", shape, torch.int32, device)
    if rope_table is None and max_positions is None:
        raise ValueError("positions need max_positions (every position is below it) or rope_table")
    if max_positions is None:
        return _table(rope, theta, D, 1, device, rope_table)
    if int(max_positions) < 1:
        raise ValueError(f"max_positions must be at least 1 (it is {max_positions})")
    return _table(rope, theta, D, int(max_positions), device, rope_table)[:int(max_positions)]


def _sections(sections, section_order, frequencies, D):
    """Sections, checked, as a tuple of whole numbers, and their order."""
    given, sections = sections, tuple(int(n) for n in sections)
    if section_order not in SECTION_ORDER or frequencies not in FREQUENCIES:
        raise ValueError("section_order is 'blocks' or 'turns', frequencies 'shared' or 'own'")
    if not 1 <= len(sections) <= 4 or min(sections) < 1 or 2 * sum(sections) != D or any(a != b for a, b in zip(sections, given)):
        raise ValueError(f"sections must be one to four whole numbers of pairs, {D // 2} in all (they are {given})")
    return sections, section_order


def _axes(sections, section_order, frequencies, norm, rope, D, positions):
    """The sections of positions of several axes, as a tuple, and their order; None without any."""
    if sections is None:
        if not norm:
            raise ValueError("norm=False needs sections (one axis: sections=(D // 2,) and positions [1, ...])")
        return None
    axes = _sections(sections, section_order, frequencies, D)
    if rope not in ("neox", "interleaved") or positions is None:
        raise ValueError("sections need positions and rope='neox' or 'interleaved'")
    return axes


def _axes_table(axes, frequencies, rope, theta, D, device, max_positions, rope_table):
    """The table of a call with sections, whatever rows it has from max_positions on."""
    if rope_table is None and max_positions is None:
        raise ValueError("positions need max_positions (every position is below it) or rope_table")
    if max_positions is not None and int(max_positions) < 1:
        raise ValueError(f"max_positions must be at least 1 (it is {max_positions})")
    return _table(rope, theta, D, 1 if max_positions is None else int(max_positions), device, rope_table,
                  axes if frequencies == "own" else None)


def _axes_args(axes):
    """axes, sections, section_order of the library's calls."""
    return len(axes[0]), (ctypes.c_int * len(axes[0]))(*axes[0]), SECTION_ORDER[axes[1]]


def _axes_rows(table, max_positions):
    return table.data_ptr(), table.shape[0] if max_positions is None else int(max_positions)


def _qknorm_shape(q, k):
    dev = _device(q)
    if q.dim() != 4 or (k is not None and (not isinstance(k, torch.Tensor) or k.dim() != 4)):
        raise ValueError("q must be [B, H, S, D] and k [B, H_kv, S, D]")
    B, H, S, D = q.shape
    Hkv = 0 if k is None else k.shape[1]
    qs = _rows(q, "q", (B, H, S, D), q.dtype, dev)
    ks = [0, 0, 0] if k is None else _rows(k, "k", (B, Hkv, S, D), q.dtype, dev)
    return dev, (B, H, Hkv, S, D), qs, ks


def attnfuse_qknorm_rope(q, k=None, q_weight=None, k_weight=None, *, eps=1e-6, rope="neox", theta=10000.0, positions=None,
                         max_positions=None, out_q=None, out_k=None, rope_table=None, sections=None,
                         section_order="blocks", frequencies="shared", norm=True):
    """Qr, Kr: the rows of q and k over their root mean square, times the weights, rotated at their positions (0..S-1, or
    ``positions`` int32 [B, S], all below ``max_positions``: a row at another one comes out as NaN); see
    attnfuse_qknorm_rope in include/attnfuse_llm.h.  q and k may be slices whose rows lie apart; Qr and Kr are
    contiguous.

    With ``sections``, ``positions`` is int32 [axes, B, S]: a row has one on each of up to four axes (time, height, width),
    and sections[a] of its D / 2 pairs turn by axis a, in "blocks" or dealt out in "turns", with the "shared" frequencies
    theta^(-2i/D) or a ladder of each axis's "own"; norm=False is then the rotation alone.  See attnfuse_qknorm_axes."""
    if sections is not None or not norm:
        return _axes_fwd(q, k, q_weight, k_weight, eps, rope, theta, positions, max_positions, out_q, out_k, rope_table,
                         sections, section_order, frequencies, norm)
    if _native is not None:
        r = _native.qknorm(q, k, q_weight, k_weight, out_q, out_k, positions, rope_table, _TABLES, eps, ROPE.get(rope, -1),
                           theta, max_positions)
        if r is not None:
            return _result(r, "attnfuse_qknorm_rope")
    dev, (B, H, Hkv, S, D), qs, ks = _qknorm_shape(q, k)
    wt = _norm_weights(q_weight, k_weight, D, q.dtype, dev)
    out_q = _opt(out_q, "out_q", (B, H, S, D), q.dtype, dev)
    if k is not None:
        out_k = _opt(out_k, "out_k", (B, Hkv, S, D), q.dtype, dev)
    elif out_k is not None or k_weight is not None:
        raise ValueError("out_k and k_weight need k")
    tp, tr = _tab(tab := _position_table(rope, theta, D, S, dev, positions, (B, S), max_positions, rope_table))
    with torch.cuda.device(dev):
        code = _lib.load().attnfuse_qknorm_rope(_ptr(q), _ptr(k), _ptr(out_q), _ptr(out_k), _ptr(q_weight), _ptr(k_weight), wt,
                                                float(eps), *qs, *ks, B, H, Hkv, S, D, DTYPE[q.dtype], ROPE[rope],
                                                float(theta), tp, tr, _ptr(positions), _stream())
    _check(code, "attnfuse_qknorm_rope")
    return out_q, out_k


def _axes_fwd(q, k, q_weight, k_weight, eps, rope, theta, positions, max_positions, out_q, out_k, rope_table, sections,
              section_order, frequencies, norm):
    if _native is not None:
        r = _native.axes(q, k, q_weight, k_weight, out_q, out_k, positions, rope_table, _TABLES, eps, ROPE.get(rope, -1),
                         theta, max_positions, int(bool(norm)), sections, section_order, SECTION_ORDER.get(section_order, -1),
                         FREQUENCIES.get(frequencies, -1))
        if r is not None:
            return _result(r, "attnfuse_qknorm_axes")
    dev = _device(q)
    axes = _axes(sections, section_order, frequencies, norm, rope, q.shape[-1], positions)
    tab = _axes_table(axes, frequencies, rope, theta, q.shape[-1], dev, max_positions, rope_table)
    dev, (B, H, Hkv, S, D), qs, ks = _qknorm_shape(q, k)
    wt = _axes_weights(q_weight, k_weight, norm, D, q.dtype, dev)
    _need(positions, "positions", (len(axes[0]), B, S), torch.int32, dev)
    out_q = _opt(out_q, "out_q", (B, H, S, D), q.dtype, dev)
    if k is not None:
        out_k = _opt(out_k, "out_k", (B, Hkv, S, D), q.dtype, dev)
    elif out_k is not None or k_weight is not None:
        raise ValueError("out_k and k_weight need k")
    with torch.cuda.device(dev):
        code = _lib.load().attnfuse_qknorm_axes(_ptr(q), _ptr(k), _ptr(out_q), _ptr(out_k), _ptr(q_weight), _ptr(k_weight), wt,
                                                int(bool(norm)), float(eps), *qs, *ks, B, H, Hkv, S, D, DTYPE[q.dtype],
                                                ROPE[rope], float(theta), *_axes_rows(tab, max_positions), _ptr(positions),
                                                *_axes_args(axes), _stream())
    _check(code, "attnfuse_qknorm_axes")
    return out_q, out_k


def _axes_weights(q_weight, k_weight, norm, D, dtype, dev):
    if not norm and (q_weight is not None or k_weight is not None):
        raise ValueError("norm=False takes no weights")
    return _norm_weights(q_weight, k_weight, D, dtype, dev)


def attnfuse_qknorm_rope_bwd_workspace_bytes(B, H, H_kv, S, D, dtype=torch.bfloat16):
    return _lib.load().attnfuse_qknorm_rope_bwd_workspace_bytes(B, H, H_kv, S, D, DTYPE[dtype])


def attnfuse_qknorm_rope_bwd(q, k, dqr, dkr, q_weight=None, k_weight=None, *, eps=1e-6, rope="neox", theta=10000.0,
                             positions=None, max_positions=None, weight_grads=True, dq=None, dk=None, workspace=None,
                             rope_table=None, sections=None, section_order="blocks", frequencies="shared", norm=True):
    """dQ, dK, dq_weight, dk_weight of attnfuse_qknorm_rope (k and dkr None: of q alone; without ``weight_grads`` the last
    two are None); see attnfuse_qknorm_rope_bwd.  dQ and dK lie in memory as q and k do, without gaps.  With norm=False q
    and k are not used (None will do), there are no weights, and dQ and dK are contiguous where none are given."""
    if sections is not None or not norm:
        return _axes_bwd(q, k, dqr, dkr, q_weight, k_weight, eps, rope, theta, positions, max_positions, weight_grads, dq, dk,
                         workspace, rope_table, sections, section_order, frequencies, norm)
    if _native is not None:
        r = _native.qknorm_bwd(q, k, dqr, dkr, q_weight, k_weight, dq, dk, workspace, positions, rope_table, _TABLES, eps,
                               ROPE.get(rope, -1), theta, max_positions, int(bool(weight_grads)))
        if r is not None:
            return _result(r, "attnfuse_qknorm_rope_bwd")
    dev, (B, H, Hkv, S, D), qs, ks = _qknorm_shape(q, k)
    wt = _norm_weights(q_weight, k_weight, D, q.dtype, dev)
    _need(dqr, "dqr", (B, H, S, D), q.dtype, dev)
    dq = torch.empty_like(q) if dq is None else dq
    dqs, dks, dwq, dwk, wbytes = _rows(dq, "dq", q.shape, q.dtype, dev), [0, 0, 0], None, None, 0
    if k is not None:
        _need(dkr, "dkr", (B, Hkv, S, D), q.dtype, dev)
        dk = torch.empty_like(k) if dk is None else dk
        dks = _rows(dk, "dk", k.shape, q.dtype, dev)
    elif dkr is not None or dk is not None or k_weight is not None:
        raise ValueError("dkr, dk and k_weight need k")
    if weight_grads:
        t = torch.float32 if wt else torch.bfloat16
        dwq = torch.empty(D, device=dev, dtype=t)
        dwk = None if k is None else torch.empty(D, device=dev, dtype=t)
        workspace, wbytes = _workspace(workspace, attnfuse_qknorm_rope_bwd_workspace_bytes(B, H, Hkv, S, D, q.dtype), dev)
    tp, tr = _tab(tab := _position_table(rope, theta, D, S, dev, positions, (B, S), max_positions, rope_table))
    with torch.cuda.device(dev):
        code = _lib.load().attnfuse_qknorm_rope_bwd(
            _ptr(q), _ptr(k), _ptr(dqr), _ptr(dkr), _ptr(dq), _ptr(dk), _ptr(dwq), _ptr(dwk), _ptr(q_weight), _ptr(k_weight),
            wt, float(eps), *qs, *ks, *dqs, *dks, _ptr(workspace), wbytes, B, H, Hkv, S, D, DTYPE[q.dtype], ROPE[rope],
            float(theta), tp, tr, _ptr(positions), _stream())
    _check(code, "attnfuse_qknorm_rope_bwd")
    return dq, dk, dwq, dwk


def _axes_bwd(q, k, dqr, dkr, q_weight, k_weight, eps, rope, theta, positions, max_positions, weight_grads, dq, dk, workspace,
              rope_table, sections, section_order, frequencies, norm):
    if not norm:
        q = k = None
        weight_grads = False
    if _native is not None:
        r = _native.axes_bwd(q, k, dqr, dkr, q_weight, k_weight, dq, dk, workspace, positions, rope_table, _TABLES, eps,
                             ROPE.get(rope, -1), theta, max_positions, int(bool(weight_grads)), int(bool(norm)), sections,
                             section_order, SECTION_ORDER.get(section_order, -1), FREQUENCIES.get(frequencies, -1))
        if r is not None:
            return _result(r, "attnfuse_qknorm_axes_bwd")
    dev = _device(dqr)
    if dqr.dim() != 4 or (dkr is not None and (not isinstance(dkr, torch.Tensor) or dkr.dim() != 4)):
        raise ValueError("dqr must be [B, H, S, D] and dkr [B, H_kv, S, D]")
    axes = _axes(sections, section_order, frequencies, norm, rope, dqr.shape[-1], positions)
    tab = _axes_table(axes, frequencies, rope, theta, dqr.shape[-1], dev, max_positions, rope_table)
    if norm:
        dev, (B, H, Hkv, S, D), qs, ks = _qknorm_shape(q, k)
        if k is None and (dkr is not None or dk is not None or k_weight is not None):
            raise ValueError("dkr, dk and k_weight need k")
        if k is not None and dkr is None:
            raise ValueError("k needs dkr")
        dtype = q.dtype
    else:
        (B, H, S, D), Hkv, dtype, qs, ks = dqr.shape, 0 if dkr is None else dkr.shape[1], dqr.dtype, [0] * 3, [0] * 3
        if dkr is None and dk is not None:
            raise ValueError("dk needs dkr")
    wt = _axes_weights(q_weight, k_weight, norm, D, dtype, dev)
    _need(dqr, "dqr", (B, H, S, D), dtype, dev)
    _need(positions, "positions", (len(axes[0]), B, S), torch.int32, dev)
    dq = torch.empty_like(q if norm else dqr) if dq is None else dq
    dqs, dks, dwq, dwk, wbytes = _rows(dq, "dq", (B, H, S, D), dtype, dev), [0, 0, 0], None, None, 0
    if dkr is not None:
        _need(dkr, "dkr", (B, Hkv, S, D), dtype, dev)
        dk = torch.empty_like(k if norm else dkr) if dk is None else dk
        dks = _rows(dk, "dk", (B, Hkv, S, D), dtype, dev)
    if weight_grads:
        t = torch.float32 if wt else torch.bfloat16
        dwq = torch.empty(D, device=dev, dtype=t)
        dwk = None if k is None else torch.empty(D, device=dev, dtype=t)
        workspace, wbytes = _workspace(workspace, attnfuse_qknorm_rope_bwd_workspace_bytes(B, H, Hkv, S, D, dtype), dev)
    with torch.cuda.device(dev):
        code = _lib.load().attnfuse_qknorm_axes_bwd(
            _ptr(q), _ptr(k), _ptr(dqr), _ptr(dkr), _ptr(dq), _ptr(dk), _ptr(dwq), _ptr(dwk), _ptr(q_weight), _ptr(k_weight),
            wt, int(bool(norm)), float(eps), *qs, *ks, *dqs, *dks, _ptr(workspace), wbytes, B, H, Hkv, S, D, DTYPE[dtype],
            ROPE[rope], float(theta), *_axes_rows(tab, max_positions), _ptr(positions), *_axes_args(axes), _stream())
    _check(code, "attnfuse_qknorm_axes_bwd")
    return dq, dk, dwq, dwk


def _pages(k_cache, v_cache, Hkv, D, dtype, device):
    """(pages, page size, strides of both) of a paged cache [num_pages, H_kv, page_size, D]."""
    if not isinstance(k_cache, torch.Tensor) or k_cache.dim() != 4:
        raise ValueError("the caches must be [num_pages, H_kv, page_size, D]")
    shape = (k_cache.shape[0], Hkv, k_cache.shape[2], D)
    return shape[0], shape[2], (_rows(k_cache, "k_cache", shape, dtype, device),
                                _rows(v_cache, "v_cache", shape, dtype, device))


def attnfuse_qknorm_rope_append(q, k, v, k_cache, v_cache, slots, q_weight=None, k_weight=None, *, norm=True, eps=1e-6,
                                rope="neox", theta=10000.0, positions=None, max_positions=None, out_q=None,
                                rope_table=None, sections=None, section_order="blocks", frequencies="shared"):
    """Qr [T, H, D]: the queries of T new tokens, normed (unless ``norm`` is False) and rotated at ``positions`` (int32
    [T], all below ``max_positions``, or NaN); their keys, likewise, and values are written to the pages [num_pages, H_kv,
    page_size, D] at ``slots`` (int64 [T]: page * page_size + place; -1: nowhere); see attnfuse_qknorm_rope_append in
    include/attnfuse_llm.h.  q, k, v and the pages may lie apart (a fused projection's slices, pages [num_pages, page_size,
    H_kv, D] transposed).  With ``sections`` the positions are int32 [axes, T], as in attnfuse_qknorm_rope."""
    if sections is not None:
        return _axes_append(q, k, v, k_cache, v_cache, slots, q_weight, k_weight, norm, eps, rope, theta, positions,
                            max_positions, out_q, rope_table, sections, section_order, frequencies)
    if _native is not None:
        r = _native.append(q, k, v, k_cache, v_cache, slots, q_weight, k_weight, out_q, positions, rope_table, _TABLES,
                           int(bool(norm)), eps, ROPE.get(rope, -1), theta, max_positions)
        if r is not None:
            return _result(r, "attnfuse_qknorm_rope_append")[0]
    dev = _device(q)
    if q.dim() != 3 or not isinstance(k, torch.Tensor) or k.dim() != 3:
        raise ValueError("q must be [T, H, D] and k/v [T, H_kv, D]")
    T, H, D = q.shape
    Hkv = k.shape[1]
    qs = _rows(q, "q", (T, H, D), q.dtype, dev)
    ks, vs = _rows(k, "k", (T, Hkv, D), q.dtype, dev), _rows(v, "v", (T, Hkv, D), q.dtype, dev)
    wt = _norm_weights(q_weight, k_weight, D, q.dtype, dev)
    pages, page, (kps, vps) = _pages(k_cache, v_cache, Hkv, D, q.dtype, dev)
    _need(slots, "slots", (T,), torch.int64, dev)
    out_q = _opt(out_q, "out_q", (T, H, D), q.dtype, dev)
    if ROPE[rope] != ROPE["none"] and positions is None:
        raise ValueError("positions are needed with RoPE")
    tp, tr = _tab(tab := _position_table(rope, theta, D, 1, dev, positions, (T,), max_positions, rope_table))
    with torch.cuda.device(dev):
        code = _lib.load().attnfuse_qknorm_rope_append(
            _ptr(q), _ptr(k), _ptr(v), _ptr(out_q), _ptr(k_cache), _ptr(v_cache), _ptr(slots), _ptr(q_weight), _ptr(k_weight),
            wt, int(bool(norm)), float(eps), *qs, *ks, *vs, *kps, *vps, T, H, Hkv, D, pages, page, DTYPE[q.dtype],
            ROPE[rope], float(theta), tp, tr, _ptr(positions), _stream())
    _check(code, "attnfuse_qknorm_rope_append")
    return out_q


def _axes_append(q, k, v, k_cache, v_cache, slots, q_weight, k_weight, norm, eps, rope, theta, positions, max_positions, out_q,
                 rope_table, sections, section_order, frequencies):
    if _native is not None:
        r = _native.axes_append(q, k, v, k_cache, v_cache, slots, q_weight, k_weight, out_q, positions, rope_table, _TABLES,
                                eps, ROPE.get(rope, -1), theta, max_positions, int(bool(norm)), sections, section_order,
                                SECTION_ORDER.get(section_order, -1), FREQUENCIES.get(frequencies, -1))
        if r is not None:
            return _result(r, "attnfuse_qknorm_axes_append")[0]
    dev = _device(q)
    axes = _axes(sections, section_order, frequencies, norm, rope, q.shape[-1], positions)
    tab = _axes_table(axes, frequencies, rope, theta, q.shape[-1], dev, max_positions, rope_table)
    if q.dim() != 3 or not isinstance(k, torch.Tensor) or k.dim() != 3:
        raise ValueError("q must be [T, H, D] and k/v [T, H_kv, D]")
    T, H, D = q.shape
    Hkv = k.shape[1]
    qs = _rows(q, "q", (T, H, D), q.dtype, dev)
    ks, vs = _rows(k, "k", (T, Hkv, D), q.dtype, dev), _rows(v, "v", (T, Hkv, D), q.dtype, dev)
    wt = _axes_weights(q_weight, k_weight, norm, D, q.dtype, dev)
    pages, page, (kps, vps) = _pages(k_cache, v_cache, Hkv, D, q.dtype, dev)
    _need(slots, "slots", (T,), torch.int64, dev)
    _need(positions, "positions", (len(axes[0]), T), torch.int32, dev)
    out_q = _opt(out_q, "out_q", (T, H, D), q.dtype, dev)
    with torch.cuda.device(dev):
        code = _lib.load().attnfuse_qknorm_axes_append(
            _ptr(q), _ptr(k), _ptr(v), _ptr(out_q), _ptr(k_cache), _ptr(v_cache), _ptr(slots), _ptr(q_weight), _ptr(k_weight),
            wt, int(bool(norm)), float(eps), *qs, *ks, *vs, *kps, *vps, T, H, Hkv, D, pages, page, DTYPE[q.dtype],
            ROPE[rope], float(theta), *_axes_rows(tab, max_positions), _ptr(positions), *_axes_args(axes), _stream())
    _check(code, "attnfuse_qknorm_axes_append")
    return out_q


def attnfuse_decode_paged_workspace_bytes(B, H, H_kv, S_kv, D, window=0, sinks=0):
    return _lib.load().attnfuse_decode_paged_workspace_bytes(B, H, H_kv, S_kv, D, _count(window), _count(sinks))


def _need_sinks(sinks, mask, window, alibi_slopes):
    """(window, sinks): sinks belong to a sliding window, without ALiBi."""
    if sinks < 0 or mask != "sliding_window" or not window or window < 1:
        raise ValueError("sinks (>= 1) need mask='sliding_window' and a window")
    if alibi_slopes is not None:
        raise ValueError("sinks do not go with ALiBi slopes")
    return _count(window), _count(sinks)


def _fwd_sinks(q, k, v, rope, theta, mask, window, alibi_slopes, scale, out, lse, rope_table, sinks):
    window, sinks = _need_sinks(sinks, mask, window, alibi_slopes)
    if _native is not None:
        r = _native.fwd_sinks(q, k, v, out, lse, rope_table, _TABLES, ROPE.get(rope, -1), theta, window, sinks, scale)
        if r is not None:
            return _result(r, "attnfuse_fwd_sinks")
    dev = _device(q)
    B, H, Hkv, S, D = _shape(q, k)
    _inputs(q, k, v, dev)
    out = _opt(out, "out", q.shape, q.dtype, dev)
    lse = _opt(lse, "lse", (B, H, S), torch.float32, dev)
    r, th, _, w, sc = _variant(rope, theta, mask, window, None, scale, D)
    tp, tr = _tab(tab := _table(rope, theta, D, S, dev, rope_table))
    nbytes = _lib.load().attnfuse_fwd_sinks_workspace_bytes(B, Hkv, S, D, DTYPE[q.dtype], r)
    ws = torch.empty(nbytes, device=dev, dtype=torch.uint8) if nbytes else None
    with torch.cuda.device(dev):
        code = _lib.load().attnfuse_fwd_sinks(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), _ptr(ws), nbytes, B, H, Hkv, S,
                                              D, DTYPE[q.dtype], r, th, tp, tr, w, sinks, sc, _stream())
    _check(code, "attnfuse_fwd_sinks")
    return out, lse


def attnfuse_bwd_sinks_workspace_bytes(B, H, H_kv, S, D, rope, window, sinks):
    return _lib.load().attnfuse_bwd_sinks_workspace_bytes(B, H, H_kv, S, D, ROPE[rope], _count(window), _count(sinks))


def _bwd_sinks(q, k, v, o, do, lse, rope, theta, mask, window, alibi_slopes, scale, dq, dk, dv, workspace, rope_table, sinks):
    window, sinks = _need_sinks(sinks, mask, window, alibi_slopes)
    if _native is not None:
        r = _native.bwd_sinks(q, k, v, o, do, lse, dq, dk, dv, workspace, rope_table, _TABLES, ROPE.get(rope, -1), theta,
                              window, sinks, scale)
        if r is not None:
            return _result(r, "attnfuse_bwd_sinks")
    dev = _device(q)
    B, H, Hkv, S, D = _shape(q, k)
    _bwd_inputs(q, k, v, o, do, lse, dev, lse_needed=True)
    dq, dk, dv = _grads(q, k, dq, dk, dv, dev)
    r, th, _, w, sc = _variant(rope, theta, mask, window, None, scale, D)
    workspace, wbytes = _workspace(workspace, attnfuse_bwd_sinks_workspace_bytes(B, H, Hkv, S, D, rope, w, sinks), dev)
    tp, tr = _tab(tab := _table(rope, theta, D, S, dev, rope_table))
    with torch.cuda.device(dev):
        code = _lib.load().attnfuse_bwd_sinks(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(do), _ptr(lse), _ptr(dq), _ptr(dk),
                                              _ptr(dv), _ptr(workspace), wbytes, B, H, Hkv, S, D, DTYPE[q.dtype], r, th, tp,
                                              tr, w, sinks, sc, _stream())
    _check(code, "attnfuse_bwd_sinks")
    return dq, dk, dv


def _decode_sinks(q, k_cache, v_cache, cache_lens, rope, theta, mask, window, alibi_slopes, scale, out, lse, workspace,
                  rope_table, sinks):
    window, sinks = _need_sinks(sinks, mask, window, alibi_slopes)
    if _native is not None:
        r = _native.decode_sinks(q, k_cache, v_cache, cache_lens, out, lse, workspace, rope_table, _TABLES,
                                 ROPE.get(rope, -1), theta, window, sinks, scale)
        if r is not None:
            return _result(r, "attnfuse_decode_sinks")
    dev, (B, H, Hkv, S_kv, D), out, lse = _decode_args(q, k_cache, v_cache, cache_lens, out, lse)
    if q.dtype != torch.bfloat16:
        raise ValueError("decode with sinks takes bf16 tensors")
    nbytes = attnfuse_decode_paged_workspace_bytes(B, H, Hkv, S_kv, D, window, sinks)
    workspace, wbytes = _workspace(workspace, nbytes, dev)
    r, th, _, w, sc = _variant(rope, theta, mask, window, None, scale, D)
    tp, tr = _tab(tab := _table(rope, theta, D, S_kv, dev, rope_table))
    with torch.cuda.device(dev):
        code = _lib.load().attnfuse_decode_sinks(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(cache_lens), _ptr(out),
                                                 _ptr(lse), _ptr(workspace), wbytes, B, H, Hkv, S_kv, D, r, th, tp, tr, w,
                                                 sinks, sc, _stream())
    _check(code, "attnfuse_decode_sinks")
    return out, lse


def attnfuse_decode_paged(q, k_cache, v_cache, block_table, cache_lens=None, *, rope="none", theta=10000.0, mask="causal",
                          window=None, sinks=0, alibi_slopes=None, scale=None, out=None, lse=None, workspace=None,
                          rope_table=None, prefix_table=None, prefix_len=None):
    """O [B,H,D], LSE [B,H] of one query per sequence against pages [num_pages, H_kv, page_size, D] of already-rotated
    keys and their values, key n of sequence b in page ``block_table[b, n // page_size]`` (int32 [B, max_pages]); see
    attnfuse_decode_paged in include/attnfuse_llm.h.  The pages may lie apart (pages [num_pages, page_size, H_kv, D]
    transposed).

    With ``prefix_table`` (int32 [prefix_pages]) every sequence sees, before its own keys, those of a prefix that the
    batch shares and that is read once for all of it: ``prefix_len`` keys (int32 [1] on the GPU; None: all) in those pages.
    The queries come rotated then (rope="none"), and there are no windows and no ALiBi; see attnfuse_fwd_paged."""
    if prefix_table is not None or prefix_len is not None:
        if rope != "none" or mask not in ("none", "causal") or window or sinks or alibi_slopes is not None or rope_table is not None:
            raise ValueError("a shared prefix goes with rotated queries (rope='none'), without windows, sinks and ALiBi")
        if prefix_table is None:
            raise ValueError("prefix_len needs prefix_table")
        return _fwd_paged(q, k_cache, v_cache, block_table, None, cache_lens, prefix_table, prefix_len, scale, out, lse, workspace)
    if sinks:
        window, sinks = _need_sinks(sinks, mask, window, alibi_slopes)
    if _native is not None:
        r = _native.decode_paged(q, k_cache, v_cache, block_table, cache_lens, out, lse, workspace, alibi_slopes, rope_table,
                                 _TABLES, ROPE.get(rope, -1), theta, MASK.get(mask, -1), window, sinks, scale)
        if r is not None:
            return _result(r, "attnfuse_decode_paged")
    dev = _device(q)
    if q.dim() != 3 or q.dtype != torch.bfloat16:
        raise ValueError("q must be a bf16 tensor [B, H, D]")
    if not isinstance(k_cache, torch.Tensor) or k_cache.dim() != 4:
        raise ValueError("the caches must be [num_pages, H_kv, page_size, D]")
    B, H, D = q.shape
    Hkv = k_cache.shape[1]
    _need(q, "q", (B, H, D), q.dtype, dev)
    pages, page, (kps, vps) = _pages(k_cache, v_cache, Hkv, D, q.dtype, dev)
    if not isinstance(block_table, torch.Tensor) or block_table.dim() != 2:
        raise ValueError("block_table must be an int32 tensor [B, max_pages]")
    S = block_table.shape[1] * page
    _need(block_table, "block_table", (B, block_table.shape[1]), torch.int32, dev)
    if cache_lens is not None:
        _need(cache_lens, "cache_lens", (B,), torch.int32, dev)
    out = _opt(out, "out", (B, H, D), q.dtype, dev)
    lse = _opt(lse, "lse", (B, H), torch.float32, dev)
    r, th, m, w, sc = _variant(rope, theta, mask, window, alibi_slopes, scale, D, H, dev)
    nbytes = attnfuse_decode_paged_workspace_bytes(B, H, Hkv, S, D, w if m == MASK["sliding_window"] else 0, sinks)
    workspace, wbytes = _workspace(workspace, nbytes, dev)
    tp, tr = _tab(tab := _table(rope, theta, D, S, dev, rope_table))
    with torch.cuda.device(dev):
        code = _lib.load().attnfuse_decode_paged(
            _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(block_table), _ptr(cache_lens), _ptr(out), _ptr(lse),
            _ptr(workspace), wbytes, *kps, *vps, B, H, Hkv, D, pages, page, block_table.shape[1], r, th, tp, tr, m, w, sinks,
            _ptr(alibi_slopes), sc, _stream())
    _check(code, "attnfuse_decode_paged")
    return out, lse


def attnfuse_fwd_paged_workspace_bytes(T, B, H, H_kv, D, own_keys, prefix_keys=0):
    return _lib.load().attnfuse_fwd_paged_workspace_bytes(T, B, H, H_kv, D, own_keys, prefix_keys)


def attnfuse_fwd_paged(q, k_cache, v_cache, block_table, q_starts, cache_lens=None, *, prefix_table=None, prefix_len=None,
                       scale=None, out=None, lse=None, workspace=None):
    """O [T,H,D], LSE [T,H] of several new tokens per sequence, queries q [T,H,D] already rotated, against pages as
    attnfuse_decode_paged takes them: tokens ``q_starts[b]`` .. ``q_starts[b + 1] - 1`` (int32 [B + 1]) are the last ones
    of sequence b's ``cache_lens[b]`` own keys and see those up to their own, after the prefix that the batch shares
    (``prefix_table`` int32 [prefix_pages], ``prefix_len`` int32 [1]), if any.  Rows of ``out`` and ``lse`` of tokens that no
    sequence has are left as they are.  See attnfuse_fwd_paged in include/attnfuse_llm.h."""
    if q_starts is None:
        raise ValueError("q_starts must be an int32 tensor [B + 1]")
    return _fwd_paged(q, k_cache, v_cache, block_table, q_starts, cache_lens, prefix_table, prefix_len, scale, out, lse, workspace)


def _fwd_paged(q, k_cache, v_cache, block_table, q_starts, cache_lens, prefix_table, prefix_len, scale, out, lse, workspace):
    if _native is not None:
        r = _native.fwd_paged(q, k_cache, v_cache, block_table, q_starts, cache_lens, prefix_table, prefix_len, out, lse,
                              workspace, scale)
        if r is not None:
            return _result(r, "attnfuse_fwd_paged")
    dev = _device(q)
    if q.dim() != 3 or q.dtype != torch.bfloat16:
        raise ValueError("q must be a bf16 tensor [T, H, D]")
    if not isinstance(k_cache, torch.Tensor) or k_cache.dim() != 4:
        raise ValueError("the caches must be [num_pages, H_kv, page_size, D]")
    T, H, D = q.shape
    Hkv = k_cache.shape[1]
    _need(q, "q", (T, H, D), q.dtype, dev)
    pages, page, (kps, vps) = _pages(k_cache, v_cache, Hkv, D, q.dtype, dev)
    if not isinstance(block_table, torch.Tensor) or block_table.dim() != 2:
        raise ValueError("block_table must be an int32 tensor [B, max_pages]")
    B, most = block_table.shape
    _need(block_table, "block_table", (B, most), torch.int32, dev)
    if q_starts is not None:
        _need(q_starts, "q_starts", (B + 1,), torch.int32, dev)
    elif B != T:
        raise ValueError(f"block_table must have {T} rows, one for each query (it has {B})")
    if cache_lens is not None:
        _need(cache_lens, "cache_lens", (B,), torch.int32, dev)
    ahead = 0
    if prefix_table is not None:
        if not isinstance(prefix_table, torch.Tensor) or prefix_table.dim() != 1 or prefix_table.shape[0] < 1:
            raise ValueError("prefix_table must be an int32 tensor [prefix_pages]")
        ahead = prefix_table.shape[0]
        _need(prefix_table, "prefix_table", (ahead,), torch.int32, dev)
        if prefix_len is not None:
            _need(prefix_len, "prefix_len", (1,), torch.int32, dev)
    elif prefix_len is not None:
        raise ValueError("prefix_len needs prefix_table")
    out = _opt(out, "out", (T, H, D), q.dtype, dev)
    lse = _opt(lse, "lse", (T, H), torch.float32, dev)
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    workspace, wbytes = _workspace(workspace, attnfuse_fwd_paged_workspace_bytes(T, B, H, Hkv, D, most * page, ahead * page), dev)
    with torch.cuda.device(dev):
        code = _lib.load().attnfuse_fwd_paged(
            _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(block_table), _ptr(q_starts), _ptr(cache_lens), _ptr(prefix_table),
            _ptr(prefix_len), _ptr(out), _ptr(lse), _ptr(workspace) if wbytes else None, wbytes, *kps, *vps, T, B, H, Hkv, D,
            pages, page, most, ahead, scale, _stream())
    _check(code, "attnfuse_fwd_paged")
    return out, lse


def attnfuse_strerror(code):
    return _lib.load().attnfuse_strerror(code).decode()


def attnfuse_version():
    return _lib.load().attnfuse_version()
