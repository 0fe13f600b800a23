"""Thin Python binding of libdamp's serving operators (include/damp_serving.h):
linear attention with one decay a head, the verification of drafted tokens,
and the slots of a state pool as the pages of its cache.

Argument marshalling only, as in damp.py. Strides are the exception to its
contiguous operands: q, k and v may keep any distance between tokens (a slice
of a fused projection's output), and g may be one decay a head ([HV]).

What a call allocates by itself, outputs and scratch, is allocated (and cleared)
on the stream that it runs on, so that the memory is taken and given back in
that stream's order.
"""
from __future__ import annotations

import ctypes

import torch

from . import damp as D
from .damp import Pool, _at, _check, _raw_stream

DAMP_SLOT_ZERO = -1

EXPORTS = ("damp_linear_update", "damp_linear_prefill_workspace_bytes", "damp_linear_prefill",
           "damp_verify_workspace_bytes", "damp_verify_drafts", "damp_slots_alloc",
           "damp_slots_retain", "damp_slots_release", "damp_slots_fork",
           "damp_slots_compact_workspace_bytes", "damp_slots_compact")

_lib = None


def lib() -> ctypes.CDLL:
    """libdamp.so with the serving operators' signatures (raises if it has not
    been built)."""
    global _lib
    if _lib is not None:
        return _lib
    L = D.lib()
    P, i32, i64, sz, f32, st = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t,
                                ctypes.c_float, ctypes.c_int)
    PP = ctypes.POINTER(D.damp_pool)
    operands = [i32, P, i64, P, i64, P, i64, P, i64, f32, P, i32]  # num_k_heads .. o_dtype
    sig = {
        "damp_linear_update": (st, [PP, i32, P, P, i32, *operands, P]),
        "damp_linear_prefill_workspace_bytes": (sz, [PP, i32, i32]),
        "damp_linear_prefill": (st, [PP, i32, P, P, i32, i64, i32, P, P, *operands, P, sz, P]),
        "damp_verify_workspace_bytes": (sz, [i32, i32]),
        "damp_verify_drafts": (st, [P, P, i32, P, P, P, i32, i32, i32, P, P, P, sz, P]),
        "damp_slots_alloc": (st, [P, i32, P, i32, P]),
        "damp_slots_retain": (st, [P, i32, P, i32, P]),
        "damp_slots_release": (st, [P, i32, P, i32, P]),
        "damp_slots_fork": (st, [PP, i32, P, P, i32, i32, P]),
        "damp_slots_compact_workspace_bytes": (sz, [PP]),
        "damp_slots_compact": (st, [PP, P, P, P, P, sz, P]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    _lib = L
    return L


def _new(make, shape, dtype, device, stream):
    """make(shape) - torch.empty or torch.zeros - in the order of the call's stream."""
    if stream is None:
        return make(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return make(shape, dtype=dtype, device=device)


def _ids(t, name: str, n=None) -> int:
    """The address of int32 device ids, [n] if n is given."""
    return _at(t, torch.int32, name, t.shape if n is None else (n,))


def _tokens(t, name: str, rows: int, heads: int, d: int):
    """(address, elements between tokens) of a [rows, heads, d] bf16 operand
    whose tokens are contiguous in themselves."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA (HIP) tensor")
    if t.dtype is not torch.bfloat16:
        raise ValueError(f"{name} must be torch.bfloat16, got {t.dtype}")
    if t.shape != (rows, heads, d):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {(rows, heads, d)}")
    if t.is_contiguous():
        return t.data_ptr(), heads * d
    s = t.stride()
    if s[2] != 1 or s[1] != d and heads != 1:
        raise ValueError(f"{name}: the heads of a token must be contiguous")
    return t.data_ptr(), s[0] if rows > 1 else heads * d


def _operands(pool: Pool, q, k, v, g, scale, o, stream):
    """The arguments num_k_heads .. o_dtype of both linear-attention calls, and o."""
    HV, dk, dv = pool.num_v_heads, pool.layout.d_k, pool.layout.d_v
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q must be a [tokens, HK, d_k] tensor")
    n, HK = q.shape[0], q.shape[1]
    if o is None:
        o = _new(torch.empty, (n, HV, dv), torch.float32, q.device, stream)
    if o.dtype is torch.float32:
        o_dt = D.DAMP_DT_FP32
    elif o.dtype is torch.bfloat16:
        o_dt = D.DAMP_DT_BF16
    else:
        raise ValueError("o must be float32 or bfloat16")
    if g.dim() == 1:
        gs, g_at = 0, _at(g, torch.float32, "g", (HV,))
    else:
        gs, g_at = HV, _at(g, torch.float32, "g", (n, HV))
    return [HK, *_tokens(q, "q", n, HK, dk), *_tokens(k, "k", n, HK, dk),
            *_tokens(v, "v", n, HV, dv), g_at, gs, float(scale), _at(o, o.dtype, "o", (n, HV, dv)),
            o_dt], o


# -------------------------------------------------------- linear attention

def damp_linear_update(pool: Pool, layer: int, slot_in, q, k, v, g, slot_out=None,
                       scale: float = 1.0, o=None, stream=None):
    """One token for each request (q, k [B, HK, d_k], v [B, HV, d_v], fp32 g
    [B, HV] or [HV]) from slot_in into slot_out (default: in place); returns
    o [B, HV, d_v]."""
    args, o = _operands(pool, q, k, v, g, scale, o, stream)
    B = q.shape[0]
    into = None if slot_out is None else _ids(slot_out, "slot_out", B)
    _check(lib().damp_linear_update(ctypes.byref(pool.desc), layer, _ids(slot_in, "slot_in", B),
                                    into, B, *args, _raw_stream(stream)))
    return o


def damp_linear_prefill_workspace_bytes(pool: Pool, B: int, max_len: int) -> int:
    return int(lib().damp_linear_prefill_workspace_bytes(ctypes.byref(pool.desc), B, max_len))


def damp_linear_prefill(pool: Pool, layer: int, slot_in, q, k, v, g, seq_start, seq_len,
                        max_len: int, slot_out=None, scale: float = 1.0, o=None, workspace=None,
                        stream=None):
    """Packed prompts (operands as damp_linear_update's, over the token axis;
    int32 seq_start and seq_len [B]); returns o [tokens, HV, d_v], of which
    only the requests' tokens are written. Without a workspace one is
    allocated for the call."""
    args, o = _operands(pool, q, k, v, g, scale, o, stream)
    _ids(slot_in, "slot_in")
    B = slot_in.numel()
    into = None if slot_out is None else _ids(slot_out, "slot_out", B)
    if workspace is None:
        workspace = _new(torch.empty, damp_linear_prefill_workspace_bytes(pool, B, max_len),
                         torch.uint8, q.device, stream)
    ws = _at(workspace, torch.uint8, "workspace", workspace.shape)
    _check(lib().damp_linear_prefill(ctypes.byref(pool.desc), layer, slot_in.data_ptr(), into, B,
                                     q.shape[0], max_len, _ids(seq_start, "seq_start", B),
                                     _ids(seq_len, "seq_len", B), *args, ws, workspace.numel(),
                                     _raw_stream(stream)))
    return o


# ---------------------------------------------------- drafted tokens

def damp_verify_workspace_bytes(B: int, V: int) -> int:
    return int(lib().damp_verify_workspace_bytes(B, V))


def damp_verify_drafts(p, q, tokens, u, lens=None, workspace=None, accepted=None, out=None,
                       stream=None):
    """The drafts that stand and the token after them: p [B, K + 1, V] and
    q [B, K, V] (fp32 or bf16), int32 tokens [B, K], fp32 u [B, K + 1], int32
    lens [B] or None; returns int32 (accepted [B], out [B, K + 1]). The
    workspace must be zero before its first call (one is allocated and cleared
    for the call if none is given)."""
    if not isinstance(p, torch.Tensor) or p.dim() != 3 or p.shape[1] < 1:
        raise ValueError("p must be a [B, K + 1, V] tensor")
    if p.dtype is torch.float32:
        dtype = D.DAMP_DT_FP32
    elif p.dtype is torch.bfloat16:
        dtype = D.DAMP_DT_BF16
    else:
        raise ValueError("p must be float32 or bfloat16")
    B, K, V = p.shape[0], p.shape[1] - 1, p.shape[2]
    if accepted is None:
        accepted = _new(torch.empty, B, torch.int32, p.device, stream)
    if out is None:
        out = _new(torch.empty, (B, K + 1), torch.int32, p.device, stream)
    if workspace is None:
        workspace = _new(torch.zeros, damp_verify_workspace_bytes(B, V), torch.uint8, p.device,
                         stream)
    ws = _at(workspace, torch.uint8, "workspace", workspace.shape)
    _check(lib().damp_verify_drafts(
        _at(p, p.dtype, "p", (B, K + 1, V)), _at(q, p.dtype, "q", (B, K, V)) if K else None, dtype,
        _at(tokens, torch.int32, "tokens", (B, K)) if K else None,
        None if lens is None else _ids(lens, "lens", B), _at(u, torch.float32, "u", (B, K + 1)), B,
        K, V, _ids(accepted, "accepted", B), _at(out, torch.int32, "out", (B, K + 1)), ws,
        workspace.numel(), _raw_stream(stream)))
    return accepted, out


# ------------------------------------------------------------------ slots

def damp_slots_alloc(refs, n: int, out=None, stream=None):
    """The n lowest free slots (int32 [n], -1 where none is left), each taken."""
    if out is None:
        out = _new(torch.empty, n, torch.int32, refs.device, stream)
    _check(lib().damp_slots_alloc(_ids(refs, "refs"), refs.numel(), _ids(out, "out", n), n,
                                  _raw_stream(stream)))
    return out


def damp_slots_retain(refs, slots, stream=None) -> None:
    _check(lib().damp_slots_retain(_ids(refs, "refs"), refs.numel(), _ids(slots, "slots"),
                                   slots.numel(), _raw_stream(stream)))


def damp_slots_release(refs, slots, stream=None) -> None:
    _check(lib().damp_slots_release(_ids(refs, "refs"), refs.numel(), _ids(slots, "slots"),
                                    slots.numel(), _raw_stream(stream)))


def damp_slots_fork(pool: Pool, src, dst, layer: int = -1, stream=None) -> None:
    """Copies slot src[i] into the slots dst[i] (int32 [n] and [n] or [n, fan])
    of one layer, or of all."""
    n = src.numel()
    if dst.dim() not in (1, 2) or dst.shape[0] != n:
        raise ValueError(f"dst has shape {tuple(dst.shape)}, expected ({n},) or ({n}, fan)")
    fan = 1 if dst.dim() == 1 else dst.shape[1]
    _check(lib().damp_slots_fork(ctypes.byref(pool.desc), layer, _ids(src, "src", n),
                                 _ids(dst, "dst"), n, fan, _raw_stream(stream)))


def damp_slots_compact_workspace_bytes(pool: Pool) -> int:
    return int(lib().damp_slots_compact_workspace_bytes(ctypes.byref(pool.desc)))


def damp_slots_compact(pool: Pool, refs, workspace=None, map_out=None, live=None, stream=None):
    """Moves the live slots down to 0 .. L - 1 in every layer, refs with them;
    returns int32 (map [num_slots], live [1])."""
    n = pool.num_slots
    dev = refs.device
    if map_out is None:
        map_out = _new(torch.empty, n, torch.int32, dev, stream)
    if live is None:
        live = _new(torch.empty, (), torch.int32, dev, stream)
    if workspace is None:
        workspace = _new(torch.empty, damp_slots_compact_workspace_bytes(pool), torch.uint8, dev,
                         stream)
    if live.numel() != 1:
        raise ValueError("live must hold one number")
    _check(lib().damp_slots_compact(ctypes.byref(pool.desc), _ids(refs, "refs", n),
                                    _ids(map_out, "map_out", n), _ids(live, "live"),
                                    _at(workspace, torch.uint8, "workspace", workspace.shape),
                                    workspace.numel(), _raw_stream(stream)))
    return map_out, live
