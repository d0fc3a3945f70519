"""Row operators of a decoder stack on torch tensors (span_qk_norm_rope, span_adapter_apply,
span_verify_drafts).  Argument marshalling only: types, shapes and devices are checked here,
sizes, strides and alignment by the library.

Tensors lie on one GPU; a call is enqueued on `stream`, by default that GPU's current one.
A workspace that is not given comes from torch's allocator, on the call's stream, and goes
back to it when the call has been enqueued, as torch's own temporaries do.
"""
from __future__ import annotations

import ctypes
import struct
from typing import Optional, Sequence

from ._lib import SPAN_BF16, SPAN_EINVAL, SPAN_F32, SpanError, _check, load, torch

SPAN_MAX_DRAFTS = 64

# span_qk_norm, span_adapter_call and span_verify_call (include/spanq.h) as packed records
_QK_REC = struct.Struct("<10Q8q5i2fi")
_ADAPTER_REC = struct.Struct("<10Q4q10i")
_VERIFY_REC = struct.Struct("<14Q4q4i")


def _bad(who: str, what: str):
    return SpanError(SPAN_EINVAL, f"{who}: {what}")


def _at(who: str, name: str, t, dtype, device, shape=None, dense: bool = True) -> int:
    """Address of a tensor argument, 0 for None."""
    if t is None:
        return 0
    if t.dtype != dtype or t.device != device:
        raise _bad(who, f"{name} must be {dtype} on {device}, not {t.dtype} on {t.device}")
    if shape is not None and t.shape != shape:
        raise _bad(who, f"{name} must have the shape {tuple(shape)}, not {tuple(t.shape)}")
    if dense and not t.is_contiguous():
        raise _bad(who, f"{name} must be contiguous")
    return t.data_ptr()


def _stream_of(stream, device) -> int:
    if stream is None:
        return torch.cuda.current_stream(device).cuda_stream
    return stream if isinstance(stream, int) else stream.cuda_stream


def _scratch(nbytes: int, stream, device):
    if stream is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device) if stream else torch.cuda.default_stream(device)
    with torch.cuda.stream(stream):  # memory freed there by earlier work on that stream, not on the current one
        return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _gpu(who: str, name: str, t):
    if torch is None or not isinstance(t, torch.Tensor) or t.device.type != "cuda":
        raise _bad(who, f"{name} must be a tensor on a GPU")
    return t.device


def _stride(who: str, name: str, t) -> int:
    """Row stride of a [rows][width] or [rows][heads][dim] tensor whose rows are dense."""
    st = t.stride()
    if (t.shape[-1] > 1 and st[-1] != 1) or (len(st) == 3 and t.shape[1] > 1 and st[1] != t.shape[2]):
        raise _bad(who, f"the elements of a row of {name} must follow one another")
    if t.shape[0] > 1:
        return st[0]
    width = t.shape[-1] * (t.shape[1] if len(st) == 3 else 1)
    return max(st[0], width)  # one row: its stride says nothing


def qk_norm_rope(q, k, v, q_gain, k_gain, eps: float, q_out, k_out, v_out, rows=None, positions=None,
                 rope_theta: float = 1e4, stream=None):
    """Head norms of q and k [rows, heads, dim] (a gain of None: no norm), rotation at `positions`
    (None: none), and the rows' way to the outputs at `rows` (None: in order); v is copied
    (span_qk_norm_rope).  Any of q, k, v may be None with its output."""
    who = "qk_norm_rope"
    lead = next((t for t in (q, k, v) if t is not None), None)
    if lead is None:
        raise _bad(who, "needs at least one of q, k, v")
    dev, dtype = _gpu(who, "q, k, v", lead), lead.dtype
    if dtype not in (torch.bfloat16, torch.float32):
        raise _bad(who, "rows must be bfloat16 or float32")
    n, out_rows, dim = lead.shape[0], None, lead.shape[-1]
    at, strides, heads = [], [], {}
    for name, t, o, kind in (("q", q, q_out, "q"), ("k", k, k_out, "kv"), ("v", v, v_out, "kv")):
        if (t is None) != (o is None):
            raise _bad(who, f"{name} and {name}_out go together")
        if t is None:
            at.append((0, 0))
            strides.append((0, 0))
            continue
        if t.dim() != 3 or o.dim() != 3 or t.shape[0] != n or t.shape[1:] != o.shape[1:] or t.shape[2] != dim:
            raise _bad(who, f"{name} and {name}_out must be [rows, heads, dim] with the same heads and dim")
        if heads.setdefault(kind, t.shape[1]) != t.shape[1]:
            raise _bad(who, "k and v must have the same heads")
        if out_rows is None:
            out_rows = o.shape[0]
        elif out_rows != o.shape[0]:
            raise _bad(who, "the outputs must have the same rows")
        at.append((_at(who, name, t, dtype, dev, dense=False), _at(who, name + "_out", o, dtype, dev, dense=False)))
        strides.append((_stride(who, name, t), _stride(who, name + "_out", o)))
    rec = _QK_REC.pack(
        at[0][0], at[1][0], at[2][0], at[0][1], at[1][1], at[2][1],
        _at(who, "q_gain", q_gain, dtype, dev, (dim,)), _at(who, "k_gain", k_gain, dtype, dev, (dim,)),
        _at(who, "rows", rows, torch.int32, dev, (n,)), _at(who, "positions", positions, torch.int32, dev, (n,)),
        strides[0][0], strides[1][0], strides[2][0], strides[0][1], strides[1][1], strides[2][1],
        n, out_rows, heads.get("q", 0), heads.get("kv", 0), dim, SPAN_BF16 if dtype == torch.bfloat16 else SPAN_F32,
        dev.index, eps, rope_theta, 0)
    _check(load().span_qk_norm_rope(rec, _stream_of(stream, dev)))


def _workspace(entry, rec: bytes) -> int:
    n = ctypes.c_size_t()
    _check(entry(rec, ctypes.byref(n)))
    return n.value


def _adapter_rec(x, base, out, ids, a, b, scale, ranks, ws, ws_bytes, strides, n, sizes, parts, index) -> bytes:
    cols = list(parts) + [0] * (4 - len(parts))
    return _ADAPTER_REC.pack(x, base, out, ids, a, b, scale, ranks, ws, ws_bytes, *strides, n, *sizes, len(parts),
                             *cols, index, 0)


def adapter_workspace(n_rows: int, in_features: int, max_rank: int, parts: Sequence[int]) -> int:
    """Bytes of workspace of an adapter_apply call (span_adapter_workspace)."""
    if not 1 <= len(parts) <= 4:
        raise _bad("adapter_workspace", "one to four parts")
    rec = _adapter_rec(0, 0, 0, 0, 0, 0, 0, 0, 0, 0, (0, 0, 0), n_rows, (in_features, 0, max_rank), parts, 0)
    return _workspace(load().span_adapter_workspace, rec)


def adapter_apply(x, base, ids, a, b, scale, out, parts: Optional[Sequence[int]] = None, ranks=None, workspace=None,
                  stream=None):
    """out = base + scale[id] (x a[id]^T) b[id]^T for each row's own adapter id (none outside
    [0, n)) (span_adapter_apply).  x [rows, in], base and out [rows, cols] (may be one tensor), ids int32
    [rows], a [n, parts, rank, in], b [n, cols, rank], scale float32 [n] or None, ranks int32 [n] or None;
    parts: the columns of each part, by default one part."""
    who = "adapter_apply"
    dev = _gpu(who, "x", x)
    bf16 = torch.bfloat16
    if x.dim() != 2 or out.dim() != 2 or a.dim() != 4 or b.dim() != 3:
        raise _bad(who, "x and out must have two dimensions, a four, b three")
    n, width = x.shape
    cols = out.shape[1]
    parts = (cols,) if parts is None else parts
    count, n_parts, rank, _ = a.shape
    if n_parts != len(parts) or sum(parts) != cols or not 1 <= n_parts <= 4:
        raise _bad(who, "parts must be one to four column counts, as many as a has, adding up to out's columns")
    at = (_at(who, "x", x, bf16, dev, dense=False), _at(who, "base", base, bf16, dev, (n, cols), dense=False),
          _at(who, "out", out, bf16, dev, (n, cols), dense=False), _at(who, "ids", ids, torch.int32, dev, (n,)),
          _at(who, "a", a, bf16, dev, (count, n_parts, rank, width)), _at(who, "b", b, bf16, dev, (count, cols, rank)),
          _at(who, "scale", scale, torch.float32, dev, (count,)), _at(who, "ranks", ranks, torch.int32, dev, (count,)))
    strides = (_stride(who, "x", x), _stride(who, "base", base), _stride(who, "out", out))
    sizes = (width, count, rank)
    if workspace is None:
        need = _workspace(load().span_adapter_workspace,
                          _adapter_rec(*at, 0, 0, strides, n, sizes, parts, dev.index))
        workspace = _scratch(need, stream, dev)
    ws, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _check(load().span_adapter_apply(_adapter_rec(*at, ws, ws_bytes, strides, n, sizes, parts, dev.index),
                                     _stream_of(stream, dev)))


def verify_workspace(n_requests: int, max_drafts: int, vocab: int) -> int:
    """Bytes of workspace of a verify_drafts call (span_verify_workspace)."""
    rec = _VERIFY_REC.pack(*[0] * 18, n_requests, max_drafts, vocab, 0)
    return _workspace(load().span_verify_workspace, rec)


def verify_drafts(target_logits, drafts, u_accept, u_sample, temperature, accepted, tokens, draft_logits=None,
                  n_drafts=None, row0=None, draft_row0=None, logprobs=None, workspace=None, stream=None):
    """Keeps each request's drafts as far as the target's probabilities allow and draws the next token
    (span_verify_drafts).  target_logits float32 [rows, vocab]; drafts int32 and u_accept float32 [n, k]
    (None for k = 0: a token is sampled); u_sample and temperature float32 [n] (None: 1; 0: greedy);
    accepted int32 [n], tokens int32 and logprobs float32 [n, k + 1] are written; draft_logits float32 [draft
    rows, vocab] or None; n_drafts, row0, draft_row0 int32 [n] or None."""
    who = "verify_drafts"
    dev = _gpu(who, "target_logits", target_logits)
    f32, i32 = torch.float32, torch.int32
    if target_logits.dim() != 2 or tokens.dim() != 2 or (draft_logits is not None and draft_logits.dim() != 2):
        raise _bad(who, "logits and tokens must have two dimensions")
    n, k = tokens.shape[0], tokens.shape[1] - 1
    vocab = target_logits.shape[1]
    if k > 0 and (drafts is None or u_accept is None):
        raise _bad(who, "drafts need their tokens and random numbers")
    if draft_logits is not None and draft_logits.shape[1] != vocab:
        raise _bad(who, "draft_logits must have the target's vocabulary")
    at = (_at(who, "target_logits", target_logits, f32, dev, dense=False),
          _at(who, "draft_logits", draft_logits, f32, dev, dense=False),
          _at(who, "row0", row0, i32, dev, (n,)), _at(who, "draft_row0", draft_row0, i32, dev, (n,)),
          _at(who, "drafts", drafts, i32, dev, (n, k)), _at(who, "n_drafts", n_drafts, i32, dev, (n,)),
          _at(who, "u_accept", u_accept, f32, dev, (n, k)), _at(who, "u_sample", u_sample, f32, dev, (n,)),
          _at(who, "temperature", temperature, f32, dev, (n,)), _at(who, "accepted", accepted, i32, dev, (n,)),
          _at(who, "tokens", tokens, i32, dev), _at(who, "logprobs", logprobs, f32, dev, (n, k + 1)))
    strides = (_stride(who, "target_logits", target_logits) if target_logits.shape[0] else vocab,
               _stride(who, "draft_logits", draft_logits) if draft_logits is not None and draft_logits.shape[0] else vocab)
    rest = (target_logits.shape[0], 0 if draft_logits is None else draft_logits.shape[0], n, k, vocab, dev.index)
    if workspace is None:
        workspace = _scratch(verify_workspace(n, k, vocab), stream, dev)
    ws, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _check(load().span_verify_drafts(_VERIFY_REC.pack(*at, ws, ws_bytes, *strides, *rest), _stream_of(stream, dev)))
