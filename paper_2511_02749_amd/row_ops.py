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
from functools import lru_cache
from typing import Optional, Sequence

from ._lib import SPAN_BF16, SPAN_EINVAL, SPAN_F32, SpanError, _check, load, torch

SPAN_MAX_DRAFTS = 64

# span_qk_norm, span_adapter_call and span_verify_call (include/spanq.h) as packed records
_QK_REC = struct.Struct("<10Q8q5i2fi")
_ADAPTER_REC = struct.Struct("<10Q4q10i")
_VERIFY_REC = struct.Struct("<14Q4q4i")


# the current stream's address: without a Stream object, if torch can
_raw_stream = getattr(getattr(torch, "_C", None), "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _bad(who: str, what: str):
    return SpanError(SPAN_EINVAL, f"{who}: {what}")


def _list(who: str, name: str, t, dtype, index: int, n: int) -> int:
    """Address of a dense tensor of n elements, 0 for None."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.get_device() != index or t.numel() != n or not t.is_contiguous():
        raise _bad(who, f"{name} must be contiguous, {dtype} on GPU {index}, with {n} elements, not {t.dtype} "
                        f"{tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _rows(who: str, name: str, t, dtype, index: int, shape):
    """(address, row stride) of a [rows, width] or [rows, heads, dim] tensor of that shape whose rows are dense."""
    if t.dtype is not dtype or t.get_device() != index or t.shape != shape:
        raise _bad(who, f"{name} must be {dtype} {tuple(shape)} on GPU {index}, not {t.dtype} {tuple(t.shape)} on {t.device}")
    width = shape[-1]
    if t.is_contiguous():  # (asked first: strides cost more than this)
        return t.data_ptr(), width * shape[1] if len(shape) == 3 else width
    stride = t.stride()
    if stride[-1] != 1 and width > 1:
        raise _bad(who, f"the elements of a row of {name} must follow one another")
    if len(stride) == 3:
        if stride[1] != width and shape[1] > 1:
            raise _bad(who, f"the heads of a row of {name} must follow one another")
        width *= shape[1]
    # the stride of a single row says nothing
    return t.data_ptr(), stride[0] if shape[0] > 1 else max(stride[0], width)


def _stream_of(stream, index: int) -> int:
    if stream is None:
        return _raw_stream(index)
    return stream if isinstance(stream, int) else stream.cuda_stream


def _scratch(nbytes: int, stream, device):
    """(address, bytes, owner) of a workspace on the call's stream."""
    if stream is None:
        t = torch.empty(nbytes, dtype=torch.uint8, device=device)
    else:
        if isinstance(stream, int):
            stream = torch.cuda.ExternalStream(stream, device) if stream else torch.cuda.default_stream(device)
        with torch.cuda.stream(stream):  # memory freed there by that stream's work, not by the current one's
            t = torch.empty(nbytes, dtype=torch.uint8, device=device)
    return t.data_ptr(), nbytes, t


def _given(who: str, t, index: int):
    if t.get_device() != index or not t.is_contiguous():
        raise _bad(who, f"workspace must be contiguous on GPU {index}")
    return t.data_ptr(), t.numel() * t.element_size(), t


def _gpu(who: str, name: str, t) -> int:
    if torch is None or not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise _bad(who, f"{name} must be a tensor on a GPU")
    return t.get_device()


def qk_norm_rope(q, k, v, q_gain, k_gain, eps: float, q_out, k_out, v_out, rows=None, positions=None,
                 rope_theta: float = 1e4, stream=None):
    """Head norms of q and k [rows, heads, dim] (a gain of None: no norm), rotation at `positions`
    (None: none), and the rows' way to the outputs at `rows` (None: in order); v is copied
    (span_qk_norm_rope).  Any of q, k, v may be None with its output."""
    who = "qk_norm_rope"
    lead = q if q is not None else k if k is not None else v
    index = _gpu(who, "q, k or v", lead)
    dtype = lead.dtype
    if (dtype is not torch.bfloat16 and dtype is not torch.float32) or lead.dim() != 3:
        raise _bad(who, "rows must be bfloat16 or float32 [rows, heads, dim]")
    n, heads, dim = lead.shape
    out_rows, kv_heads = -1, 0
    at, strides = [], []
    for name, t, o in (("q", q, q_out), ("k", k, k_out), ("v", v, v_out)):
        if t is None and o is None:
            at += (0, 0)
            strides += (0, 0)
            continue
        if t is None or o is None:
            raise _bad(who, f"{name} and {name}_out go together")
        if t is not lead and t.dim() == 3:
            heads = t.shape[1]
        if name != "q":
            if kv_heads not in (0, heads):
                raise _bad(who, "k and v must have the same heads")
            kv_heads = heads
        if out_rows < 0:
            out_rows = o.shape[0] if o.dim() else 0
        at_in, st_in = _rows(who, name, t, dtype, index, (n, heads, dim))
        at_out, st_out = _rows(who, name + "_out", o, dtype, index, (out_rows, heads, dim))
        at += (at_in, at_out)
        strides += (st_in, st_out)
    _check(load().span_qk_norm_rope(_QK_REC.pack(
        at[0], at[2], at[4], at[1], at[3], at[5], _list(who, "q_gain", q_gain, dtype, index, dim),
        _list(who, "k_gain", k_gain, dtype, index, dim), _list(who, "rows", rows, torch.int32, index, n),
        _list(who, "positions", positions, torch.int32, index, n), strides[0], strides[2], strides[4], strides[1],
        strides[3], strides[5], n, out_rows, q.shape[1] if q is not None else 0, kv_heads, dim,
        SPAN_BF16 if dtype is torch.bfloat16 else SPAN_F32, index, eps, rope_theta, 0), _stream_of(stream, index)))


def _adapter_rec(at, ws, ws_bytes, strides, n, width, count, rank, parts, index) -> bytes:
    cols = (*parts, 0, 0, 0)[:4]
    return _ADAPTER_REC.pack(*at, ws, ws_bytes, *strides, n, width, count, rank, len(parts), *cols, index, 0)


@lru_cache(maxsize=1024)
def _adapter_bytes(n: int, width: int, rank: int, parts: tuple) -> int:
    size = ctypes.c_size_t()
    _check(load().span_adapter_workspace(_adapter_rec((0,) * 8, 0, 0, (0, 0, 0), n, width, 0, rank, parts, 0),
                                         ctypes.byref(size)))
    return size.value


def adapter_workspace(n_rows: int, in_features: int, max_rank: int, parts: Sequence[int]) -> int:
    """Bytes of workspace of an adapter_apply call (span_adapter_workspace)."""
    if not 1 <= len(parts) <= 4:
        raise _bad("adapter_workspace", "one to four parts")
    return _adapter_bytes(n_rows, in_features, max_rank, tuple(parts))


def adapter_apply(x, base, ids, a, b, scale, out, parts: Optional[Sequence[int]] = None, ranks=None, workspace=None,
                  stream=None):
    """out = base + scale[id] (x a[id]^T) b[id]^T for each row's own adapter id (none outside
    [0, n)) (span_adapter_apply).  x [rows, in], base and out [rows, cols] (may be one tensor), ids int32
    [rows], a [n, parts, rank, in], b [n, cols, rank], scale float32 [n] or None, ranks int32 [n] or None;
    parts: the columns of each part, by default one part."""
    who = "adapter_apply"
    index = _gpu(who, "x", x)
    bf16 = torch.bfloat16
    shape, wide, weights = x.shape, out.shape, a.shape
    if len(shape) != 2 or len(wide) != 2 or len(weights) != 4:
        raise _bad(who, "x and out must have two dimensions, a four")
    n, width = shape
    cols = wide[1]
    parts = (cols,) if parts is None else tuple(parts)
    count, n_parts, rank, _ = weights
    if n_parts != len(parts) or sum(parts) != cols or not 1 <= n_parts <= 4 or weights[3] != width or wide[0] != n or \
            b.shape != (count, cols, rank):
        raise _bad(who, "a must be [n, parts, rank, in], b [n, cols, rank], parts one to four column counts that add "
                        "up to out's columns, out as many rows as x")
    at_x, st_x = _rows(who, "x", x, bf16, index, shape)
    at_out, st_out = _rows(who, "out", out, bf16, index, wide)
    at_base, st_base = (at_out, st_out) if base is out else _rows(who, "base", base, bf16, index, wide)
    at = (at_x, at_base, at_out, _list(who, "ids", ids, torch.int32, index, n),
          _list(who, "a", a, bf16, index, count * n_parts * rank * width), _list(who, "b", b, bf16, index, count * cols * rank),
          _list(who, "scale", scale, torch.float32, index, count), _list(who, "ranks", ranks, torch.int32, index, count))
    if workspace is None:
        ws = _scratch(_adapter_bytes(n, width, rank, parts), stream, x.device)
    else:
        ws = _given(who, workspace, index)
    _check(load().span_adapter_apply(_adapter_rec(at, ws[0], ws[1], (st_x, st_base, st_out), n, width, count, rank,
                                                  parts, index), _stream_of(stream, index)))


@lru_cache(maxsize=1024)
def verify_workspace(n_requests: int, max_drafts: int, vocab: int) -> int:
    """Bytes of workspace of a verify_drafts call (span_verify_workspace)."""
    size = ctypes.c_size_t()
    _check(load().span_verify_workspace(_VERIFY_REC.pack(*(0,) * 18, n_requests, max_drafts, vocab, 0),
                                        ctypes.byref(size)))
    return size.value


def verify_drafts(target_logits, drafts, u_accept, u_sample, temperature, accepted, tokens, draft_logits=None,
                  n_drafts=None, row0=None, draft_row0=None, logprobs=None, workspace=None, stream=None):
    """Keeps each request's drafts as far as the target's probabilities allow and draws the next token
    (span_verify_drafts).  target_logits float32 [rows, vocab]; drafts int32 and u_accept float32 [n, k]
    (None for k = 0: a token is sampled); u_sample and temperature float32 [n] (None: 1; 0: greedy);
    accepted int32 [n], tokens int32 and logprobs float32 [n, k + 1] are written; draft_logits float32 [draft
    rows, vocab] or None; n_drafts, row0, draft_row0 int32 [n] or None."""
    who = "verify_drafts"
    index = _gpu(who, "target_logits", target_logits)
    f32, i32 = torch.float32, torch.int32
    shape, wide = target_logits.shape, tokens.shape
    if len(shape) != 2 or len(wide) != 2 or wide[1] < 1:
        raise _bad(who, "target_logits must be [rows, vocab], tokens [requests, drafts + 1]")
    n, k, vocab = wide[0], wide[1] - 1, shape[1]
    if k > 0 and (drafts is None or u_accept is None):
        raise _bad(who, "drafts need their tokens and random numbers")
    if u_sample is None:
        raise _bad(who, "u_sample is needed")
    at_target, st_target = _rows(who, "target_logits", target_logits, f32, index, shape)
    at_draft, st_draft, draft_rows = 0, vocab, 0
    if draft_logits is not None:
        if draft_logits.dim() != 2:
            raise _bad(who, "draft_logits must be [rows, vocab]")
        draft_rows = draft_logits.shape[0]
        at_draft, st_draft = _rows(who, "draft_logits", draft_logits, f32, index, (draft_rows, vocab))
    at = (at_target, at_draft, _list(who, "row0", row0, i32, index, n), _list(who, "draft_row0", draft_row0, i32, index, n),
          _list(who, "drafts", drafts, i32, index, n * k), _list(who, "n_drafts", n_drafts, i32, index, n),
          _list(who, "u_accept", u_accept, f32, index, n * k), _list(who, "u_sample", u_sample, f32, index, n),
          _list(who, "temperature", temperature, f32, index, n), _list(who, "accepted", accepted, i32, index, n),
          _list(who, "tokens", tokens, i32, index, n * (k + 1)), _list(who, "logprobs", logprobs, f32, index, n * (k + 1)))
    if workspace is None:
        ws = _scratch(verify_workspace(n, k, vocab), stream, target_logits.device)
    else:
        ws = _given(who, workspace, index)
    _check(load().span_verify_drafts(_VERIFY_REC.pack(*at, ws[0], ws[1], st_target, st_draft, shape[0], draft_rows, n, k,
                                                      vocab, index), _stream_of(stream, index)))
