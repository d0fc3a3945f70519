"""Row operators of a decoder stack on torch tensors (span_qk_norm_rope, span_adapter_apply,
span_verify_drafts).  Argument marshalling only, most of it native (binding/rowops.cpp): types,
shapes and devices are checked there, sizes, strides and alignment by the library.

Tensors lie on one GPU; a call is enqueued on `stream`, by default that GPU's current one.
Outputs are written in place, as by torch's own in-place calls, but carry no history: the operators have no
gradients, and none flow through them to inputs that require them.
A workspace that is not given comes from torch's allocator, on the call's stream, and goes
back to it when the call has been enqueued, as torch's own temporaries do.
"""
from __future__ import annotations

import ctypes
import struct
from typing import Optional, Sequence

from ._lib import SPAN_EINVAL, SPAN_ENOMEM, SpanError, _check, load, torch

SPAN_MAX_DRAFTS = 64

# span_adapter_call and span_verify_call (include/spanq.h) as packed records
_ADAPTER_REC = struct.Struct("<10Q4q10i")
_VERIFY_REC = struct.Struct("<14Q4q4i")


def _scratch(nbytes: int, stream, index: int):
    """Memory of a stream that is not the current one."""
    device = torch.device("cuda", index)
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device) if stream else torch.cuda.default_stream(device)
    try:
        with torch.cuda.stream(stream):  # freed there by that stream's work, not by the current one's
            return torch.empty(nbytes, dtype=torch.uint8, device=device)
    except torch.OutOfMemoryError as e:
        raise SpanError(SPAN_ENOMEM, f"workspace: {e}") from None


_native = None


def _bind():
    """The native calls, once they have the library's entries."""
    global _native
    if torch is None:
        raise SpanError(SPAN_EINVAL, "the row operators take torch tensors")
    lib = load()
    try:
        from . import _rowops
    except ImportError as e:
        raise FileNotFoundError("_rowops.so not built: run python -m paper_2511_02749_amd.build") from e
    entries = (lib.span_qk_norm_rope, lib.span_adapter_workspace, lib.span_adapter_apply, lib.span_verify_workspace,
               lib.span_verify_drafts)
    # the current stream's address: without a Stream object, if torch can
    raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
        lambda index: torch.cuda.current_stream(index).cuda_stream)
    _rowops.bind(*[ctypes.cast(f, ctypes.c_void_p).value for f in entries], SpanError, _check, raw_stream, _scratch)
    _native = _rowops
    return _native


def qk_norm_rope(q, k, v, q_gain, k_gain, eps: float, q_out, k_out, v_out, rows=None, positions=None,
                 rope_theta: float = 1e4, stream=None):
    """Head norms of q and k [rows, heads, dim] (a gain of None: no norm), rotation at `positions`
    (None: none), and the rows' way to the outputs at `rows` (None: in order); v is copied
    (span_qk_norm_rope).  Any of q, k, v may be None with its output."""
    (_native or _bind()).qk_norm_rope(q, k, v, q_gain, k_gain, eps, q_out, k_out, v_out, rows, positions, rope_theta, stream)


def adapter_workspace(n_rows: int, in_features: int, max_rank: int, parts: Sequence[int]) -> int:
    """Bytes of workspace of an adapter_apply call (span_adapter_workspace)."""
    if not 1 <= len(parts) <= 4:
        raise SpanError(SPAN_EINVAL, "adapter_workspace: one to four parts")
    size = ctypes.c_size_t()
    _check(load().span_adapter_workspace(_ADAPTER_REC.pack(*(0,) * 13, n_rows, in_features, 0, max_rank, len(parts),
                                                           *(*parts, 0, 0, 0)[:4], 0, 0), ctypes.byref(size)))
    return size.value


def adapter_apply(x, base, ids, a, b, scale, out, parts: Optional[Sequence[int]] = None, ranks=None, workspace=None,
                  stream=None):
    """out = base + scale[id] (x a[id]^T) b[id]^T for each row's own adapter id (none outside
    [0, n)) (span_adapter_apply).  x [rows, in], base and out [rows, cols] (may be one tensor), ids int32
    [rows], a [n, parts, rank, in], b [n, cols, rank], scale float32 [n] or None, ranks int32 [n] or None;
    parts: the columns of each part, by default one part."""
    (_native or _bind()).adapter_apply(x, base, ids, a, b, scale, out, parts, ranks, workspace, stream)


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
    (_native or _bind()).verify_drafts(target_logits, drafts, u_accept, u_sample, temperature, accepted, tokens, draft_logits,
                                       n_drafts, row0, draft_row0, logprobs, workspace, stream)
