"""Oracle of a decoder stack with head norms and adapters, in float64 on the CPU: the layer of
oracle/stack.py with, on the way, the norms of each head of q and k and the low-rank adapter of
the rows from a token on, every stored tensor rounded to bfloat16 as the library stores it."""
from dataclasses import dataclass
from typing import Optional, Sequence

import numpy as np

from oracle import attention as A
from oracle import stack as OS


@dataclass
class Extras:
    q_norm: Optional[Sequence[np.ndarray]] = None   # per layer [head_dim], or None
    k_norm: Optional[Sequence[np.ndarray]] = None
    # product name -> per layer (a [n, parts, rank, in], b [n, out, rank]) or None; parts of the product
    adapters: Optional[dict] = None
    scale: Optional[np.ndarray] = None
    ranks: Optional[np.ndarray] = None


def forward(tokens, lay, W, n_layers, theta, eps, ex: Extras, adapter: int, first: int):
    """Hidden states [N, hidden] after n_layers; `adapter` acts on the rows from `first` on (-1: none)."""
    rnd = OS.round_bf16
    hq, hkv, d = W.n_q_heads, W.n_kv_heads, W.head_dim
    f = W.w_down[0].shape[0]
    widths = {"qkv": (hq * d, hkv * d, hkv * d), "gate_up": (f, f), "o": None, "down": None}

    def adapt(name, l, x, y):
        pair = (ex.adapters or {}).get(name)
        if adapter < 0 or pair is None or pair[l] is None:
            return y
        a, b = (np.asarray(t[adapter], np.float64) for t in pair[l])
        rank = int(ex.ranks[adapter])
        y, col = y.copy(), 0
        for p, w in enumerate(widths[name] or (y.shape[1],)):
            low = x[first:] @ a[p, :rank].T
            y[first:, col:col + w] = rnd(y[first:, col:col + w] + float(ex.scale[adapter]) * (low @ b[col:col + w, :rank].T))
            col += w
        return y

    def heads(x, gain):
        return x if gain is None else rnd(OS.rms_norm(x, gain, eps))

    x = np.asarray(np.asarray(W.embed)[np.asarray(tokens, np.int64)], np.float64)
    for l in range(n_layers):
        n_tok = x.shape[0]
        n = rnd(OS.rms_norm(x, W.attn_norm[l], eps))
        qkv = adapt("qkv", l, n, rnd(n @ np.asarray(W.w_qkv[l], np.float64)))
        q = heads(qkv[:, :hq * d].reshape(n_tok, hq, d), ex.q_norm and ex.q_norm[l])
        k = heads(qkv[:, hq * d:(hq + hkv) * d].reshape(n_tok, hkv, d), ex.k_norm and ex.k_norm[l])
        v = qkv[:, (hq + hkv) * d:].reshape(n_tok, hkv, d)
        o = rnd(A.span_attention(q, k, v, lay, theta)).reshape(n_tok, hq * d)
        h = adapt("o", l, o, rnd(x + o @ np.asarray(W.w_o[l], np.float64)))
        n2 = rnd(OS.rms_norm(h, W.ffn_norm[l], eps))
        gu = adapt("gate_up", l, n2, rnd(n2 @ np.asarray(W.w_gate_up[l], np.float64)))
        act = rnd(OS.silu(gu[:, :f]) * gu[:, f:])
        x = adapt("down", l, act, rnd(h + act @ np.asarray(W.w_down[l], np.float64)))
    return x


def query_states(swl, Wt, query, ex, adapter, extra=()):
    """Hidden states of S = prefix | fragments | cross | extra (tokens generated after it)."""
    cross = list(query.cross.tokens) + list(extra)
    toks = OS.query_tokens(query.prefix.tokens, [f.tokens for f in query.frags], cross)
    pre, frags = len(query.prefix.tokens), [len(f.tokens) for f in query.frags]
    lay = A.layout(pre, frags, len(cross))
    first = pre + sum(frags)
    return forward(toks, lay, Wt, swl.weights.n_layers, swl.rope_theta, swl.rms_eps, ex, adapter, first), first
