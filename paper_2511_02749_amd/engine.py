"""Execution of span queries on a pool and a decoder stack.

The generate callbacks that ``spanquery.expand_generates`` takes, backed by the
library: a batch of lowered span queries is laid out in one row space, planned
(``span_plan``: hashing, lookup, allocation), run through the stack for its first
token (``span_model_forward``), then decoded greedily one token per step
(``span_model_decode`` over the plan's block tables), and committed, so that the
prefixes and fragments it computed stay cached for the queries after it.  Every
step of the path runs in the native library; this module only lays out rows and
loops over steps.

With n_drafts > 0 a step feeds, after a query's last token, the tokens that followed the
latest earlier place in its own tokens where the same few tokens stand (an answer over
retrieved documents copies from them), and keeps those that the stack would have
generated (``span_model_decode_drafts``).  With temperature > 0 tokens are sampled, from
random numbers of `seed`.
"""
from __future__ import annotations

from dataclasses import dataclass, field
from typing import List, Optional, Sequence

import numpy as np

from . import spanquery as sq
from ._lib import SPAN_ENOMEM, SpanError
from .row_ops import SPAN_MAX_DRAFTS


@dataclass
class CallStats:
    """What one generate call planned: pages and tokens served from the cache or computed."""
    queries: int
    pages_hit: int
    tokens_hit: int
    tokens_new: int
    decode_steps: int
    drafts_fed: int = 0
    drafts_kept: int = 0


def lookup_drafts(tokens: Sequence[int], n: int, longest: int = 3) -> List[int]:
    """Up to n tokens that followed the latest earlier place of the last tokens: of the last
    `longest`, else of fewer, down to one; [] if even that stands nowhere else."""
    toks = np.asarray(tokens, np.int32)
    for m in range(min(longest, len(toks) - 1), 0, -1):
        starts = len(toks) - m  # of earlier places
        same = toks[:starts] == toks[starts]
        for i in range(1, m):
            same &= toks[i:starts + i] == toks[starts + i]
        at = np.flatnonzero(same)
        if at.size:
            return toks[at[-1] + m:at[-1] + m + n].tolist()
    return []


def _check_weight(tokens):
    """Raises for -1, which stands where the logits leave no token any weight."""
    if any(t < 0 for t in tokens):
        raise RuntimeError("a query's logits leave no token any weight")


@dataclass
class Engine:
    pool: object                       # paper_2511_02749_amd.Pool (device, bf16)
    model: object                      # paper_2511_02749_amd.Model on that pool
    stream: object = None
    calls: List[CallStats] = field(default_factory=list)
    n_drafts: int = 0                  # drafted tokens that a decode step checks, at most SPAN_MAX_DRAFTS; 0: none
    temperature: float = 0.0           # 0: greedy
    seed: int = 0

    def __post_init__(self):
        if not 0 <= self.n_drafts <= SPAN_MAX_DRAFTS:
            raise ValueError(f"n_drafts must lie in [0, {SPAN_MAX_DRAFTS}]")
        self._rng = np.random.default_rng(self.seed)

    def generate_many(self, spans: Sequence[sq.Spans], max_tokens: int,
                      adapters: Optional[Sequence[Optional[int]]] = None) -> List[List[int]]:
        """Up to max_tokens tokens for each query (one plan, one batch), through the model's
        adapter adapters[q] if given.  Every query needs a cross segment: its first token is
        read at the last cross row."""
        if max_tokens < 1:
            raise ValueError("max_tokens must be at least 1")
        queries, rows, at, history = [], [], 0, []
        for sp in spans:
            if not sp.cross:
                raise ValueError("a generate needs a cross segment to read its first token at")
            queries.append(sq.to_query(sp, row0=at))
            toks = list(sp.prefix) + [t for f in sp.fragments for t in f] + list(sp.cross)
            rows.extend(toks)
            history.append(toks)
            at += len(toks)
        plan = self.pool.plan(queries, self.stream)
        fed = kept = 0
        try:
            if adapters is not None:
                plan.set_adapters(adapters)
            rows = np.asarray(rows, np.int32)
            if self.temperature > 0:
                cur = self._sample_first(plan, rows, len(queries))
            else:
                cur = self.model.forward(plan, rows, stream=self.stream)
            out = [[t] for t in cur]
            if self.n_drafts == 0 and not self.temperature > 0:
                for _ in range(max_tokens - 1):
                    cur = self.model.decode(plan, cur, stream=self.stream)
                    for o, t in zip(out, cur):
                        o.append(t)
            else:
                _check_weight(cur)
                fed, kept = self._decode_checked(plan, history, out, max_tokens)
            st = plan.stats()
            self.calls.append(CallStats(queries=len(queries), pages_hit=st["pages_hit"], tokens_hit=st["tokens_hit"],
                                        tokens_new=st["tokens_new"], decode_steps=st["decode_steps"],
                                        drafts_fed=fed, drafts_kept=kept))
            plan.commit()
        finally:
            plan.destroy()
        return out

    def _sample_first(self, plan, rows, n: int) -> List[int]:
        import torch

        from .row_ops import verify_drafts
        dev = torch.device("cuda", self.pool.cfg.device)
        stream = torch.cuda.ExternalStream(self.stream, dev) if isinstance(self.stream, int) and self.stream else \
            self.stream or torch.cuda.current_stream(dev)
        with torch.cuda.stream(stream):
            logits = torch.empty((n, self.model.cfg.vocab), dtype=torch.float32, device=dev)
            self.model.forward(plan, rows, logits_out=logits, first_tokens=False, stream=stream)
            tokens = torch.empty((n, 1), dtype=torch.int32, device=dev)
            verify_drafts(logits, None, None, torch.from_numpy(self._rng.random(n, np.float32)).to(dev),
                          torch.full((n,), self.temperature, device=dev), torch.empty(n, dtype=torch.int32, device=dev),
                          tokens)
            return tokens[:, 0].tolist()

    def _step(self, plan, out, open_, drafts):
        n = len(out)
        return self.model.decode_drafts(
            plan, [o[-1] if go else -1 for o, go in zip(out, open_)], drafts,
            u_accept=[self._rng.random(len(d), np.float32) for d in drafts], u_sample=self._rng.random(n, np.float32),
            temperature=np.full(n, self.temperature, np.float32), stream=self.stream)

    def _decode_checked(self, plan, history, out, max_tokens: int):
        """Steps of drafts and sampled tokens until every query has max_tokens; (drafts fed, kept)."""
        n, fed, kept = len(out), 0, 0
        seen = []  # each query's own tokens, with room for those to come
        for h, o in zip(history, out):
            seen.append(np.empty(len(h) + max_tokens, np.int32))
            seen[-1][:len(h) + len(o)] = h + o
        while any(len(o) < max_tokens for o in out):
            open_ = [len(o) < max_tokens for o in out]
            drafts = [lookup_drafts(s[:len(h) + len(o)], min(self.n_drafts, max_tokens - len(o) - 1)) if go else []
                      for s, h, o, go in zip(seen, history, out, open_)]
            try:
                got = self._step(plan, out, open_, drafts)
            except SpanError as e:
                if e.code != SPAN_ENOMEM or not any(drafts):
                    raise
                drafts = [[]] * n  # no pages for drafted tokens: a step without them needs fewer
                got = self._step(plan, out, open_, drafts)
            _check_weight(t for g in got for t in g)
            fed += sum(len(d) for d in drafts)
            kept += sum(len(g) - 1 for g in got if g)
            for s, h, o, g in zip(seen, history, out, got):
                s[len(h) + len(o):len(h) + len(o) + len(g)] = g
                o.extend(g)
        return fed, kept

    def generate(self, tokens: Sequence[int], max_tokens: int) -> List[int]:
        """A generate over plain messages: the tokens are the cross segment."""
        return self.generate_many([sq.Spans(prefix=[], fragments=[], cross=list(tokens))], max_tokens)[0]

    def generate_join(self, spans: sq.Spans, max_tokens: int) -> List[int]:
        return self.generate_many([spans], max_tokens)[0]

    def run(self, tree: sq.Node) -> List[int]:
        """Run an optimized tree: its inner generates innermost first, then the root."""
        ex = sq.expand_generates(tree, self.generate, self.generate_join)
        root = sq.to_spans(ex)
        return self.generate_join(root, max(1, root.max_tokens))
