"""A decode step that samples with drafts, where each draft's verdict is forced by its random number alone or by its
distribution alone, against the float64 oracle of tests/stack_rows.py.

Tolerances are tests/test_gpu_stack_row_ops.py's: logits within 2e-2 of the oracle's, so log-probabilities at
temperature T within 4e-2 / T, and a token's place in the running sum within 4e-2 / T of the whole.  The verdicts
have no tolerance: a probability is above 0 and below 0.9 with far more room than that.
"""
import numpy as np
import pytest

import workloads as W
from tests.helpers import StackRun, oracle_weights
from tests.stack_rows import Extras
from tests.test_gpu_stack_row_ops import LOGIT_TOL, _logits_after

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
spanq = pytest.importorskip("paper_2511_02749_amd")


@pytest.fixture(autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    print(flush=True)


@pytest.mark.parametrize("by", ["random number", "distribution", "random number, no distribution"])
def test_each_draft_gets_its_own_random_number_and_distribution(by):
    swl = W.stack_small()
    run, Wt = StackRun(swl, num_pages=256), oracle_weights(swl.weights)
    batch = swl.batches[0]
    n, V = len(batch), swl.weights.vocab
    rng = np.random.default_rng(len(by))
    plan = run.pool.plan(batch)
    out = [[t] for t in run.model.forward(plan, swl.row_tokens)]
    kept = refused = 0
    for step in range(20):
        heat = rng.uniform(0.6, 1.4, n).astype(np.float32)
        keep = [[bool(rng.random() < 0.7) for _ in range(int(rng.integers(0, 5)))] for _ in range(n)]
        drafts = [[int(t) for t in rng.integers(0, V, len(k))] for k in keep]
        idle = step % n  # a query that sits out, another one each step; its drafts have no row
        rows, ua = [], []
        for qi in range(n):
            ua.append([])
            for ok, d in zip(keep[qi], drafts[qi]):
                at = d if by != "distribution" or not ok else (d + 1) % V  # where q has all its weight
                ua[qi].append(0.9 if by == "distribution" or not ok else 0.0)
                if qi != idle:
                    rows.append(at)
        logits = None
        if "no dist" not in by:
            logits = torch.full((len(rows), V), -float("inf"), device="cuda")
            logits[torch.arange(len(rows)), torch.tensor(rows, dtype=torch.long)] = 3.0
        us = rng.random(n).astype(np.float32)
        got, lps = run.model.decode_drafts(plan, [o[-1] if qi != idle else -1 for qi, o in enumerate(out)], drafts, u_accept=ua,
                                           u_sample=us, temperature=heat, draft_logits=logits, logprobs=True)
        for qi, q in enumerate(batch):
            if qi == idle:
                assert got[qi] == []
                continue
            a = next((j for j, ok in enumerate(keep[qi]) if not ok), len(keep[qi]))
            assert got[qi][:-1] == drafts[qi][:a], (step, qi, keep[qi], drafts[qi], got[qi])
            lg = _logits_after(run, Wt, q, Extras(), -1, out[qi] + got[qi])[len(out[qi]):-1] / float(heat[qi])
            p = np.exp(lg - lg.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            tol, t, left = 2 * LOGIT_TOL / float(heat[qi]), got[qi][-1], p[a].copy()
            assert np.max(p) < 0.8  # (as the verdicts assume)
            assert np.max(np.abs(np.array(lps[qi]) - np.log(p[np.arange(a + 1), got[qi]]))) <= tol
            if a < len(keep[qi]):
                assert t != drafts[qi][a]
                left[drafts[qi][a]] = 0.0
            run_sum = np.cumsum(left) / left.sum()
            assert run_sum[t] - left[t] / left.sum() - tol <= us[qi] <= run_sum[t] + tol, (step, qi)
            kept, refused = kept + a, refused + (a < len(keep[qi]))
            out[qi] += got[qi]
    print(f"by {by}: {kept} drafts kept, {refused} refused", flush=True)
    assert kept > 5 and refused > 5
    plan.destroy()
    run.close()
