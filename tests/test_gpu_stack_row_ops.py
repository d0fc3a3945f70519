"""GPU parity of the decoder stack with head norms, adapters and drafted tokens, against the
float64 oracle of tests/stack_rows.py.

Tolerances are those of the plain small stacks (tests/test_gpu_stack.py): hidden states within
2e-2 + 2^-6 |oracle|, logits within 2e-2, three layers.  The operators add one bf16 rounding a
product (2^-8 of it, as every stored tensor) and none elsewhere.  A generated token must be one
whose oracle logit is within twice the logit tolerance of the oracle's maximum (both logits are off
by at most the tolerance); a drafted token further below must be refused, one that leads every
other by more must be kept.
"""
import numpy as np
import pytest

import workloads as W
from oracle import stack as OS
from tests.helpers import StackRun, computed_rows, oracle_weights, query_rows
from tests.stack_rows import Extras, query_states

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
spanq = pytest.importorskip("paper_2511_02749_amd")

ATOL, RTOL, LOGIT_TOL = 2e-2, 2.0 ** -6, 2e-2


@pytest.fixture(autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    print(flush=True)


def _bf16(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(torch.bfloat16)


def _extras(run, norms=True, adapters=0, rank=16, seed=0, products=("qkv", "o", "gate_up", "down")):
    """Head norms and adapters for a stack, given to its model; the oracle's view of them."""
    sw = run.swl.weights
    rng = np.random.default_rng(seed)
    ex, f64 = Extras(), lambda t: t.float().numpy().astype(np.float64)  # noqa: E731
    L, hq, hkv, d, H, F = sw.n_layers, sw.n_q_heads, sw.n_kv_heads, sw.head_dim, sw.hidden, sw.ffn
    if norms:
        gains = [[_bf16(0.8 + 0.2 * rng.standard_normal(d)) for _ in range(L)] for _ in range(2)]
        gains[1][L - 1] = None  # the last layer's keys go without
        run.model.set_qk_norm(*[[None if g is None else g.cuda() for g in side] for side in gains])
        ex.q_norm, ex.k_norm = [[None if g is None else f64(g) for g in side] for side in gains]
    if adapters:
        sizes = {"qkv": (3, H, (hq + 2 * hkv) * d), "o": (1, hq * d, H), "gate_up": (2, H, 2 * F), "down": (1, F, H)}
        ranks = rng.integers(1, rank + 1, adapters).astype(np.int32)
        ranks[0] = rank
        scale = rng.uniform(0.5, 1.5, adapters).astype(np.float32)
        dev, ex.adapters = {}, {}
        for name in products:
            parts, k, n = sizes[name]
            pairs = []
            for l in range(L):
                a = _bf16(rng.standard_normal((adapters, parts, rank, k)) * 0.02)
                b = _bf16(rng.standard_normal((adapters, n, rank)) * 0.05)
                for i, r in enumerate(ranks):  # what lies past a rank does not count
                    a[i, :, r:] = float("nan")
                    b[i, :, r:] = float("nan")
                pairs.append((a, b))
            if name == "o":
                pairs[0] = None  # one layer without this product's adapters
            dev[name] = tuple([None if p is None else p[s].cuda() for p in pairs] for s in (0, 1))
            ex.adapters[name] = [None if p is None else (f64(p[0]), f64(p[1])) for p in pairs]
        run.model.set_adapters(adapters, rank, scale=torch.from_numpy(scale).cuda(), ranks=torch.from_numpy(ranks).cuda(), **dev)
        ex.scale, ex.ranks = scale, ranks
    return ex


def _check_hidden(run, Wt, batch, rows, ex, ids, what):
    left, worst = set(int(r) for r in rows), 0.0
    for q, i in zip(batch, ids):
        mine = [(at, int(r)) for at, r in enumerate(query_rows(q)) if int(r) in left]
        if not mine:
            continue
        ref, _ = query_states(run.swl, Wt, q, ex, i)
        got = run.hidden_rows([r for _, r in mine]).astype(np.float64)
        ref = ref[[at for at, _ in mine]]
        worst = max(worst, float(np.max(np.abs(got - ref) - RTOL * np.abs(ref))))
        left -= {r for _, r in mine}
    print(f"{what}: {len(rows)} rows, max of err - rtol|ref| {worst:.4g}", flush=True)
    assert not left and worst <= ATOL, what


def _logits_after(run, Wt, q, ex, adapter, extra):
    """Oracle logits after the last cross token and after each of `extra`."""
    x, first = query_states(run.swl, Wt, q, ex, adapter, extra)
    return np.stack([OS.final_logits(r, Wt, run.swl.rms_eps) for r in x[first + len(q.cross.tokens) - 1:]])


def _check_tokens(run, Wt, batch, ex, ids, out, what):
    worst = 0.0
    for q, i, o in zip(batch, ids, out):
        lg = _logits_after(run, Wt, q, ex, i, o)[:len(o)]
        worst = max(worst, float(np.max(lg.max(1) - lg[np.arange(len(o)), o])))
    print(f"{what}: tokens at most {worst:.3g} below the oracle's best", flush=True)
    assert worst <= 2 * LOGIT_TOL, what


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("norms,adapters", [(True, 0), (False, 3), (True, 3)])
def test_forward_whole_output(head_dim, norms, adapters):
    """Every computed row of a cold batch; the fragments' rows know no adapter, so a second query
    of the batch with another adapter reads the same pages."""
    swl = W.stack_small(head_dim=head_dim)
    run, Wt = StackRun(swl), oracle_weights(swl.weights)
    ex = _extras(run, norms, adapters)
    batch = swl.batches[0]
    ids = [(-1, 0, 2, 1)[i % 4] if adapters and i else (1 if adapters else -1) for i in range(len(batch))]
    plan = run.pool.plan(batch)
    plan.set_adapters(ids)
    n = len(batch)
    lg = torch.zeros((n, swl.weights.vocab), dtype=torch.float32, device="cuda")
    toks = run.model.forward(plan, swl.row_tokens, hidden_out=run.hidden, logits_out=lg)
    torch.cuda.synchronize()
    _check_hidden(run, Wt, batch, computed_rows(plan), ex, ids, f"d{head_dim} norms {norms} adapters {ids}")
    for qi, (q, i) in enumerate(zip(batch, ids)):
        ref = _logits_after(run, Wt, q, ex, i, [])[0]
        assert float(np.max(np.abs(lg[qi].cpu().numpy() - ref))) <= LOGIT_TOL
        assert ref[toks[qi]] >= ref.max() - 2 * LOGIT_TOL
    plan.commit()
    plan.destroy()
    run.close()


def test_cached_fragments_serve_every_adapter():
    """Pages computed for a query without an adapter are hits for a query with one, whose cross rows and
    tokens are the oracle's; with the adapters taken away the stack is the plain one again."""
    swl = W.stack_small(orders=((0, 1, 2, 3), (3, 1, 0, 2)), batch_split=(1, 1))
    run, Wt = StackRun(swl), oracle_weights(swl.weights)
    plain, _, lg0 = run.run(swl.batches[0])
    plain.destroy()
    ex = _extras(run, norms=False, adapters=2)
    for adapter in (1, 0, -1):
        plan = run.pool.plan(swl.batches[1])
        assert plan.stats()["tokens_new"] == 0
        plan.set_adapters([adapter])
        out = [run.model.forward(plan, swl.row_tokens, hidden_out=run.hidden)[0]]
        _check_hidden(run, Wt, swl.batches[1], plan.rows()[1], ex, [adapter], f"warm, adapter {adapter}")
        for _ in range(4):
            out.append(run.model.decode(plan, [out[-1]])[0])
        _check_tokens(run, Wt, swl.batches[1], ex, [adapter], [out], f"decode, adapter {adapter}")
        plan.destroy()
    plan = run.pool.plan(swl.batches[1])
    plan.set_adapters([2])
    with pytest.raises(spanq.SpanError) as e:
        run.model.forward(plan, swl.row_tokens)
    assert e.value.code == -1
    run.model.set_adapters()
    plan.set_adapters([0])
    with pytest.raises(spanq.SpanError):
        run.model.forward(plan, swl.row_tokens)
    plan.destroy()
    run.pool.reset()
    again, _, lg1 = run.run(swl.batches[0])
    assert np.array_equal(lg0, lg1)  # the plain stack, bit for bit
    again.destroy()
    run.close()


@pytest.mark.parametrize("rows", [5, 40])
def test_many_adapted_rows_and_depths(rows):
    """Cross segments of a few and of many rows (the GEMV, GEMM and adapter kernels of either), two
    queries of one batch with adapters and one without."""
    sw = W.stack_weights(2, 2, 512, 8, 2, 64, 1024, 1000)
    batches, rt = W.stack_queries(3, 1000, 24, (50, 33), rows * 4, [[0, 1], [1, 0], [0, 1]])
    swl = W.StackWorkload(name="adapted", weights=sw, batches=batches, row_tokens=rt)
    run, Wt = StackRun(swl), oracle_weights(sw)
    ex = _extras(run, norms=True, adapters=2, rank=8, products=("qkv", "down"))
    batch = swl.batches[0]
    ids = [1, -1, 0][:len(batch)]
    plan = run.pool.plan(batch)
    plan.set_adapters(ids)
    run.model.forward(plan, swl.row_tokens, hidden_out=run.hidden, first_tokens=False)
    torch.cuda.synchronize()
    _check_hidden(run, Wt, batch, computed_rows(plan), ex, ids, f"{rows * 4} rows a query")
    plan.destroy()
    run.close()


def _drafts_for(lg, rng, wrong):
    """A draft chain from oracle logits: the argmax where it leads clearly, and at `wrong` a token far below."""
    best = int(np.argmax(lg))
    return best if not wrong else int(np.argsort(lg)[int(rng.integers(0, 100))])


@pytest.mark.parametrize("norms,adapters", [(False, 0), (True, 3)])
def test_drafts_are_kept_and_refused_as_the_oracle_says(norms, adapters):
    """Greedy steps with drafts: chains that follow the oracle's argmax up to a wrong token, of other
    lengths for each query, one of them without drafts.  What is kept, the token after it and, since steps follow
    one another over what was taken back, everything generated are the oracle's."""
    swl = W.stack_small()
    run, Wt = StackRun(swl), oracle_weights(swl.weights)
    ex = _extras(run, norms, adapters)
    batch = swl.batches[0]
    n = len(batch)
    ids = [(2, -1, 0)[i % 3] if adapters else -1 for i in range(n)]
    plan = run.pool.plan(batch)
    plan.set_adapters(ids)
    out = [[t] for t in run.model.forward(plan, swl.row_tokens)]
    rng = np.random.default_rng(0)
    kept = refused = 0
    for step, (length, wrong) in enumerate([(3, 1), (4, 4), (1, 0), (0, 0), (20, 2), (2, 2)]):
        drafts, ok = [], []
        for qi, q in enumerate(batch):
            chain, sure = [], []
            for j in range(length if (qi + step) % 3 else 0):
                lg = _logits_after(run, Wt, q, ex, ids[qi], out[qi] + chain)[-1]
                t = _drafts_for(lg, rng, j == wrong)
                lead = np.sort(lg)[-1] - np.sort(lg)[-2]
                sure.append(True if t == int(np.argmax(lg)) and lead > 2 * LOGIT_TOL else
                            False if lg[t] < lg.max() - 2 * LOGIT_TOL else None)
                chain.append(t)
            drafts.append(chain)
            ok.append(sure)
        feed = [o[-1] for o in out]
        if step == 3:
            feed[0] = -1  # a query that sits out
        got, lps = run.model.decode_drafts(plan, feed, drafts, logprobs=True)
        for qi in range(n):
            if feed[qi] < 0:
                assert got[qi] == []
                continue
            a = len(got[qi]) - 1
            assert got[qi][:a] == drafts[qi][:a] and len(lps[qi]) == a + 1
            assert False not in ok[qi][:a]
            assert a == len(drafts[qi]) or ok[qi][a] is not True
            lg = _logits_after(run, Wt, batch[qi], ex, ids[qi], out[qi] + got[qi])[len(out[qi]):-1]
            lg = lg - np.log(np.exp(lg).sum(-1, keepdims=True))
            assert np.max(np.abs(np.array(lps[qi]) - lg[np.arange(a + 1), got[qi]])) <= 2 * LOGIT_TOL
            kept += a
            refused += len(drafts[qi]) - a
            out[qi] += got[qi]
    assert kept > 0 and refused > 0
    _check_tokens(run, Wt, batch, ex, ids, out, f"drafts kept {kept}, refused {refused}")
    plan.commit()
    assert run.pool.info()["free_pages"] == run.pool.info()["num_pages"] - run.pool.info()["cached_pages"]
    plan.destroy()
    run.close()


def test_sampled_steps_follow_their_random_numbers():
    """Temperature: the token's place in the oracle's running sum is the random number's, as far as
    logits off by 2e-2 move that (4e-2 / T of the whole), its log-probability the oracle's; drafts with a
    distribution of their own go through; greedy and sampling queries stand in one step."""
    swl = W.stack_small()
    run, Wt = StackRun(swl), oracle_weights(swl.weights)
    ex = Extras()
    batch = swl.batches[0]
    n, V = len(batch), swl.weights.vocab
    plan = run.pool.plan(batch)
    out = [[t] for t in run.model.forward(plan, swl.row_tokens)]
    rng = np.random.default_rng(4)
    heat = np.array([(0.5, 0.0, 1.0)[i % 3] for i in range(n)], np.float32)
    for step in range(3):
        us = rng.random(n).astype(np.float32)
        got, lps = run.model.decode_drafts(plan, [o[-1] for o in out], u_sample=us, temperature=heat, logprobs=True)
        for qi, q in enumerate(batch):
            lg = _logits_after(run, Wt, q, ex, -1, out[qi])[-1]
            t, = got[qi]
            T = float(heat[qi]) or 1.0
            p = np.exp((lg - lg.max()) / T)
            p /= p.sum()
            assert abs(lps[qi][0] - np.log(p[t])) <= 2 * LOGIT_TOL / T
            if heat[qi] > 0:
                cum = np.cumsum(p)
                assert cum[t] - p[t] - 4e-2 / T <= us[qi] <= cum[t] + 4e-2 / T
            else:
                assert lg[t] >= lg.max() - 2 * LOGIT_TOL
            out[qi].append(t)
    drafts = [list(rng.integers(0, V, i % 3)) for i in range(n)]
    rows = sum(len(d) for d in drafts)
    dl = torch.randn(rows, V, device="cuda")
    got = run.model.decode_drafts(plan, [o[-1] for o in out], drafts, u_accept=[rng.random(len(d)) for d in drafts],
                                  u_sample=rng.random(n), temperature=np.full(n, 0.7), draft_logits=dl)
    assert all(1 <= len(g) <= len(d) + 1 and all(0 <= t < V for t in g) for g, d in zip(got, drafts))
    for bad in (dict(draft_logits=dl[:-1]), dict(u_sample=None), dict(u_accept=None), dict(drafts=drafts[:-1]),
                dict(drafts=[[V]] + drafts[1:]), dict(drafts=[[0] * 65] + drafts[1:])):
        args = {**dict(tokens=[o[-1] for o in out], drafts=drafts, u_accept=[rng.random(70) for _ in drafts],
                       u_sample=rng.random(n), temperature=np.full(n, 0.7)), **bad}
        with pytest.raises(spanq.SpanError) as e:
            run.model.decode_drafts(plan, **args)
        assert e.value.code == -1
    plan.destroy()
    run.close()


def test_weights_of_other_sizes_types_and_devices_are_refused():
    swl = W.stack_small()
    run = StackRun(swl)
    sw, bf = swl.weights, torch.bfloat16
    L, H, F = sw.n_layers, sw.hidden, sw.ffn
    a, b = torch.zeros(2, 1, 8, F, dtype=bf, device="cuda"), torch.zeros(2, H, 8, dtype=bf, device="cuda")
    run.model.set_adapters(2, 8, down=([a] * L, [b] * L))
    for bad in (dict(max_rank=16), dict(down=([a] * L, [b[:1]] * L)), dict(down=([a.cpu()] * L, [b] * L)),
                dict(down=([a.float()] * L, [b] * L)), dict(down=([a] * (L - 1), [b] * L)), dict(down=([a] * L, None)),
                dict(scale=torch.ones(2)), dict(scale=torch.ones(1, device="cuda")), dict(ranks=torch.ones(2, device="cuda")),
                dict(down=([a.transpose(2, 3)] * L, [b] * L))):
        with pytest.raises(spanq.SpanError) as e:
            run.model.set_adapters(**{**dict(n_adapters=2, max_rank=8, down=([a] * L, [b] * L)), **bad})
        assert e.value.code == -1
    gain = torch.ones(sw.head_dim, dtype=bf, device="cuda")
    for bad in ([gain] * (L + 1), [gain.float()] * L, [gain[:-8]] * L, [gain.cpu()] * L):
        with pytest.raises(spanq.SpanError):
            run.model.set_qk_norm(bad)
    plan = run.pool.plan(swl.batches[0])
    toks = run.model.forward(plan, swl.row_tokens)
    with pytest.raises(spanq.SpanError):  # on the host
        run.model.decode_drafts(plan, toks, [[1]] * len(toks), draft_logits=torch.zeros(len(toks), sw.vocab))
    plan.destroy()
    run.close()


@pytest.mark.parametrize("temperature", [0.0, 0.8])
def test_engine_with_lookup_drafts_and_adapters(temperature):
    """The engine's steps with drafts looked up in each query's own tokens: as many tokens as asked
    for, greedy ones the oracle's, over adapters and head norms, and nothing left in the pool."""
    from paper_2511_02749_amd import spanquery as sq
    from paper_2511_02749_amd.engine import Engine
    swl = W.stack_small()
    run, Wt = StackRun(swl, num_pages=256), oracle_weights(swl.weights)
    ex = _extras(run, norms=True, adapters=2)
    eng = Engine(run.pool, run.model, n_drafts=4, temperature=temperature, seed=3)
    loop = [5, 6, 7, 8, 9] * 6
    spans = [sq.Spans(prefix=list(range(30)), fragments=[loop, [40 + i for i in range(20)]], cross=[5, 6, 7]),
             sq.Spans(prefix=list(range(30)), fragments=[loop], cross=[8, 9, 5, 6]),
             sq.Spans(prefix=[], fragments=[], cross=[11])]
    ids = [1, None, 0]
    out = eng.generate_many(spans, 12, adapters=ids)
    assert [len(o) for o in out] == [12, 12, 12]
    call = eng.calls[-1]
    print(f"T {temperature}: {call.decode_steps} steps, {call.drafts_fed} drafts fed, {call.drafts_kept} kept", flush=True)
    assert call.drafts_kept <= call.drafts_fed and call.decode_steps <= 11
    if temperature == 0:  # (a token sampled from nearly flat logits hardly ever stood before: nothing to look up)
        assert call.drafts_fed > 0
        batch = []
        for s in spans:
            q = sq.to_query(s, row0=0)
            batch.append(q)
        _check_tokens(run, Wt, batch, ex, [1, -1, 0], out, "engine")
    i = run.pool.info()
    assert i["pinned_pages"] == 0 and i["free_pages"] == i["num_pages"] - i["cached_pages"]
    assert eng.generate(list(range(5)), 3) and len(eng.calls) == 2
    run.close()

