"""Cases of the decoder stack's row operators, with their plain forms.

Three operators that a decode step of many requests goes through beside its products and
its attention:

- ``adapt``: low-rank adapters of many requests beside a shared projection,
  out = base + s (x A^T) B^T with each row's own A, B and s;
- ``verify``: drafted tokens checked against the target's logits with given random numbers
  (without drafts: a token sampled for each request);
- ``qk``: the norms of queries and keys for each head, their rotation in the same pass, and
  the rows' way into the caller's order.

A case is a dict of plain values; inputs follow from the case and the seed alone.  Where
``own`` is false, ``run`` is elementary torch operations.
"""
import math

import numpy as np
import torch

own = False

THETA = 1e4
EPS = 1e-5

_ADAPT = dict(op="adapt", rows=1, width=4096, parts="4096", rank=16, adapters=1, mixed_ranks=False, bare=False,
              segments=False)
_VERIFY = dict(op="verify", requests=1, drafts=4, vocab=128256, draft_logits=True, ragged=False, masked=False,
               greedy=False)
_QK = dict(op="qk", rows=1, heads=32, kv_heads=8, dim=128, dtype="bf16", rotate=True, scatter=False)


def listed():
    return [
        # one request decoding with an adapter on q, k and v: latency
        dict(_ADAPT, name="adapt_one_row_qkv", parts="4096,1024,1024"),
        # a decode step of many requests, each with its own adapter, on the output projection
        dict(_ADAPT, name="adapt_decode_64_adapters", rows=64, adapters=64),
        # a decode step on the down projection: a long reduction, larger ranks, few adapters shared
        dict(_ADAPT, name="adapt_decode_down", rows=48, width=14336, rank=64, adapters=12),
        # cross segments of a few requests through gate|up: the largest activations
        dict(_ADAPT, name="adapt_cross_rows_gate_up", rows=2048, parts="14336,14336", rank=32, adapters=4,
             segments=True),
        # ragged segments, mixed ranks, rows without an adapter, sizes of the smaller stack
        dict(_ADAPT, name="adapt_ragged_mixed_ranks", rows=777, width=2048, parts="2048", rank=24, adapters=7,
             mixed_ranks=True, bare=True, segments=True),
        # one request, drafts copied from its documents: latency
        dict(_VERIFY, name="verify_one_lookup", draft_logits=False),
        # a batch with a draft model's logits, temperatures mixed with greedy requests
        dict(_VERIFY, name="verify_batch_draft_model", requests=64, greedy=True),
        # a token sampled for each of many requests under grammar masks, no drafts
        dict(_VERIFY, name="sample_batch_masked", requests=256, drafts=0, draft_logits=False, masked=True),
        # an odd vocabulary, ragged draft counts packed one after another
        dict(_VERIFY, name="verify_ragged_odd_vocab", requests=17, drafts=7, vocab=50257, ragged=True),
        # one decoding row, as the stack calls it (no rotation): latency
        dict(_QK, name="qk_one_row", rotate=False),
        # a cold prefill's rows
        dict(_QK, name="qk_prefill", rows=8192),
        # an fp32 pool's rows in the caller's order, three query heads for each kv head
        dict(_QK, name="qk_f32_scattered", rows=1333, heads=24, dim=64, dtype="f32", scatter=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["adapt", "verify", "qk"])
    if op == "adapt":
        rows = _log_int(rng, 1, 2048)
        n_parts = rng.choice([1, 1, 2, 3])
        parts = [8 * _log_int(rng, 32, 1792) for _ in range(n_parts)]
        return dict(_ADAPT, rows=rows, width=8 * _log_int(rng, 32, 1792), parts=",".join(map(str, parts)),
                    rank=rng.choice([8, 16, 24, 32, 40, 64, 128]), adapters=_log_int(rng, 1, min(rows, 32)),
                    mixed_ranks=rng.random() < 0.4, bare=rows > 1 and rng.random() < 0.4, segments=rng.random() < 0.5)
    if op == "verify":
        drafts = rng.randint(0, 8)
        vocab = _log_int(rng, 1000, 128256)
        most = 64 * 9 * 128256 // ((2 * drafts + 1) * vocab)
        return dict(_VERIFY, requests=_log_int(rng, 1, min(256, most)), drafts=drafts, vocab=vocab,
                    draft_logits=drafts > 0 and rng.random() < 0.6, ragged=rng.random() < 0.4,
                    masked=rng.random() < 0.3, greedy=rng.random() < 0.3)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    heads, kv_heads = rng.choice([(32, 8), (32, 8), (16, 16), (24, 8), (8, 1), (28, 4)])
    return dict(_QK, rows=_log_int(rng, 1, 8192 if dtype == "bf16" else 4096), heads=heads, kv_heads=kv_heads,
                dim=rng.choice([64, 128]), dtype=dtype, rotate=rng.random() < 0.7, scatter=rng.random() < 0.5)


# ------------------------------------------------------------------------ inputs

def _parts(case):
    return [int(x) for x in case["parts"].split(",")]


def _prepare_adapt(case, gen, bf16):
    T, K, parts, R, S = case["rows"], case["width"], _parts(case), case["rank"], case["adapters"]
    N, P = sum(parts), len(parts)

    def randn(*shape, std):
        return (torch.randn(*shape, device="cuda", generator=gen) * std).to(bf16)

    # every adapter has a row; the rest fall as they may, in runs (prefilled segments) or mixed (a decode step)
    ids = torch.cat([torch.arange(S, device="cuda"), torch.randint(0, S, (T - S,), device="cuda", generator=gen)])
    ids = ids.sort().values if case["segments"] else ids[torch.randperm(T, device="cuda", generator=gen)]
    if case["bare"]:
        ids = torch.where(torch.rand(T, device="cuda", generator=gen) < 0.25, torch.full_like(ids, -1), ids)
    ranks = torch.full((S,), R, device="cuda", dtype=torch.int32)
    if case["mixed_ranks"]:
        ranks = torch.randint(1, R + 1, (S,), device="cuda", generator=gen).to(torch.int32)
    a, b = randn(S, P, R, K, std=K ** -0.5), randn(S, N, R, std=0.3)
    keep = torch.arange(R, device="cuda") < ranks[:, None]  # a smaller rank is padded with zeros
    return dict(x=randn(T, K, std=1.0), base=randn(T, N, std=1.0), out=torch.empty(T, N, device="cuda", dtype=bf16),
                ids=ids.to(torch.int32), a=a * keep[:, None, :, None], b=b * keep[:, None, :],
                scale=torch.rand(S, device="cuda", generator=gen) + 0.5, ranks=ranks, parts=parts)


def _prepare_verify(case, gen):
    n, k, V = case["requests"], case["drafts"], case["vocab"]
    n_drafts = torch.full((n,), k, device="cuda", dtype=torch.int32)
    if case["ragged"]:
        n_drafts = torch.randint(0, k + 1, (n,), device="cuda", generator=gen).to(torch.int32)
    temperature = torch.rand(n, device="cuda", generator=gen) * 0.8 + 0.4
    if case["greedy"]:
        temperature[::4] = 0.0
    # packed rows: each request's follow those of the one before; rows past the last are room a server keeps
    row0 = (n_drafts + 1).cumsum(0) - (n_drafts + 1)
    draft_row0 = n_drafts.cumsum(0) - n_drafts
    target = torch.randn(n * (k + 1), V, device="cuda", generator=gen) * 2.5
    if case["masked"]:
        banned = torch.rand(n * (k + 1), V, device="cuda", generator=gen) < 0.5
        banned[:, V // 3] = False
        target = target.masked_fill(banned, -math.inf)
    s = dict(target=target, row0=row0.to(torch.int32), n_drafts=n_drafts, temperature=temperature, draft=None,
             draft_row0=None, drafts=None, u_accept=None,
             u_sample=torch.rand(n, device="cuda", generator=gen),
             accepted=torch.zeros(n, device="cuda", dtype=torch.int32),
             tokens=torch.zeros(n, k + 1, device="cuda", dtype=torch.int32),
             logprobs=torch.zeros(n, k + 1, device="cuda"))
    if k == 0:
        return s
    s["u_accept"] = torch.rand(n, k, device="cuda", generator=gen)
    at = (row0[:, None] + torch.arange(k, device="cuda")).clamp(max=n * (k + 1) - 1)
    if case["draft_logits"]:
        # a draft model is near its target; its drafts are drawn from its own distribution
        noise = torch.randn(n * k, V, device="cuda", generator=gen)
        draft = torch.empty(n * k, V, device="cuda")
        dat = (draft_row0[:, None] + torch.arange(k, device="cuda")).clamp(max=n * k - 1)
        live = torch.arange(k, device="cuda") < n_drafts[:, None]
        draft.copy_(noise * 2.5)
        draft[dat[live]] = target[at[live]] + noise[dat[live]] * 0.8
        heat = torch.where(temperature > 0, temperature, torch.full_like(temperature, 1e-3))
        races = -torch.log(torch.empty(n, k, V, device="cuda").exponential_(generator=gen))
        s["drafts"] = (draft[dat] / heat[:, None, None] + races).argmax(-1).to(torch.int32)
        s["draft"], s["draft_row0"] = draft, draft_row0.to(torch.int32)
    else:
        # drafts looked up in the documents: mostly the likeliest token, sometimes another
        top = target[at].argmax(-1)
        other = torch.randint(0, V, (n, k), device="cuda", generator=gen)
        s["drafts"] = torch.where(torch.rand(n, k, device="cuda", generator=gen) < 0.8, top, other).to(torch.int32)
    return s


def _prepare_qk(case, gen, bf16):
    T, hq, hkv, d = case["rows"], case["heads"], case["kv_heads"], case["dim"]
    dtype = bf16 if case["dtype"] == "bf16" else torch.float32
    fused = torch.randn(T, (hq + 2 * hkv) * d, device="cuda", generator=gen).to(dtype)  # one product's rows q | k | v
    R = T + 5 if case["scatter"] else T
    rows = torch.randperm(R, device="cuda", generator=gen)[:T].to(torch.int32) if case["scatter"] else None
    start = torch.randint(0, 120000, (1,), device="cuda", generator=gen)
    gains = [(1 + 0.1 * torch.randn(d, device="cuda", generator=gen)).to(dtype) for _ in range(2)]
    return dict(q=fused[:, :hq * d].view(T, hq, d), k=fused[:, hq * d:(hq + hkv) * d].view(T, hkv, d),
                v=fused[:, (hq + hkv) * d:].view(T, hkv, d), q_gain=gains[0], k_gain=gains[1], rows=rows,
                positions=(start + torch.arange(T, device="cuda")).to(torch.int32) if case["rotate"] else None,
                q_out=torch.zeros(R, hq, d, device="cuda", dtype=dtype),
                k_out=torch.zeros(R, hkv, d, device="cuda", dtype=dtype),
                v_out=torch.zeros(R, hkv, d, device="cuda", dtype=dtype))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] == "adapt":
        return dict(_prepare_adapt(case, gen, torch.bfloat16), op="adapt")
    if case["op"] == "verify":
        return dict(_prepare_verify(case, gen), op="verify")
    return dict(_prepare_qk(case, gen, torch.bfloat16), op="qk")


# ------------------------------------------------------------------------ plain forms

def _plain_adapt(s):
    """Every adapter's product for every row, the others' masked out: two dense products for each part."""
    S, P, R, K = s["a"].shape
    mine = (s["ids"][:, None] == torch.arange(S, device="cuda")) * s["scale"]
    h = (s["x"].float() @ s["a"].float().view(S * P * R, K).T).view(-1, S, P, R)
    h = h * mine[:, :, None, None] * (torch.arange(R, device="cuda") < s["ranks"][:, None])[:, None, :]
    b = s["b"].float().split(s["parts"], dim=1)
    delta = [h[:, :, p].reshape(-1, S * R) @ b[p].permute(0, 2, 1).reshape(S * R, -1) for p in range(P)]
    s["out"].copy_(s["base"].float() + torch.cat(delta, dim=1))
    return s["out"]


def _softmax64(x, c):
    z = x.double() * c[:, None, None]
    w = torch.exp(z - z.amax(-1, keepdim=True))
    return w / w.sum(-1, keepdim=True)


def _plain_verify(s):
    # in 64 bits: a token's border in the running sum of 128 k weights lies closer than 32 bits tell apart
    n, k1 = s["tokens"].shape
    k, rows = k1 - 1, s["target"].shape[0]
    j = torch.arange(k1, device="cuda")
    x = s["target"][(s["row0"][:, None] + j).clamp(max=rows - 1)]
    hot = s["temperature"] > 0
    c = torch.where(hot, 1 / s["temperature"], 1.0).double()
    p = _softmax64(x, c)
    V = x.shape[-1]
    ids = torch.arange(V, device="cuda")
    best = torch.where(x == x.amax(-1, keepdim=True), ids, V).amin(-1)
    a = torch.zeros(n, device="cuda", dtype=torch.long)
    r = p[:, 0]
    if k:
        drafts = s["drafts"].long()
        live = j[:k] < s["n_drafts"][:, None]
        pd = p[:, :k].gather(-1, drafts[..., None])[..., 0]
        if s["draft"] is not None:
            q = _softmax64(s["draft"][(s["draft_row0"][:, None] + j[:k]).clamp(max=s["draft"].shape[0] - 1)], c)
            qd = q.gather(-1, drafts[..., None])[..., 0]
        else:
            qd = torch.ones_like(pd)
        keep = torch.where(hot[:, None], s["u_accept"].double() * qd < pd, drafts == best[:, :k]) & live
        a = keep.int().cumprod(1).sum(1).long()
        at = a.clamp(max=k - 1)[:, None]
        if s["draft"] is not None:
            qa = q.gather(1, at[..., None].expand(-1, -1, V))[:, 0]
        else:
            qa = (ids == drafts.gather(1, at)).double()
        pa = p.gather(1, a[:, None, None].expand(-1, -1, V))[:, 0]
        r = (pa - qa * (a < s["n_drafts"])[:, None]).clamp(min=0)
        r = torch.where(r.sum(-1, keepdim=True) > 0, r, pa)
    cum = r.cumsum(-1)
    pick = (cum <= s["u_sample"].double()[:, None] * cum[:, -1:]).sum(-1).clamp(max=V - 1)
    pick = torch.where(hot, pick, best.gather(1, a[:, None])[:, 0])
    tokens = torch.full_like(s["tokens"], -1, dtype=torch.long)
    if k:
        tokens[:, :k] = torch.where(j[:k] < a[:, None], drafts, tokens[:, :k])
    tokens.scatter_(1, a[:, None], pick[:, None])
    lp = torch.log(p.gather(-1, tokens.clamp(min=0)[..., None])[..., 0])
    s["accepted"].copy_(a)
    s["tokens"].copy_(tokens)
    s["logprobs"].copy_(torch.where(tokens >= 0, lp, 0.0))
    return s["accepted"], s["tokens"], s["logprobs"]


def _plain_head(x, gain, positions):
    d = x.shape[-1]
    y = x.float()
    y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * gain.float()
    if positions is not None:
        inv = THETA ** (torch.arange(d // 2, device="cuda", dtype=torch.float64) * (-2.0 / d))
        angle = positions.double()[:, None] * inv  # far positions: 32 bits lose the angle
        cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
        lo, hi = y[..., :d // 2], y[..., d // 2:]
        y = torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], dim=-1)
    return y


def _plain_qk(s):
    q, k = _plain_head(s["q"], s["q_gain"], s["positions"]), _plain_head(s["k"], s["k_gain"], s["positions"])
    rows = s["rows"].long() if s["rows"] is not None else torch.arange(q.shape[0], device="cuda")
    s["q_out"][rows] = q.to(s["q_out"].dtype)
    s["k_out"][rows] = k.to(s["k_out"].dtype)
    s["v_out"][rows] = s["v"]
    return s["q_out"], s["k_out"], s["v_out"]


def _own(s):
    import paper_2511_02749_amd as spanq
    if s["op"] == "adapt":
        spanq.adapter_apply(s["x"], s["base"], s["ids"], s["a"], s["b"], s["scale"], s["out"], parts=s["parts"],
                            ranks=s["ranks"])
        return s["out"]
    if s["op"] == "verify":
        spanq.verify_drafts(s["target"], s["drafts"], s["u_accept"], s["u_sample"], s["temperature"], s["accepted"],
                            s["tokens"], draft_logits=s["draft"], n_drafts=s["n_drafts"], row0=s["row0"],
                            draft_row0=s["draft_row0"], logprobs=s["logprobs"])
        return s["accepted"], s["tokens"], s["logprobs"]
    spanq.qk_norm_rope(s["q"], s["k"], s["v"], s["q_gain"], s["k_gain"], EPS, s["q_out"], s["k_out"], s["v_out"],
                       rows=s["rows"], positions=s["positions"], rope_theta=THETA)
    return s["q_out"], s["k_out"], s["v_out"]


def run(state):
    if own:
        return _own(state)
    return {"adapt": _plain_adapt, "verify": _plain_verify, "qk": _plain_qk}[state["op"]](state)


# ------------------------------------------------------------------------ what a pass needs

def work(case):
    if case["op"] == "adapt":
        T, K, parts, R, S = case["rows"], case["width"], _parts(case), case["rank"], case["adapters"]
        N, P = sum(parts), len(parts)
        if case["mixed_ranks"]:
            R = (R + 1) / 2  # on average
        return {"bytes": 2 * T * (K + 2 * N) + 2 * S * R * (P * K + N) + 4 * T + 8 * S,
                "flops": 2 * T * R * (P * K + N)}
    if case["op"] == "verify":
        n, k, V = case["requests"], case["drafts"], case["vocab"]
        if case["ragged"]:
            k = k / 2  # on average
        logits = n * V * (k + 1 + (k if case["draft_logits"] else 0))
        return {"bytes": 4 * logits + 4 * n * (5 * k + 8), "flops": 25 * logits}
    T, H = case["rows"], case["heads"] + 2 * case["kv_heads"]
    size = 2 if case["dtype"] == "bf16" else 4
    return {"bytes": 2 * size * T * H * case["dim"] + 8 * T, "flops": 10 * T * H * case["dim"]}


# ------------------------------------------------------------------------ in 64 bits, from the definitions

def _exact_adapt(s):
    out = s["base"].double()
    for i in range(s["a"].shape[0]):
        mine = (s["ids"] == i).nonzero()[:, 0]
        rank, col = int(s["ranks"][i]), 0
        for p, width in enumerate(s["parts"]):
            low = s["x"][mine].double() @ s["a"][i, p, :rank].double().T
            out[mine, col:col + width] += s["scale"][i].double() * (low @ s["b"][i, col:col + width, :rank].double().T)
            col += width
    return out


def _exact_verify(s):
    """Request by request on the host: the tokens are whole numbers, their log-probabilities computed ones."""
    cut = {key: v.cpu().numpy() if isinstance(v, torch.Tensor) else v for key, v in s.items()}
    lp = np.zeros(cut["logprobs"].shape)
    for i in range(lp.shape[0]):
        heat = float(cut["temperature"][i])
        greedy, heat = heat <= 0, heat if heat > 0 else 1.0
        r0, nd = int(cut["row0"][i]), int(cut["n_drafts"][i])

        def dist(row):
            w = np.exp((row.astype(np.float64) - row.max().astype(np.float64)) / heat)
            return w / w.sum()

        for j in range(nd + 1):
            p = dist(cut["target"][r0 + j])
            left = p
            if j < nd:
                d = int(cut["drafts"][i, j])
                q = np.zeros_like(p)
                if cut["draft"] is None:
                    q[d] = 1.0
                else:
                    q = dist(cut["draft"][int(cut["draft_row0"][i]) + j])
                if (int(np.argmax(p)) == d) if greedy else (float(cut["u_accept"][i, j]) * q[d] < p[d]):
                    lp[i, j] = math.log(p[d])
                    continue
                left = np.maximum(p - q, 0)
            run_sum = np.cumsum(left)
            token = int(np.argmax(p)) if greedy else int(np.searchsorted(
                run_sum, float(cut["u_sample"][i]) * run_sum[-1], side="right"))
            lp[i, j] = math.log(p[token])
            break
    return None, None, torch.from_numpy(lp)


def _exact_qk(s):
    def head(x, gain, out):
        x, d = x.double(), x.shape[-1]
        norm = x / (x.pow(2).sum(-1, keepdim=True) / d + EPS).sqrt() * gain.double()
        if s["positions"] is not None:
            pair = torch.complex(norm[..., :d // 2], norm[..., d // 2:])
            turn = s["positions"].double()[:, None] * torch.exp(
                -math.log(THETA) * 2 * torch.arange(d // 2, device=x.device, dtype=torch.float64) / d)
            pair = pair * torch.polar(torch.ones_like(turn), turn)[:, None]
            norm = torch.cat([pair.real, pair.imag], -1)
        full = out.double() * 0
        full[slice(None) if s["rows"] is None else s["rows"].long()] = norm
        return full

    v = s["v_out"].double() * 0
    v[slice(None) if s["rows"] is None else s["rows"].long()] = s["v"].double()
    return head(s["q"], s["q_gain"], s["q_out"]), head(s["k"], s["k_gain"], s["k_out"]), v


def exact(case, seed):
    s = prepare(case, seed)
    return {"adapt": _exact_adapt, "verify": _exact_verify, "qk": _exact_qk}[case["op"]](s)
