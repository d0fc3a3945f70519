"""GPU parity of the row operators against their formulas in float64.

Bounds, per element, u = 2^-24 (a float32 rounding), r = 2^-8 (bf16 out) or 2^-24 (float32 out):
- head norms with rotation: the sum of D squares is within D u of itself, its root within half
  that; the norm, the gain, the angle's and the sine's rounding and the rotation's three
  operations add at most 16 u of the pair's length.  |y - exact| <= r |exact| + (1 + r) (D/2 + 16) u |pair|.
- adapters: h = sum of K products, any order: within K u sum|x a|; its two bf16 parts hold it to 2^-16; the
  second product's 2 R terms add 2 R u sum|b h|, scale and base two roundings.
  |y - exact| <= 2^-8 |exact| + (1 + 2^-8) (s (sum_r |b_r| dh_r + 2 R u sum_r |b_r| (|h_r| + dh_r)) + 2 u (|exact| + |base|)),
  dh_r = K u sum_k|x_k a_rk| + 2^-16 |h_r|.
- verification: 64-bit sums of V weights are within V 2^-53 of themselves, a weight within 2^-46 (its
  series) of itself: a decision may differ from the oracle's only where the two sides are closer than
  d = V 2^-52 + 2^-44 relative to the whole.  Log-probabilities: 2^-24 |lp| + d + 2^-40.
"""
import numpy as np
import pytest

import paper_2511_02749_amd as spanq

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
U = 2.0 ** -24


@pytest.fixture(autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    print(flush=True)
    yield
    if torch.cuda.memory_reserved() > 8 << 30:  # for the pools of other tests
        torch.cuda.empty_cache()


def _gen(seed):
    return torch.Generator().manual_seed(seed)


# ------------------------------------------------------------------------ head norms

def _heads_exact(x, gain, eps, positions, theta):
    """(result, length of each value's pair) in float64 on the CPU."""
    x = x.double()
    d = x.shape[-1]
    if gain is not None:
        x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / d + eps) * gain.double()
    lo, hi = x[..., :d // 2], x[..., d // 2:]
    length = torch.sqrt(lo * lo + hi * hi).repeat(1, 1, 2)
    if positions is not None:
        f = theta ** (-2.0 * torch.arange(d // 2, dtype=torch.float64) / d)
        t = (positions.double()[:, None] * f)[:, None]
        x = torch.cat([lo * torch.cos(t) - hi * torch.sin(t), hi * torch.cos(t) + lo * torch.sin(t)], -1)
    return x, length


def _check_heads(got, x, gain, eps, positions, theta, what):
    ref, length = _heads_exact(x, gain, eps, positions, theta)
    r = 2.0 ** -8 if got.dtype == torch.bfloat16 else U
    err = (got.double() - ref).abs()
    bound = r * ref.abs() + (1 + r) * (x.shape[-1] / 2 + 16) * U * length
    print(f"{what}: max err {err.max():.3g}, worst err/bound {(err / bound.clamp(min=1e-300)).max():.3g}", flush=True)
    assert bool((err <= bound).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("rows,hq,hkv,rotate,scatter", [
    (1, 32, 8, False, False), (1, 1, 1, True, True), (3, 24, 8, True, False), (257, 8, 1, True, True),
    (1025, 3, 3, False, True), (64, 28, 4, True, False)])
def test_head_norms(dtype, dim, rows, hq, hkv, rotate, scatter):
    g = _gen(rows + dim)
    eps, theta = 1e-5, 1e4
    fused = torch.randn(rows, (hq + 2 * hkv) * dim + 16, generator=g).to(dtype)  # rows with a gap behind them
    gains = [(1 + 0.3 * torch.randn(dim, generator=g)).to(dtype) for _ in range(2)]
    pos = torch.randint(-50, 200000, (rows,), generator=g).to(torch.int32) if rotate else None
    out_rows = rows + 3 if scatter else rows
    to = torch.randperm(out_rows, generator=g)[:rows].to(torch.int32) if scatter else None
    fd = fused.cuda()
    q, k, v = (fd[:, a * dim:b * dim].view(rows, b - a, dim) for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv)))
    outs = [torch.full((out_rows, h, dim), 7.0, dtype=dtype, device="cuda") for h in (hq, hkv, hkv)]
    print(f"head norms {dtype} dim {dim} rows {rows} heads {hq}/{hkv} rotate {rotate} scatter {scatter}", flush=True)
    spanq.qk_norm_rope(q, k, v, gains[0].cuda(), gains[1].cuda(), eps, *outs, rows=None if to is None else to.cuda(),
                       positions=None if pos is None else pos.cuda(), rope_theta=theta)
    at = torch.arange(rows) if to is None else to.long()
    got = [o.cpu() for o in outs]
    cpu = [t.cpu() for t in (q, k, v)]
    _check_heads(got[0][at], cpu[0], gains[0], eps, pos, theta, "q")
    _check_heads(got[1][at], cpu[1], gains[1], eps, pos, theta, "k")
    assert torch.equal(got[2][at], cpu[2])
    left = torch.ones(out_rows, dtype=torch.bool)
    left[at] = False
    assert all(bool((o[left] == 7.0).all()) for o in got)  # rows that none names
    assert torch.equal(fd.cpu(), fused)


def test_head_norms_parts_in_place_and_rows_outside():
    g = _gen(5)
    x = torch.randn(9, 4, 128, generator=g).to(torch.bfloat16)
    gain = torch.rand(128, generator=g).to(torch.bfloat16)
    d, gd = x.cuda(), gain.cuda()
    spanq.qk_norm_rope(d, None, None, gd, None, 1e-6, d, None, None)  # in place, queries alone
    _check_heads(d.cpu(), x, gain, 1e-6, None, 1e4, "in place")
    # only rotated, keys alone; the inverse rotation gives the keys back within two roundings
    pos = torch.arange(9, dtype=torch.int32) * 1000
    k, y = x.cuda(), torch.empty(9, 4, 128, dtype=torch.bfloat16, device="cuda")
    spanq.qk_norm_rope(None, k, None, None, None, 0.0, None, y, None, positions=pos.cuda(), rope_theta=5e5)
    _check_heads(y.cpu(), x, None, 0.0, pos, 5e5, "rotated only")
    # a row outside the output is not written, the others are
    rows = torch.tensor([2, -1, 0, 9, 1 << 30, 4, -2 ** 31, 5, 3], dtype=torch.int32)
    v, o = x.cuda(), torch.full((9, 4, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    spanq.qk_norm_rope(None, None, v, None, None, 0.0, None, None, o, rows=rows.cuda())
    o = o.cpu()
    for i, r in enumerate(rows.tolist()):
        if 0 <= r < 9:
            assert torch.equal(o[r], x[i])
    assert all(bool((o[r] == 3.0).all()) for r in (1, 6, 7, 8))


def test_head_norms_of_zero_and_nonfinite_heads():
    x = torch.randn(4, 2, 64, generator=_gen(1))
    x[0, 0] = 0.0
    x[1, 1, 5] = float("nan")
    x[2, 0, 63] = float("inf")
    gain = torch.ones(64)
    y = torch.empty_like(x, device="cuda")
    spanq.qk_norm_rope(x.cuda(), None, None, gain.cuda(), None, 1e-5, y, None, None,
                       positions=torch.arange(4, dtype=torch.int32).cuda())
    y = y.cpu()
    assert bool((y[0, 0] == 0).all())
    assert bool(torch.isnan(y[1, 1]).all())  # the whole head: its norm is no number
    fine = torch.ones(4, 2, dtype=torch.bool)
    fine[1, 1] = fine[2, 0] = False
    assert bool(torch.isfinite(y[fine]).all())
    ref, _ = _heads_exact(torch.where(torch.isfinite(x), x, 0.0), gain, 1e-5, torch.arange(4), 1e4)
    assert float((y.double() - ref)[fine].abs().max()) < 1e-5


def test_head_norms_of_more_rows_than_a_grid_takes():
    n, d = (1 << 24) + 3, 64
    x = torch.randn(n, 1, d, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda", dtype=torch.bfloat16)
    gain = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    y = torch.zeros_like(x)
    spanq.qk_norm_rope(x, None, None, gain, None, 1e-5, y, None, None)
    for rows in (slice(0, 100), slice((1 << 24) - 50, n)):  # both ends of the first launch, and the second
        _check_heads(y[rows].cpu(), x[rows].cpu(), gain.cpu(), 1e-5, None, 1e4, str(rows))
    assert bool((y != 0).any(-1).all())


# ------------------------------------------------------------------------ adapters

def _adapt_exact(x, base, ids, a, b, scale, ranks, parts):
    """(result, bound) in float64 on the CPU."""
    x, ref = x.double(), base.double().clone()
    K, R = x.shape[1], a.shape[2]
    slack = torch.zeros_like(ref)
    for i in set(ids.tolist()):
        if not 0 <= i < a.shape[0]:
            continue
        mine = (ids == i).nonzero()[:, 0]
        rank, col, s = int(ranks[i]), 0, float(scale[i])
        for p, w in enumerate(parts):
            aa, bb = a[i, p, :rank].double(), b[i, col:col + w, :rank].double()
            h = x[mine] @ aa.T
            dh = K * U * (x[mine].abs() @ aa.abs().T) + 2.0 ** -16 * h.abs()
            ref[mine, col:col + w] += s * (h @ bb.T)
            slack[mine, col:col + w] = abs(s) * (dh @ bb.abs().T + 2 * R * U * ((h.abs() + dh) @ bb.abs().T))
            col += w
    slack = (1 + 2.0 ** -8) * (slack + 2 * U * (ref.abs() + base.double().abs())) + 2.0 ** -8 * ref.abs()
    return ref, slack


def _adapt_case(T, K, parts, R, S, seed, ids=None, pad=True):
    g = _gen(seed)
    N = sum(parts)
    x = torch.randn(T, K, generator=g).to(torch.bfloat16)
    base = torch.randn(T, N, generator=g).to(torch.bfloat16)
    ids = torch.randint(-1, S, (T,), generator=g).to(torch.int32) if ids is None else torch.tensor(ids, dtype=torch.int32)
    ranks = torch.randint(0, R + 1, (S,), generator=g).to(torch.int32)
    ranks[0] = R
    a = (torch.randn(S, len(parts), R, K, generator=g) / K ** 0.5).to(torch.bfloat16)
    b = torch.randn(S, N, R, generator=g).to(torch.bfloat16)
    if pad:  # what lies past a rank does not count
        past = torch.arange(R) >= ranks[:, None]
        a = torch.where(past[:, None, :, None], torch.full_like(a, float("nan")), a)
        b = torch.where(past[:, None, :], torch.full_like(b, float("inf")), b)
    scale = torch.rand(S, generator=g) * 2 - 0.5
    return x, base, ids, a, b, scale, ranks


def _check_adapt(got, case, parts, what):
    ref, bound = _adapt_exact(*case, parts)
    err = (got.double() - ref).abs()
    print(f"{what}: max err {err.max():.3g}, worst err/bound {(err / bound.clamp(min=1e-300)).max():.3g}", flush=True)
    assert bool((err <= bound).all())
    none = (case[2] < 0) | (case[2] >= case[3].shape[0])
    assert torch.equal(got[none], case[1][none])  # rows without an adapter, bit for bit


@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 100, 256, 257, 300, 1031])
@pytest.mark.parametrize("K,parts,R,S", [(64, (8,), 8, 1), (520, (264, 24, 512), 24, 5), (2048, (1000, 1000), 16, 40)])
def test_adapters(T, K, parts, R, S):
    case = _adapt_case(T, K, parts, R, S, seed=T + K)
    print(f"adapters T {T} K {K} parts {parts} R {R} S {S}", flush=True)
    d = [t.cuda() for t in case]
    out = torch.full((T, sum(parts)), float("nan"), dtype=torch.bfloat16, device="cuda")
    spanq.adapter_apply(d[0], d[1], d[2], d[3], d[4], d[5], out, parts=parts, ranks=d[6])
    _check_adapt(out.cpu(), case, parts, "out")
    spanq.adapter_apply(d[0], d[1], d[2], d[3], d[4], d[5], d[1], parts=parts, ranks=d[6])  # in place
    assert torch.equal(d[1], out)


@pytest.mark.parametrize("T,K,parts,R,S", [(1, 8, (8, 8, 8, 8), 128, 3), (33, 14336, (64,), 64, 4), (5, 4104, (4096, 1024, 1024), 40, 5),
                                           (600, 1000, (16, 8), 128, 9), (31, 24, (2056,), 120, 31)])
def test_adapters_long_reductions_large_ranks_odd_widths(T, K, parts, R, S):
    case = _adapt_case(T, K, parts, R, S, seed=T + R)
    print(f"adapters T {T} K {K} parts {parts} R {R} S {S}", flush=True)
    d = [t.cuda() for t in case]
    out = torch.empty_like(d[1])
    spanq.adapter_apply(d[0], d[1], d[2], d[3], d[4], d[5], out, parts=parts, ranks=d[6])
    _check_adapt(out.cpu(), case, parts, "out")


@pytest.mark.parametrize("T,K,parts,R,S", [(200, 2048, (8200, 1000), 24, 5), (600, 4096, (264,), 128, 3), (1031, 520, (4104,), 40, 4),
                                           (1100, 2048, (8, 8200), 16, 2), (2100, 264, (4096,), 8, 30), (1500, 8200, (520, 4104, 8), 120, 7),
                                           (700, 1032, (8200,), 56, 6)])
def test_adapters_of_many_rows_and_columns(T, K, parts, R, S):
    """Wide products, large ranks and runs of tiles: mixed rows, and segments."""
    for ids in (None, [i * S // T - (i % 97 == 5) for i in range(T)]):
        case = _adapt_case(T, K, parts, R, S, seed=T + R, ids=ids)
        print(f"adapters T {T} K {K} parts {parts} R {R} S {S}", flush=True)
        d = [t.cuda() for t in case]
        out = torch.empty_like(d[1])
        spanq.adapter_apply(d[0], d[1], d[2], d[3], d[4], d[5], out, parts=parts, ranks=d[6])
        _check_adapt(out.cpu(), case, parts, "out")
        spanq.adapter_apply(d[0], d[1], d[2], d[3], d[4], d[5], d[1], parts=parts, ranks=d[6])  # in place
        assert torch.equal(d[1], out)


@pytest.mark.parametrize("T", [40, 300])
def test_adapters_strides_ids_outside_and_no_adapter_at_all(T):
    parts, S = (72, 16), 3
    ids = [(0, 2, -1, 3, 1 << 30, -2 ** 31, 1, 2)[i % 8] for i in range(T)]
    case = _adapt_case(T, 136, parts, 16, S, seed=T, ids=ids)
    x, base, out = (torch.full((T + 2, w + 40), 9.0, dtype=torch.bfloat16, device="cuda") for w in (136, 88, 88))
    x[1:-1, 8:144] = case[0].cuda()
    base[1:-1, 16:104] = case[1].cuda()
    d = [t.cuda() for t in case]
    xv, bv, ov = x[1:-1, 8:144], base[1:-1, 16:104], out[1:-1, 24:112]
    spanq.adapter_apply(xv, bv, d[2], d[3], d[4], d[5], ov, parts=parts, ranks=d[6])
    _check_adapt(ov.cpu(), case, parts, "strided")
    frame = out.clone()
    frame[1:-1, 24:112] = 9.0
    assert bool((frame == 9.0).all())  # nothing around the rows was written
    # no scale, no ranks
    clean = _adapt_case(T, 136, parts, 16, S, seed=T, ids=ids, pad=False)
    one = (clean[0], clean[1], clean[2], clean[3], clean[4], torch.ones(S), torch.full((S,), 16))
    spanq.adapter_apply(xv, bv, d[2], clean[3].cuda(), clean[4].cuda(), None, ov, parts=parts)
    _check_adapt(ov.cpu(), one, parts, "no scale")
    # rows that all go without
    none = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    spanq.adapter_apply(xv, bv, none, d[3], d[4], d[5], ov, parts=parts, ranks=d[6])
    assert torch.equal(ov, bv)
    spanq.adapter_apply(xv, bv, d[2], d[3][:0], d[4][:0], d[5][:0], ov, parts=parts, ranks=d[6][:0])
    assert torch.equal(ov, bv)


@pytest.mark.parametrize("T", [48, 320])
def test_adapter_rows_do_not_reach_each_other(T):
    """A row that holds NaN or inf, or whose adapter does, changes no other row, and a row's
    result is the same bits wherever it lies in the call."""
    parts, S = (128,), 4
    case = _adapt_case(T, 256, parts, 16, S, seed=T, pad=False, ids=[i % 4 for i in range(T)])
    d = [t.cuda() for t in case]
    out = torch.empty_like(d[1])
    spanq.adapter_apply(d[0], d[1], d[2], d[3], d[4], d[5], out)
    perm = torch.randperm(T, generator=_gen(2)).cuda()
    moved = torch.empty_like(out)
    spanq.adapter_apply(d[0][perm].contiguous(), d[1][perm].contiguous(), d[2][perm].contiguous(), d[3], d[4], d[5], moved)
    assert torch.equal(moved, out[perm])
    x, a = d[0].clone(), d[3].clone()
    x[5, 100] = float("nan")
    x[9, 3] = float("inf")
    a[3, 0, 2, 7] = float("inf")
    hurt = torch.empty_like(out)
    spanq.adapter_apply(x, d[1], d[2], a, d[4], d[5], hurt)
    fine = torch.ones(T, dtype=torch.bool, device="cuda")
    fine[5] = fine[9] = False
    fine &= d[2] != 3
    assert torch.equal(hurt[fine], out[fine])
    assert bool(torch.isnan(hurt[5]).all()) and not bool(torch.isfinite(hurt[9]).any())


def test_adapters_in_a_graph_follow_their_ids_and_share_no_workspace():
    parts, S, T = (256,), 6, 24
    case = _adapt_case(T, 512, parts, 16, S, seed=3, pad=False)
    d = [t.cuda() for t in case]
    outs = [torch.empty_like(d[1]) for _ in range(2)]
    ids = [d[2].clone(), d[2].flip(0).contiguous()]
    ws = [torch.empty(spanq.adapter_workspace(T, 512, 16, parts), dtype=torch.uint8, device="cuda") for _ in range(2)]
    graphs = []
    torch.cuda.synchronize()
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            spanq.adapter_apply(d[0], d[1], ids[i], d[3], d[4], d[5], outs[i], workspace=ws[i])
        graphs.append(g)
    side = torch.cuda.Stream()
    want = torch.empty_like(d[1])
    for step in range(4):
        for i in range(2):
            ids[i].copy_(torch.randint(-1, S, (T,), generator=_gen(10 * step + i)).to(torch.int32))
        torch.cuda.synchronize()
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
        torch.cuda.synchronize()
        for i in range(2):
            spanq.adapter_apply(d[0], d[1], ids[i], d[3], d[4], d[5], want)
            assert torch.equal(want, outs[i]), (step, i)


@pytest.mark.parametrize("T,S", [(300, 6), (700, 2100), (129, 40), (70000, 9)])
def test_adapters_of_many_mixed_rows_in_a_graph(T, S):
    """Rows ordered by adapter on the device: more adapters than a work-group counts apart, more
    rows than are worked at once, ids that change between replays, runs of one adapter."""
    parts = (8, 8200) if T == 129 else (8,)
    case = _adapt_case(T, 16, parts, 8, S, seed=T)
    print(f"mixed adapters T {T} S {S}", flush=True)
    d = [t.cuda() for t in case]
    out, want = torch.empty_like(d[1]), torch.empty_like(d[1])
    ids = d[2].clone()
    ws = torch.empty(spanq.adapter_workspace(T, 16, 8, parts), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        spanq.adapter_apply(d[0], d[1], ids, d[3], d[4], d[5], out, parts=parts, ranks=d[6], workspace=ws)
    at = torch.arange(T)
    for i, new in enumerate((case[2], case[2].sort().values, torch.full((T,), S - 1), at // 65 % S, at * 1023 % S - 1)):
        ids.copy_(new.to(torch.int32))
        out.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        _check_adapt(out.cpu(), (case[0], case[1], new.to(torch.int32)) + case[3:], parts, f"ids {i}")
        spanq.adapter_apply(d[0], d[1], ids, d[3], d[4], d[5], want, parts=parts, ranks=d[6])
        assert torch.equal(want, out)


def test_a_workspace_serves_smaller_calls():
    parts, S, R, K, V = (520,), 5, 24, 512, 5000
    ws = torch.empty(spanq.adapter_workspace(900, K, R, parts), dtype=torch.uint8, device="cuda")
    vs = torch.empty(spanq.verify_workspace(90, 4, V), dtype=torch.uint8, device="cuda")
    for T in (900, 257, 256, 130, 1):
        case = _adapt_case(T, K, parts, R, S, seed=T)
        d = [t.cuda() for t in case]
        out = torch.empty_like(d[1])
        spanq.adapter_apply(d[0], d[1], d[2], d[3], d[4], d[5], out, parts=parts, ranks=d[6], workspace=ws)
        _check_adapt(out.cpu(), case, parts, f"{T} rows")
    for n in (90, 30, 1):
        t = torch.randn(n * 5, V, device="cuda")
        u = torch.rand(n, 4, device="cuda")
        acc, tok = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, 5, dtype=torch.int32, device="cuda")
        d = t.view(n, 5, V)[:, :4].argmax(-1).to(torch.int32)
        spanq.verify_drafts(t, d, u * 0, u[:, 0].contiguous(), None, acc, tok, workspace=vs)
        assert bool((acc == 4).all()) and torch.equal(tok[:, :4], d)  # 0 < p keeps them all


def test_row_operators_on_another_stream():
    """Work on a stream of its own, workspace taken there, ordered by an event alone."""
    side = torch.cuda.Stream()
    case = _adapt_case(64, 1024, (512,), 16, 8, seed=4, pad=False)
    x, base, ids, a, b, scale, ranks = [t.cuda() for t in case]
    logits = torch.randn(6, 5000, generator=_gen(1)).cuda()
    u, heat = torch.rand(6, generator=_gen(2)).cuda(), torch.ones(6, device="cuda")
    want, wt, wa = torch.empty_like(base), torch.empty(6, 1, dtype=torch.int32, device="cuda"), torch.empty(6, dtype=torch.int32, device="cuda")
    spanq.adapter_apply(x, base, ids, a, b, scale, want)
    spanq.verify_drafts(logits, None, None, u, heat, wa, wt)
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        out, tok, acc = torch.zeros_like(base), torch.zeros_like(wt), torch.zeros_like(wa)
        side.wait_stream(torch.cuda.current_stream())
        spanq.adapter_apply(x, base, ids, a, b, scale, out, stream=stream)
        spanq.verify_drafts(logits, None, None, u, heat, acc, tok, stream=stream)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(out, want) and torch.equal(tok, wt)


# ------------------------------------------------------------------------ verification

class _Oracle:
    """The rule, request by request, in float64; what the kernel answers is followed, and each of its
    decisions must be the oracle's or lie closer to the border than 64-bit sums can tell."""

    def __init__(self, V):
        self.d = V * 2.0 ** -52 + 2.0 ** -44

    @staticmethod
    def dist(row, heat):
        x = row.astype(np.float64)
        x = np.where(np.isnan(x), -np.inf, x)
        m = x.max() if x.size else -np.inf
        if m == -np.inf:
            return np.zeros(x.shape)
        with np.errstate(invalid="ignore", over="ignore"):
            w = np.where(x == m, 1.0, np.exp((x - m) / heat))
        return w / w.sum()

    def check(self, target, draft, drafts, ua, us, heat, accepted, tokens, logprobs, what):
        """One request: target [n + 1][V], draft [n][V] or None, drafts [n]; outputs padded to k + 1."""
        n, V = len(drafts), target.shape[1]
        greedy = not heat > 0
        heat = 1.0 if greedy else heat
        lp = []
        for j in range(n + 1):
            p = self.dist(target[j], heat)
            left = p
            if j < n:
                t = int(drafts[j])
                inside = 0 <= t < V
                pd = p[t] if inside else 0.0
                if greedy:
                    keep, near = inside and pd > 0 and t == int(np.argmax(p)), False
                else:
                    q = self.dist(draft[j], heat) if draft is not None else None
                    qd = (q[t] if inside else 0.0) if q is not None else 1.0
                    keep = float(ua[j]) * qd < pd
                    near = abs(float(ua[j]) * qd - pd) <= self.d * max(pd, qd)
                kept = j < accepted
                assert kept == keep or near, (what, j, kept, keep)
                if kept:
                    assert tokens[j] == t, (what, j)
                    lp.append(np.log(pd))
                    continue
                if not greedy:
                    if q is None:
                        left = p.copy()
                        if inside:
                            left[t] = 0.0
                    else:
                        left = np.maximum(p - q, 0.0)
                    if not left.sum() > 0:
                        left = p
            assert accepted == j, (what, accepted, j)
            token = int(tokens[j])
            if not p.sum() > 0:
                assert token == -1, what
                lp.append(0.0)
            elif greedy:
                assert token == int(np.argmax(p)), (what, token, int(np.argmax(p)))
                lp.append(np.log(p[token]))
            else:
                assert 0 <= token < V and left[token] > 0, (what, token)
                run = np.cumsum(left)
                aim, slack = min(float(us), 1.0) * run[-1], 4 * self.d * max(run[-1], p.sum())
                before = run[token - 1] if token else 0.0
                assert before <= aim + slack and aim < run[token] + slack, (what, token, before, aim, run[token])
                lp.append(np.log(p[token]))
            break
        lp = np.array(lp + [0.0] * (len(tokens) - len(lp)))
        assert list(tokens[accepted + 1:]) == [-1] * (len(tokens) - accepted - 1), what
        assert np.all(np.abs(logprobs - lp) <= U * np.abs(lp) + self.d + 2.0 ** -40), (what, logprobs, lp)


def _verify_and_check(target, draft, drafts, n_drafts, ua, us, heat, row0, drow0, k, what, target_dev=None, draft_dev=None):
    n = len(us)
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    acc = torch.full((n,), 99, dtype=torch.int32, device="cuda")
    tok = torch.full((n, k + 1), 99, dtype=torch.int32, device="cuda")
    lp = torch.full((n, k + 1), 99.0, device="cuda")
    print(what, flush=True)
    spanq.verify_drafts(dev(target) if target_dev is None else target_dev, dev(drafts) if k else None,
                        dev(ua) if k else None, us.cuda(), dev(heat), acc, tok,
                        draft_logits=dev(draft) if draft_dev is None else draft_dev, n_drafts=dev(n_drafts),
                        row0=dev(row0), draft_row0=dev(drow0), logprobs=lp)
    acc, tok, lp = acc.cpu().numpy(), tok.cpu().numpy(), lp.cpu().numpy()
    oracle = _Oracle(target.shape[1])
    kept = 0
    for i in range(n):
        nd = k if n_drafts is None else min(max(int(n_drafts[i]), 0), k)
        r = i * (k + 1) if row0 is None else int(row0[i])
        s = i * k if drow0 is None else int(drow0[i])
        oracle.check(target[r:r + nd + 1].numpy(), None if draft is None else draft[s:s + nd].numpy(),
                     drafts[i, :nd].numpy() if k else [], ua[i].numpy() if k else [], us[i],
                     1.0 if heat is None else float(heat[i]), int(acc[i]), tok[i], lp[i], f"{what}, request {i}")
        kept += int(acc[i])
    print(f"  {n} requests, {kept} drafts kept", flush=True)
    return acc, tok, lp


def _logits(n, k, V, seed, dist):
    g = _gen(seed)
    target = torch.randn(n * (k + 1), V, generator=g) * 2
    near = target.view(n, k + 1, V)[:, :k].reshape(n * k, V)
    draft = near + torch.randn(n * k, V, generator=g) * 0.7 if dist else None
    top = (draft if dist else near).view(n, k, V).argmax(-1)
    drafts = torch.where(torch.rand(n, k, generator=g) < 0.7, top, torch.randint(0, V, (n, k), generator=g)).to(torch.int32)
    ua, us = torch.rand(n, k, generator=g), torch.rand(n, generator=g)
    heat = torch.rand(n, generator=g) + 0.2
    heat[::3] = 0.0
    return target, draft, drafts, ua, us, heat


@pytest.mark.parametrize("dist", [False, True])
@pytest.mark.parametrize("n,k,V", [(1, 1, 1), (5, 2, 7), (3, 4, 4095), (7, 3, 4097), (2, 64, 300), (9, 5, 50257), (2, 4, 128256)])
def test_verify(n, k, V, dist):
    target, draft, drafts, ua, us, heat = _logits(n, k, V, n + k + V, dist)
    _verify_and_check(target, draft, drafts, None, ua, us, heat, None, None, k, f"verify n {n} k {k} V {V} draft logits {dist}")


@pytest.mark.parametrize("dist", [False, True])
@pytest.mark.parametrize("n,k,V", [(4, 3, 511), (3, 2, 512), (5, 1, 513), (3, 2, 1025), (2, 2, 32768), (2, 2, 32769), (2, 1, 65536),
                                   (2, 1, 65537), (300, 64, 600), (300, 64, 1030), (5, 64, 600)])
def test_verify_chunks_of_every_size(n, k, V, dist):
    """Vocabularies around the borders of the chunks, and calls that take another chunk for their number
    of requests alone; of the long lists of drafts few are there, and their rows lie packed."""
    g = _gen(n + V)
    nd = torch.randint(0, min(k, 3) + 1, (n,), generator=g)
    row0 = torch.cumsum(nd + 1, 0) - nd - 1
    drow0 = torch.cumsum(nd, 0) - nd
    target = torch.randn(int((nd + 1).sum()), V, generator=g) * 2
    draft = torch.randn(int(nd.sum()), V, generator=g) * 2 if dist else None
    drafts, ua, us = torch.zeros(n, k, dtype=torch.int32), torch.rand(n, k, generator=g) ** 2, torch.rand(n, generator=g)
    for i in range(n):
        for j in range(int(nd[i])):
            drafts[i, j] = target[row0[i] + j].argmax() if j % 2 else torch.randint(0, V, (1,), generator=g)[0]
    i32 = torch.int32
    _verify_and_check(target, draft, drafts, nd.to(i32), ua, us, None, row0.to(i32), drow0.to(i32), k,
                      f"chunks n {n} k {k} V {V} draft logits {dist}")


@pytest.mark.parametrize("n,V", [(1, 1), (300, 5), (64, 4096), (33, 32001), (3, 128256)])
def test_sampling_without_drafts(n, V):
    target, _, _, _, us, heat = _logits(n, 0, V, n + V, False)
    us[0] = 0.0
    us[-1] = 1 - 2.0 ** -24
    heat[-1] = 1.0
    _verify_and_check(target, None, None, None, None, us, heat, None, None, 0, f"sample n {n} V {V}")


@pytest.mark.parametrize("dist", [False, True])
def test_verify_ragged_packed_rows_odd_strides_and_counts_outside(dist):
    n, k, V = 11, 6, 3001
    g = _gen(8)
    n_drafts = torch.tensor([3, 0, 6, 1, -4, 99, 2, 5, 0, 4, 6], dtype=torch.int32)
    nd = n_drafts.clamp(0, k)
    row0, drow0 = (nd + 1).cumsum(0) - (nd + 1), nd.cumsum(0) - nd
    rows, drows = int((nd + 1).sum()), int(nd.sum())
    target = torch.randn(rows, V, generator=g) * 2
    at = torch.cat([torch.arange(int(r), int(r) + int(c)) for r, c in zip(row0, nd)])
    draft = target[at] + torch.randn(drows, V, generator=g) * 0.5 if dist else None
    drafts = torch.randint(0, V, (n, k), generator=g).to(torch.int32)
    for i in range(n):
        for j in range(int(nd[i])):
            if (i + j) % 3:
                drafts[i, j] = target[int(row0[i]) + j].argmax()
    ua, us, heat = torch.rand(n, k, generator=g) * 0.3, torch.rand(n, generator=g), torch.ones(n)
    # rows that start off 16-byte borders, a stride that is no multiple of four
    td = torch.full((rows, V + 2), float("nan"), device="cuda")[:, 1:V + 1]
    td.copy_(target)
    dd = None
    if dist:
        dd = torch.full((drows, V + 4), float("inf"), device="cuda")[:, 3:V + 3]
        dd.copy_(draft)
    _verify_and_check(target, draft, drafts, n_drafts, ua, us, heat, row0.to(torch.int32), drow0.to(torch.int32), k,
                      f"ragged, draft logits {dist}", target_dev=td, draft_dev=dd)


@pytest.mark.parametrize("dist", [False, True])
def test_verify_masks_ties_and_nonfinite_logits(dist):
    n, k, V = 12, 2, 5003
    target, draft, drafts, ua, us, heat = _logits(n, k, V, 77, dist)
    heat[:] = torch.tensor([1.0, 0.0, 0.5] * 4)
    t = target.view(n, k + 1, V)
    banned = torch.rand(n, k + 1, V, generator=_gen(3)) < 0.9
    t[2:5][banned[2:5]] = -float("inf")
    t[5, 0] = -float("inf")                        # nothing has weight: refused, no token
    t[6, 0, :] = float("nan")
    t[7, 1, 100:200] = float("nan")                # some without weight
    t[8, 0, 4999] = float("inf")                   # all the weight in two places
    t[8, 0, 17] = float("inf")
    t[9, :, :] = 0.25                              # flat rows: ties
    t[10, 0, :] = torch.finfo(torch.float32).min   # the type's lowest value is a weight like any other
    drafts[8] = torch.tensor([17, 17])
    drafts[9] = torch.tensor([0, 5])
    drafts[11] = torch.tensor([V, -1])             # outside the vocabulary
    ua[11] = 0.0
    if dist:
        draft.view(n, k, V)[2] = -float("inf")     # a draft without a distribution of its own
        draft.view(n, k, V)[3, 0, drafts[3, 0]] = -float("inf")
    acc, tok, _ = _verify_and_check(target, draft, drafts, None, ua, us, heat, None, None, k, f"masks, draft logits {dist}")
    assert acc[5] == 0 and tok[5, 0] == -1 and acc[6] == 0 and tok[6, 0] == -1 and acc[11] == 0


def test_verify_extreme_temperatures_and_random_numbers():
    n, k, V = 8, 1, 1000
    target, _, drafts, ua, us, _ = _logits(n, k, V, 5, False)
    heat = torch.tensor([1e-30, 1e30, float("inf"), float("nan"), -1.0, 1e-3, 1.0, 1.0])
    us[6], us[7] = 0.0, 1 - 2.0 ** -24
    ua[6], ua[7] = 1 - 2.0 ** -24, 0.0
    _verify_and_check(target, None, drafts, None, ua, us, heat, None, None, k, "temperatures")
    # random numbers outside [0, 1): a token that has weight, no fault
    us[:] = torch.tensor([float("nan"), 2.0, -1.0, 0.5, 0.5, float("inf"), 1.0, -0.0])
    ua[:, 0] = torch.tensor([float("nan"), 2.0, -1.0, 0.5, 0.5, float("inf"), 1.0, -0.0])
    acc = torch.empty(n, dtype=torch.int32, device="cuda")
    tok = torch.empty(n, 2, dtype=torch.int32, device="cuda")
    spanq.verify_drafts(target.cuda(), drafts.cuda(), ua.cuda(), us.cuda(), heat.cuda(), acc, tok)
    assert bool(((acc >= 0) & (acc <= 1)).all())
    assert bool((tok.gather(1, acc.long()[:, None]) >= 0).all()) and bool((tok < V).all())


def test_verify_rows_outside_the_logits_and_rows_shared():
    n, k, V = 6, 2, 900
    target, draft, drafts, ua, us, heat = _logits(n, k, V, 21, True)
    row0 = torch.tensor([0, -1, 16, 15, 0, 2 ** 31 - 1], dtype=torch.int32)   # 18 rows: 16 + 2 is outside
    drow0 = torch.tensor([0, 0, 0, 11, 0, 0], dtype=torch.int32)              # 12 rows: 11 + 2 is outside
    acc = torch.zeros(n, dtype=torch.int32, device="cuda")
    tok = torch.zeros(n, k + 1, dtype=torch.int32, device="cuda")
    lp = torch.full((n, k + 1), 5.0, device="cuda")
    spanq.verify_drafts(target.cuda(), drafts.cuda(), ua.cuda(), us.cuda(), heat.cuda(), acc, tok, draft_logits=draft.cuda(),
                        row0=row0.cuda(), draft_row0=drow0.cuda(), logprobs=lp)
    acc, tok, lp = acc.cpu(), tok.cpu(), lp.cpu()
    for i in (1, 2, 3, 5):
        assert acc[i] == -1 and bool((tok[i] == -1).all()) and bool((lp[i] == 0).all())
    oracle = _Oracle(V)
    for i in (0, 4):  # two requests over the same rows
        oracle.check(target[:3].numpy(), draft[:2].numpy(), drafts[i].numpy(), ua[i].numpy(), us[i], float(heat[i]),
                     int(acc[i]), tok[i].numpy(), lp[i].numpy(), f"shared rows, request {i}")


def test_verify_in_a_graph_follows_its_inputs():
    n, k, V = 5, 3, 20000
    target, draft, drafts, ua, us, heat = _logits(n, k, V, 9, True)
    n_drafts = torch.full((n,), k, dtype=torch.int32)
    d = [t.cuda() for t in (target, draft, drafts, ua, us, heat, n_drafts)]
    acc, tok = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, k + 1, dtype=torch.int32, device="cuda")
    lp = torch.zeros(n, k + 1, device="cuda")
    ws = torch.empty(spanq.verify_workspace(n, k, V), dtype=torch.uint8, device="cuda")

    def call(acc, tok, lp, ws=None):
        spanq.verify_drafts(d[0], d[2], d[3], d[4], d[5], acc, tok, draft_logits=d[1], n_drafts=d[6], logprobs=lp, workspace=ws)

    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(acc, tok, lp, ws)
    for step in range(4):
        fresh = _logits(n, k, V, 30 + step, True)
        for to, t in zip(d, fresh):
            to.copy_(t)
        d[6].copy_(torch.tensor([(step + i) % (k + 1) for i in range(n)], dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        want = torch.empty_like(acc), torch.empty_like(tok), torch.empty_like(lp)
        call(*want)
        assert torch.equal(acc, want[0]) and torch.equal(tok, want[1]) and torch.equal(lp, want[2]), step


def test_a_call_leaves_the_current_device_and_refuses_tensors_of_the_wrong_kind():
    x = torch.zeros(2, 64, dtype=torch.bfloat16, device="cuda")
    i = torch.zeros(2, dtype=torch.int32, device="cuda")
    a, b = torch.zeros(1, 1, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 64, 8, dtype=torch.bfloat16, device="cuda")
    before = torch.cuda.current_device()
    spanq.adapter_apply(x, x, i, a, b, None, x)
    assert torch.cuda.current_device() == before
    bad = [dict(x=x.float()), dict(ids=i.long()), dict(ids=i[:1]), dict(a=a.cpu()), dict(b=b[:, :32]), dict(out=x[:, :32]),
           dict(base=x.t().contiguous().t()), dict(parts=(32, 16)), dict(parts=(32, 32)), dict(ranks=i.float()),
           dict(workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))]
    for change in bad:
        args = {**dict(x=x, base=x, ids=i, a=a, b=b, scale=None, out=x), **change}
        with pytest.raises(spanq.SpanError) as e:
            spanq.adapter_apply(**args)
        assert e.value.code == -1
    h = torch.zeros(2, 3, 64, device="cuda")
    for args in ((h, None, None, None, None, 1e-5, None, None, None), (h, None, None, None, None, 1e-5, h[:1], None, None),
                 (h, h[:, :1], h, None, None, 1e-5, h, h[:, :1], h), (h.half(), None, None, None, None, 1e-5, h.half(), None, None),
                 (h[..., :32], None, None, None, None, 1e-5, h[..., :32], None, None),
                 (h.transpose(0, 1), None, None, None, None, 1e-5, h.transpose(0, 1), None, None)):
        with pytest.raises(spanq.SpanError):
            spanq.qk_norm_rope(*args)
    lg, u, tok = torch.zeros(4, 10, device="cuda"), torch.zeros(2, device="cuda"), torch.zeros(2, 2, dtype=torch.int32, device="cuda")
    for args in ((lg, None, None, u, None, i, tok), (lg.double(), tok[:, :1], u[:, None], u, None, i, tok),
                 (lg, tok[:, :1], u[:, None], u, None, i, tok), (lg, tok[:, :1].contiguous(), u[:, None], u[:1], None, i, tok),
                 (lg, tok[:, :1].contiguous(), u[:, None], u, None, i.long(), tok)):
        with pytest.raises(spanq.SpanError):
            spanq.verify_drafts(*args)


def test_calls_of_two_threads_on_streams_of_their_own():
    import threading
    wrong, done = [], []

    def work(seed):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            parts, T, V = (264, 24), (40, 300)[seed], 5000
            case = _adapt_case(T, 520, parts, 24, 5, seed=seed)
            d = [t.cuda(non_blocking=False) for t in case]
            lg = torch.randn(6, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))
            u = torch.rand(6, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))
            first = None
            for _ in range(40):
                out = torch.empty_like(d[1])
                acc, tok = torch.empty(6, dtype=torch.int32, device="cuda"), torch.empty(6, 1, dtype=torch.int32, device="cuda")
                spanq.adapter_apply(d[0], d[1], d[2], d[3], d[4], d[5], out, parts=parts, ranks=d[6])
                spanq.verify_drafts(lg, None, None, u, None, acc, tok)
                if first is None:
                    first = (out, tok)
                elif not (torch.equal(out, first[0]) and torch.equal(tok, first[1])):
                    wrong.append(seed)
            stream.synchronize()
            ref, bound = _adapt_exact(*case, parts)
            if not bool(((first[0].cpu().double() - ref).abs() <= bound).all()):
                wrong.append(seed)
            done.append(seed)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong and sorted(done) == [0, 1]


def test_captured_calls_take_their_workspaces_from_the_graph():
    """Without a workspace of the caller's: calls one after another in one graph, between them other memory."""
    T, V, parts = 300, 3000, (72,)
    case = _adapt_case(T, 136, parts, 16, 3, seed=1)
    d = [t.cuda() for t in case]
    lg, u = torch.randn(20, V, device="cuda"), torch.rand(20, device="cuda")
    want, out, out2 = torch.empty_like(d[1]), torch.empty_like(d[1]), torch.empty_like(d[1])
    acc, tok, tok2 = (torch.empty(20, *s, dtype=torch.int32, device="cuda") for s in ((), (1,), (1,)))
    spanq.adapter_apply(d[0], d[1], d[2], d[3], d[4], d[5], want, ranks=d[6])
    spanq.verify_drafts(lg, None, None, u, None, acc, tok2)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        spanq.adapter_apply(d[0], d[1], d[2], d[3], d[4], d[5], out, ranks=d[6])
        mid = torch.full((T * 80,), float("nan"), device="cuda") * 2
        spanq.verify_drafts(lg, None, None, u, None, acc, tok)
        spanq.adapter_apply(d[0], d[1], d[2], d[3], d[4], d[5], out2, ranks=d[6])
    for _ in range(3):
        out.zero_()
        out2.zero_()
        tok.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(out2, want) and torch.equal(tok, tok2) and bool(torch.isnan(mid).all())


# ------------------------------------------------------------------------ the largest sizes

def _far(rows, width, stride, dtype):
    """Rows of a buffer that is not filled in between them, `stride` elements apart."""
    return torch.empty(rows * stride, dtype=dtype, device="cuda").as_strided((rows, width), (stride, 1))


@pytest.mark.parametrize("T", [200, 300])
def test_adapters_rows_far_apart(T):
    """Offsets of x past 2^32 elements, of base and out past 2^32 bytes."""
    case = _adapt_case(T, 136, (72,), 16, 3, seed=T)
    d = [t.cuda() for t in case]
    x, out = _far(T, 136, 1 << 25, torch.bfloat16), _far(T, 72, 1 << 23, torch.bfloat16)
    x.copy_(d[0])
    out.copy_(d[1])
    print(f"{T} rows, {x.stride(0) * T * 2 >> 30} GiB of x", flush=True)
    spanq.adapter_apply(x, out, d[2], d[3], d[4], d[5], out, ranks=d[6])
    _check_adapt(out.cpu(), case, (72,), "far apart")


@pytest.mark.parametrize("T", [3, 140])
def test_adapters_of_the_widest_products(T):
    g = torch.Generator(device="cuda").manual_seed(T)
    N, R, S, K = 1 << 20, 24, 3, 64
    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.bfloat16)
    x, out, a, b = randn(T, K), randn(T, N), randn(S, 1, R, K) / 8, randn(S, N, R)
    ids = torch.randint(-1, S, (T,), generator=g, device="cuda", dtype=torch.int32)
    base, cols = out.clone(), torch.cat([torch.arange(64), torch.arange(N // 2 - 32, N // 2 + 32), torch.arange(N - 64, N)]).cuda()
    print(f"{T} rows of {N} columns", flush=True)
    spanq.adapter_apply(x, out, ids, a, b, None, out)
    case = [t.cpu() for t in (x, base[:, cols], ids, a, b[:, cols], torch.ones(S), torch.full((S,), R))]
    _check_adapt(out[:, cols].cpu(), case, (len(cols),), "widest")


def test_adapters_of_the_longest_reduction():
    case = _adapt_case(5, 1 << 20, (8,), 8, 2, seed=20)
    d = [t.cuda() for t in case]
    out = torch.empty_like(d[1])
    spanq.adapter_apply(d[0], d[1], d[2], d[3], d[4], d[5], out, ranks=d[6])
    _check_adapt(out.cpu(), case, (8,), "K 2^20")


@pytest.mark.parametrize("dist", [False, True])
def test_verify_of_the_largest_vocabulary(dist):
    n, k, V = 1, 1, 1 << 24
    target, draft, drafts, ua, us, _ = _logits(n, k, V, 24, dist)
    for u in (0.0, 0.9999999):  # kept, or refused
        _verify_and_check(target, draft, drafts, None, ua * 0 + u, us, None, None, None, k, f"V 2^24, draft logits {dist}, u {u}")


def test_verify_rows_far_apart():
    n, k, V = 2, 2, 600
    target, draft, drafts, ua, us, heat = _logits(n, k, V, 5, True)
    t, y = _far(n * (k + 1), V, 1 << 29, torch.float32), _far(n * k, V, 1 << 30, torch.float32)
    t.copy_(target)
    y.copy_(draft)
    _verify_and_check(target, draft, drafts, None, ua, us, heat, None, None, k, "far apart", t, y)


def test_head_norms_far_apart_and_of_many_heads_in_a_graph():
    """Strides past 2^32 bytes, more heads than a work-group has threads; captured, with positions and rows
    that change between the replays."""
    n, hq, hkv, dim, far = 3, 517, 70, 64, 1 << 31
    g = _gen(9)
    x, kv = torch.randn(n, hq, dim, generator=g).to(torch.bfloat16), torch.randn(n, hkv, dim, generator=g).to(torch.bfloat16)
    gain = (1 + 0.3 * torch.randn(dim, generator=g)).to(torch.bfloat16)
    q = torch.empty((n - 1) * far + hq * dim, dtype=torch.bfloat16, device="cuda").as_strided((n, hq, dim), (far, dim, 1))
    q.copy_(x.cuda())
    k, gd = kv.cuda(), gain.cuda()
    qo = torch.zeros((n, hq, dim), dtype=torch.bfloat16, device="cuda")
    ko = torch.zeros((n, hkv, dim), dtype=torch.bfloat16, device="cuda")
    pos, rows = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.arange(n, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        spanq.qk_norm_rope(q, k, None, gd, gd, 1e-5, qo, ko, None, rows=rows, positions=pos)
    for step in range(3):
        at = torch.randint(0, 1 << 20, (n,), generator=g).to(torch.int32)
        to = torch.randperm(n, generator=g)
        pos.copy_(at)
        rows.copy_(to.to(torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        _check_heads(qo.cpu()[to], x, gain, 1e-5, at, 1e4, f"q, replay {step}")
        _check_heads(ko.cpu()[to], kv, gain, 1e-5, at, 1e4, f"k, replay {step}")
