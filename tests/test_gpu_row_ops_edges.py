"""Row operators where a rounding, an infinity or an empty remainder decides the answer.

Tolerances are counted in roundings of the result alone (half a step, torch.finfo(t).eps / 2 of the value):
the inputs are made so that everything before the last rounding is exact in float32.
"""
import numpy as np
import pytest

import paper_2511_02749_amd as spanq
from tests.test_gpu_row_ops import _logits, _verify_and_check

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    print(flush=True)


def _gen(seed):
    return torch.Generator().manual_seed(seed)


# ------------------------------------------------------------------------ adapters

# rows, columns: few, tiles, runs of one, two, three and more tiles of 16
FORMS = [(5, 136), (40, 8200), (300, 136), (300, 8200), (800, 8200), (1100, 8200), (2500, 8200)]


@pytest.mark.parametrize("T,N", FORMS)
@pytest.mark.parametrize("R", [8, 24, 56, 128])
def test_adapters_keep_every_bit_of_the_low_rank_sums(T, N, R):
    """Of two ranks that a column takes, one's sum is a whole number of 24 bits (three digits of 8), the other's its
    upper 16 taken away: every step is exact in float32 and what is left, a digit, in bf16."""
    g, S, K = _gen(T + R), 2, 3 * R
    x = torch.randint(0, 256, (T, K), generator=g).float()
    a = torch.zeros(S, 1, R, K)
    for r in range(0, R, 2):
        for s, of in enumerate(([1.0, 2.0 ** 8, 2.0 ** 16], [2.0 ** -4, -(2.0 ** -12), 2.0 ** -20])):
            a[s, 0, r, 3 * r:3 * r + 3] = torch.tensor(of)
            a[s, 0, r + 1, 3 * r:3 * r + 3] = -torch.tensor([w if abs(w) > min(map(abs, of)) else 0.0 for w in of])
    b = torch.zeros(S, N, R)
    pair = torch.arange(N) * 5 % (R // 2)
    b[:, torch.arange(N), 2 * pair] = b[:, torch.arange(N), 2 * pair + 1] = 1.0
    ids = torch.arange(T) % 3 - 1
    want = torch.where(ids[:, None] == 0, x[:, 6 * pair], x[:, 6 * pair + 2] * 2.0 ** -20) * (ids[:, None] >= 0)
    bf = torch.bfloat16
    print(f"exact sums T {T} N {N} R {R}", flush=True)
    out = torch.full((T, N), float("nan"), dtype=bf, device="cuda")
    spanq.adapter_apply(x.to(bf).cuda(), torch.zeros_like(out), ids.to(torch.int32).cuda(), a.to(bf).cuda(), b.to(bf).cuda(),
                        None, out)
    assert torch.equal(out.cpu().float(), want), float((out.cpu().float() - want).abs().max())


@pytest.mark.parametrize("T,N", FORMS)
@pytest.mark.parametrize("R", [8, 40, 128])
def test_adapters_with_infinite_weights(T, N, R):
    """Infinite and NaN weights of B at ranks that count, with low-rank sums that a bf16 holds (nothing is left of
    them), sums that it does not (a rest of either sign), and sums of 0: the formula's infinities and NaN, and
    nothing else changes."""
    g, S, K, bf = _gen(T * R), 3, 64, torch.bfloat16
    x = torch.randint(-3, 4, (T, K), generator=g).float()
    a = torch.randint(-2, 3, (S, 1, R, K), generator=g).float() * torch.tensor([1.0, 2.0 ** -9, 1.0])[:, None, None, None]
    a[1, ..., :32] *= 2.0 ** 9  # sums of 12 bits and more
    b = torch.randint(-2, 3, (S, N, R), generator=g).float()
    ids = (torch.arange(T) * 7 // 5 % (S + 1) - 1).to(torch.int32)
    base = torch.randint(-9, 10, (T, N), generator=g).float()
    args = [t.cuda() for t in (x.to(bf), base.to(bf), ids, a.to(bf))]
    plain, out = (torch.full((T, N), float("nan"), dtype=bf, device="cuda") for _ in range(2))
    spanq.adapter_apply(*args, b.to(bf).cuda(), None, plain)
    wild = torch.tensor([float("inf"), -float("inf"), float("nan")])
    cols = torch.arange(1, N, 5)
    for i in range(S - 1):  # (the last adapter has none)
        b[i, cols, torch.randint(0, R, (len(cols),), generator=g)] = wild[torch.randint(0, 3, (len(cols),), generator=g)]
        b[i, cols[::3], torch.randint(0, R, (len(cols[::3]),), generator=g)] = float("inf")
    print(f"infinite weights T {T} N {N} R {R}", flush=True)
    spanq.adapter_apply(*args, b.to(bf).cuda(), None, out)
    h = torch.einsum("tk,srk->tsr", x.double(), a[:, 0].double())[torch.arange(T), ids.clamp(min=0).long()]
    want = torch.zeros(T, N, dtype=torch.float64)
    for i in range(S):
        mine = (ids == i).nonzero()[:, 0]
        terms = (h[mine][:, None] * b[i, cols].double()).sum(-1)  # infinities as the formula has them
        want[mine[:, None], cols] = terms
    out, plain = out.cpu(), plain.cpu()
    assert bool((ids < 0).any()) and bool(torch.isposinf(want).any()) and bool(torch.isneginf(want).any()) and bool(want.isnan().any())
    rest = want.isfinite()
    assert torch.equal(out[rest], plain[rest])
    assert torch.equal(out[~rest].double().nan_to_num(7.0, 8.0, 9.0), want[~rest].nan_to_num(7.0, 8.0, 9.0))


@pytest.mark.parametrize("T,N", FORMS)
@pytest.mark.parametrize("R", [8, 24, 128])
def test_rows_of_an_adapter_keep_their_bits_beside_a_row_that_is_no_number(T, N, R):
    """Every eleventh row of x holds a NaN or an infinity: the others' results are the same bits."""
    g, K, bf = _gen(T + R), 264, torch.bfloat16
    x, base, a, b = (torch.randn(*s, generator=g).to(bf).cuda() for s in ((T, K), (T, N), (2, 1, R, K), (2, N, R)))
    ids = (torch.arange(T) * 3 // 2 % 3 - 1).to(torch.int32).cuda()
    out, hurt = (torch.full((T, N), 5.0, dtype=bf, device="cuda") for _ in range(2))
    spanq.adapter_apply(x, base, ids, a, b, None, out)
    x[::11, 7] = float("nan")
    x[::22, 7] = float("inf")
    print(f"beside no numbers T {T} N {N} R {R}", flush=True)
    spanq.adapter_apply(x, base, ids, a, b, None, hurt)
    fine = torch.ones(T, dtype=torch.bool, device="cuda")
    fine[::11] = False
    assert torch.equal(hurt[fine], out[fine])
    wild = ~fine & (ids >= 0)
    assert not bool(hurt[wild].isfinite().all(1).any()) and bool(out.isfinite().all())


# ------------------------------------------------------------------------ verification

@pytest.mark.parametrize("V,n", [(1500, 60), (3000, 60), (40000, 40), (128256, 20)])
def test_a_refused_draft_that_stands_alone_in_its_chunk_leaves_nothing_there(V, n):
    """Grammar masks that allow the draft and a token far from it: with a random number of 0 (and next to it)
    the first chunk with any weight decides, and that of the refused draft has none."""
    k = 2
    target, _, drafts, ua, us, heat = _logits(n, k, V, V, False)
    heat = heat.clamp(min=0.2) + 0.1
    t, g = target.view(n, k + 1, V), _gen(V)
    drafts = torch.randint(0, 400, (n, k), generator=g).to(torch.int32)  # in the first chunk, of 512 at least
    other = torch.randint(V - 300, V, (n,), generator=g)
    keep = t.clone()
    t[:] = -float("inf")
    for i in range(n):
        for j in range(k):
            t[i, j, drafts[i, j]] = keep[i, j, 0]
        t[i, :, other[i]] = keep[i, :, 1]
    ua[:] = 1 - 2.0 ** -24
    us[:] = torch.tensor([0.0, 0.0, 1e-30, 2.0 ** -24] * (n // 4))
    acc, tok, _ = _verify_and_check(target, None, drafts, None, ua, us, heat, None, None, k, f"alone in its chunk, V {V}")
    assert (acc == 0).any() and np.array_equal(tok[np.arange(n), acc], other.numpy())


def test_weights_too_small_for_a_number_are_passed_over():
    """Chunks before the row's largest logits whose single weights are no number in 64 bits, though
    their sum would be: with a random number of 0 the token is the first one that has a weight."""
    n, V = 12, 6000
    target = torch.full((n, V), -float("inf"))
    first = torch.randint(4000, V, (n,), generator=_gen(1))
    for i in range(n):
        target[i, :3000] = -744.5 - 0.25 * i  # exp: below half of the smallest number from -745.14 on
        target[i, first[i]:] = 0.0
    us = torch.zeros(n)
    _, tok, _ = _verify_and_check(target, None, None, None, None, us, None, None, None, 0, "weights that are no number")
    assert np.array_equal(tok[3:, 0], first[3:].numpy())


@pytest.mark.parametrize("V", [700, 5003, 128256])
def test_where_draft_and_target_agree_nothing_is_left_but_the_target(V):
    """p = q in every token and a draft that no row has (outside the vocabulary, or without weight): max(p - q, 0) is
    nothing, so the token comes from p itself."""
    n, k = 24, 2
    target, _, drafts, ua, us, heat = _logits(n, k, V, V, False)
    heat = heat.clamp(min=0.2) + 0.1
    t = target.view(n, k + 1, V)
    drafts[::2] = torch.tensor([-1, V])
    for i in range(1, n, 2):
        t[i, :, 3::7] = -float("inf")
        drafts[i] = 3
    draft = t[:, :k].reshape(n * k, V).clone()
    acc, _, _ = _verify_and_check(target, draft, drafts, None, ua * 0, us, heat, None, None, k, f"p = q, V {V}")
    assert (acc == 0).all()


# ------------------------------------------------------------------------ head norms

@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("theta", [1e4, 5e5])
def test_rotations_by_the_angle_and_not_by_a_float_next_to_it(dim, theta):
    """Pairs (1, 0): the rotated ones are cos and sin, off by a rounding of their own, however small they are.
    (Both sides' angles: a position of 18 bits times an inverse within 2^-51 of itself.)"""
    n, g = 3000, _gen(dim)
    pos = torch.randint(-50, 1 << 18, (n,), generator=g).to(torch.int32)
    x = torch.zeros(n, 2, dim)
    x[..., :dim // 2] = 1.0
    y = torch.empty_like(x, device="cuda")
    spanq.qk_norm_rope(x.cuda(), None, None, None, None, 0.0, y, None, None, positions=pos.cuda(), rope_theta=theta)
    t = pos.double()[:, None] * theta ** (-2.0 * torch.arange(dim // 2, dtype=torch.float64) / dim)
    want = torch.cat([torch.cos(t), torch.sin(t)], -1)[:, None].expand(-1, 2, -1)
    err = (y.cpu().double() - want).abs()
    bound = 2.0 ** -24 * want.abs() + 2.0 ** (18 - 50)
    print(f"dim {dim} theta {theta}: worst err/bound {(err / bound).max():.3g}", flush=True)
    assert bool((err <= bound).all())


@pytest.mark.parametrize("V", [300, 5003, 40000])
def test_a_token_that_is_all_of_both_rows_leaves_nothing(V):
    """Target and draft with all their weight, as far as 64 bits tell, on one token: p = q = 1 there, so that
    after a refused draft only what p has over q of the others is left, however little."""
    n, k = 40, 1
    target, draft, drafts, ua, us, heat = _logits(n, k, V, V, True)
    g, heat = _gen(V), heat.clamp(min=0.2)
    top = torch.randint(0, V, (n,), generator=g)
    t, y = target.view(n, k + 1, V), draft.view(n, k, V)
    gap = 60.0 * heat  # others: below e^-40 each, where a row's rounding is e^-37
    for i in range(n):
        t[i, :, top[i]], y[i, :, top[i]] = t[i].max() + gap[i], y[i].max() + gap[i] + 0.3
    drafts = ((top + 1 + torch.randint(0, V - 1, (n,), generator=g)) % V).to(torch.int32)[:, None]
    y[torch.arange(n), 0, drafts[:, 0].long()] += 5.0  # q(d) > p(d)
    ua[:] = 1 - 2.0 ** -24
    acc, tok, _ = _verify_and_check(target, draft, drafts, None, ua, us, heat, None, None, k, f"all of both rows, V {V}")
    assert (acc == 0).all() and not (tok[:, 0] == top.numpy()).any()


def test_logits_without_any_rows_are_not_logits_that_were_not_given():
    """Requests whose rows lie outside logits of no rows at all: -1, as outside any others; requests without drafts
    need no draft rows."""
    n, k, V = 4, 2, 100
    lg, none = torch.randn(n * (k + 1), V, device="cuda"), torch.empty(0, V, device="cuda")
    d, ua = torch.ones(n, k, dtype=torch.int32, device="cuda"), torch.zeros(n, k, device="cuda")
    us, heat = torch.rand(n, device="cuda"), torch.ones(n, device="cuda")
    for target, draft, counts, outside in ((lg, none, None, [1, 1, 1, 1]), (lg, none, [0, 2, 0, 1], [0, 1, 0, 1]),
                                           (none, None, None, [1, 1, 1, 1]), (none, none, [0, 0, 0, 0], [1, 1, 1, 1])):
        acc, tok = torch.full((n,), 9, dtype=torch.int32, device="cuda"), torch.full((n, k + 1), 9, dtype=torch.int32, device="cuda")
        spanq.verify_drafts(target, d, ua, us, heat, acc, tok, draft_logits=draft,
                            n_drafts=None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda"))
        for i, out in enumerate(outside):
            assert int(acc[i]) == (-1 if out else 0), (counts, i)
            assert bool((tok[i] == -1).all()) if out else 0 <= int(tok[i, 0]) < V


# ------------------------------------------------------------------------ tensors

def test_autograd_sees_that_outputs_were_written():
    """A tensor that a graph saved and an operator wrote afterwards is refused by the backward pass, as after
    torch's in-place calls; outputs have no history, also of inputs that require gradients."""
    bf = torch.bfloat16
    x, a, b = (torch.zeros(s, dtype=bf, device="cuda") for s in ((2, 64), (1, 1, 8, 64), (1, 64, 8)))
    ids, h = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.ones(2, 1, 64, device="cuda")
    lg, u = torch.zeros(2, 9, device="cuda"), torch.zeros(2, device="cuda")
    acc, tok, lp = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, 1, dtype=torch.int32, device="cuda"), torch.zeros(2, 1, device="cuda")
    out, qo = torch.ones_like(x), torch.ones_like(h)
    for call, written in ((lambda: spanq.adapter_apply(x.requires_grad_(), x, ids, a, b, None, out), [out]),
                          (lambda: spanq.qk_norm_rope(h.requires_grad_(), None, None, None, None, 1e-5, qo, None, None), [qo]),
                          (lambda: spanq.verify_drafts(lg, None, None, u, None, acc, tok, logprobs=lp), [lp, acc, tok])):
        w = torch.ones_like(written[0]).requires_grad_()
        y = (w * written[0]).sum()
        before = [t._version for t in written]
        call()
        assert all(t._version == v + 1 and not t.requires_grad for t, v in zip(written, before))
        with pytest.raises(RuntimeError, match="inplace"):
            y.backward()
    with torch.inference_mode():
        spanq.adapter_apply(x, x, ids, a, b, None, torch.empty_like(x))


def test_a_workspace_that_does_not_fit_is_an_error_of_memory():
    """2^18 requests of 64 drafts over 2^22 tokens: a TB of sums, on the current stream and on another one."""
    n, k, V = 1 << 18, 64, 1 << 22
    lg = torch.zeros(1, V, device="cuda")
    d, ua = torch.zeros(n, k, dtype=torch.int32, device="cuda"), torch.zeros(n, k, device="cuda")
    us, acc = torch.zeros(n, device="cuda"), torch.full((n,), 7, dtype=torch.int32, device="cuda")
    tok = torch.full((n, k + 1), 7, dtype=torch.int32, device="cuda")
    assert spanq.verify_workspace(n, k, V) > torch.cuda.get_device_properties(0).total_memory
    for stream in (None, torch.cuda.Stream()):
        with pytest.raises(spanq.SpanError) as e:
            spanq.verify_drafts(lg, d, ua, us, None, acc, tok, stream=stream)
        assert e.value.code == -2
    torch.cuda.synchronize()
    assert bool((acc == 7).all()) and bool((tok == 7).all())


def test_a_device_that_is_not_there_runs_nothing():
    """Records of a device that the machine does not have: an error, the current device stays and nothing is written."""
    from paper_2511_02749_amd import row_ops as R
    from tests.test_row_ops_refusals import QK_REC
    lib, bf, there = spanq.load(), torch.bfloat16, torch.cuda.device_count()
    x, out = torch.ones(2, 64, dtype=bf, device="cuda"), torch.full((2, 64), 7.0, dtype=bf, device="cuda")
    ids, a, b = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.ones(1, 1, 8, 64, dtype=bf, device="cuda"), torch.ones(1, 64, 8, dtype=bf, device="cuda")
    ws = torch.empty(spanq.adapter_workspace(2, 64, 8, (64,)) + spanq.verify_workspace(2, 0, 64), dtype=torch.uint8, device="cuda")
    lg, u = torch.zeros(2, 64, device="cuda"), torch.zeros(2, device="cuda")
    acc, tok = torch.full((2,), 7, dtype=torch.int32, device="cuda"), torch.full((2, 1), 7, dtype=torch.int32, device="cuda")
    p = lambda t: t.data_ptr()  # noqa: E731
    torch.cuda.synchronize()
    for entry, blob in (
            ("span_qk_norm_rope", QK_REC.pack(p(x), 0, 0, p(out), 0, 0, 0, 0, 0, 0, 64, 0, 0, 64, 0, 0, 2, 2, 1, 0, 64, 1, there,
                                              1e-5, 1e4, 0)),
            ("span_adapter_apply", R._ADAPTER_REC.pack(p(x), p(x), p(out), p(ids), p(a), p(b), 0, 0, p(ws), ws.numel(), 64, 64, 64,
                                                       2, 64, 1, 8, 1, 64, 0, 0, 0, there, 0)),
            ("span_verify_drafts", R._VERIFY_REC.pack(p(lg), 0, 0, 0, 0, 0, 0, p(u), 0, p(acc), p(tok), 0, p(ws), ws.numel(), 64,
                                                      64, 2, 0, 2, 0, 64, there))):
        assert getattr(lib, entry)(blob, None) == -3 and entry in lib.span_last_error().decode()
        assert torch.cuda.current_device() == 0
    torch.cuda.synchronize()
    assert bool((out == 7).all()) and bool((acc == 7).all()) and bool((tok == 7).all())


def test_a_stream_of_another_gpu_is_refused():
    from types import SimpleNamespace
    x, out = torch.ones(2, 1, 64, device="cuda"), torch.full((2, 1, 64), 7.0, device="cuda")
    here = torch.cuda.current_stream()
    for stream, fine in ((SimpleNamespace(cuda_stream=here.cuda_stream, device_index=1), False), (here, True),
                         (SimpleNamespace(cuda_stream=here.cuda_stream, device_index=0), True),
                         (SimpleNamespace(cuda_stream=here.cuda_stream), True)):
        out.fill_(7.0)
        if fine:
            spanq.qk_norm_rope(x, None, None, None, None, 0.0, out, None, None, stream=stream)
        else:
            with pytest.raises(spanq.SpanError) as e:
                spanq.qk_norm_rope(x, None, None, None, None, 0.0, out, None, None, stream=stream)
            assert e.value.code == -1
        assert bool((out == (1.0 if fine else 7.0)).all())
