"""What the row operators refuse, on the CPU: every bad argument is answered by the host's checks
with SPAN_EINVAL, before any HIP call, and calls without rows are no work at all.

The records are packed as include/spanq.h lays them out; addresses are never followed."""
import ctypes
import math
import struct

import pytest

spanq = pytest.importorskip("paper_2511_02749_amd")
from paper_2511_02749_amd import row_ops as R  # noqa: E402

QK_REC = struct.Struct("<10Q8q5i2fi")  # span_qk_norm
P = 1 << 20  # an address: aligned, never read
QK = dict(q=P, k=P, v=P, q_out=2 * P, k_out=2 * P, v_out=2 * P, q_gain=P, k_gain=P, rows=0, positions=0,
          q_stride=512, k_stride=128, v_stride=128, q_out_stride=512, k_out_stride=128, v_out_stride=128, n_rows=4,
          out_rows=4, num_q_heads=4, num_kv_heads=1, head_dim=128, dtype=1, device=0, eps=1e-5, rope_theta=1e4,
          reserved=0)
ADAPT = dict(x=P, base=P, out=2 * P, ids=P, a=P, b=P, scale=0, ranks=0, workspace=P, workspace_bytes=1 << 30,
             x_stride=64, base_stride=64, out_stride=64, n_rows=4, in_features=64, n_adapters=2, max_rank=16,
             n_parts=2, c0=24, c1=40, c2=0, c3=0, device=0, reserved=0)
VERIFY = dict(target=P, draft=P, row0=0, draft_row0=0, drafts=P, n_drafts=0, u_accept=P, u_sample=P, temperature=0,
              accepted=P, tokens=P, logprobs=0, workspace=P, workspace_bytes=1 << 30, target_stride=100,
              draft_stride=100, target_rows=10, draft_rows=8, n_requests=2, max_drafts=4, vocab=100, device=0)


@pytest.fixture(scope="module")
def lib():
    try:
        return spanq.load()
    except FileNotFoundError:
        pytest.skip("libspanq.so not built")


def _call(lib, entry, rec, args, n=None):
    blob = rec.pack(*args.values())
    if n is not None:
        return getattr(lib, entry)(blob, n)
    return getattr(lib, entry)(blob, None)


def _refused(lib, entry, rec, args):
    assert _call(lib, entry, rec, args) == -1
    assert entry in lib.span_last_error().decode()


@pytest.mark.parametrize("change", [
    dict(head_dim=96), dict(head_dim=0), dict(dtype=2), dict(dtype=-1), dict(n_rows=-1), dict(n_rows=1 << 31),
    dict(out_rows=3), dict(out_rows=-1), dict(out_rows=1 << 31), dict(num_q_heads=0), dict(num_kv_heads=0),
    dict(num_q_heads=-4), dict(num_kv_heads=1 << 20), dict(eps=-1e-5), dict(eps=math.nan), dict(eps=math.inf),
    dict(positions=P, rope_theta=0.0), dict(positions=P, rope_theta=math.nan), dict(positions=P, rope_theta=math.inf),
    dict(device=-1), dict(reserved=1), dict(q_out=0), dict(k=0), dict(v_out=0), dict(q=P + 8), dict(k_out=2 * P + 2),
    dict(q_gain=P + 4), dict(q_stride=504), dict(q_stride=516), dict(k_out_stride=120), dict(v_stride=0),
    dict(q_out=P, q_out_stride=520), dict(q_out=P, rows=P),
])
def test_qk_norm_rope_refuses(lib, change):
    _refused(lib, "span_qk_norm_rope", QK_REC, {**QK, **change})


@pytest.mark.parametrize("change", [
    dict(n_rows=-1), dict(n_rows=1 << 31), dict(in_features=0), dict(in_features=60), dict(in_features=(1 << 20) + 8),
    dict(max_rank=0), dict(max_rank=12), dict(max_rank=136), dict(n_parts=0), dict(n_parts=5), dict(c0=0), dict(c0=12),
    dict(c1=-8), dict(c0=1 << 20), dict(n_adapters=-1), dict(device=-1), dict(reserved=1), dict(x=0), dict(base=0),
    dict(out=0), dict(ids=0), dict(a=0), dict(b=0), dict(x=P + 8), dict(base=P + 2), dict(out=P + 4), dict(a=P + 8),
    dict(b=P + 8), dict(workspace=P + 4), dict(workspace=0), dict(workspace_bytes=0), dict(x_stride=56),
    dict(x_stride=68), dict(base_stride=56), dict(out_stride=60),
    dict(base_stride=(1 << 23) + 8), dict(out_stride=(1 << 23) + 8), dict(out=P, out_stride=72),
])
def test_adapter_apply_refuses(lib, change):
    _refused(lib, "span_adapter_apply", R._ADAPTER_REC, {**ADAPT, **change})


@pytest.mark.parametrize("change", [
    dict(n_requests=-1), dict(n_requests=(1 << 20) + 1), dict(max_drafts=-1), dict(max_drafts=65), dict(vocab=0),
    dict(vocab=(1 << 24) + 1), dict(device=-1), dict(target=0), dict(drafts=0), dict(u_accept=0), dict(u_sample=0),
    dict(accepted=0), dict(tokens=0), dict(target_rows=-1), dict(target_stride=99), dict(draft_stride=99),
    dict(draft_rows=-1), dict(target=P + 2), dict(draft=P + 1), dict(workspace=0), dict(workspace=P + 8),
    dict(workspace_bytes=16),
])
def test_verify_drafts_refuses(lib, change):
    _refused(lib, "span_verify_drafts", R._VERIFY_REC, {**VERIFY, **change})


def test_null_records_are_refused(lib):
    n = ctypes.c_size_t()
    for entry in ("span_qk_norm_rope", "span_adapter_apply", "span_verify_drafts"):
        assert getattr(lib, entry)(None, None) == -1
    for entry in ("span_adapter_workspace", "span_verify_workspace"):
        assert getattr(lib, entry)(None, ctypes.byref(n)) == -1
    assert lib.span_adapter_workspace(R._ADAPTER_REC.pack(*ADAPT.values()), None) == -1
    assert lib.span_verify_workspace(R._VERIFY_REC.pack(*VERIFY.values()), None) == -1


def test_calls_without_rows_are_no_work(lib):
    assert _call(lib, "span_qk_norm_rope", QK_REC, {**QK, "n_rows": 0}) == 0
    assert _call(lib, "span_qk_norm_rope", QK_REC, {**QK, **{n: 0 for n in ("q", "k", "v", "q_out", "k_out", "v_out")}}) == 0
    assert _call(lib, "span_adapter_apply", R._ADAPTER_REC, {**ADAPT, "n_rows": 0, "x": 0}) == 0
    assert _call(lib, "span_verify_drafts", R._VERIFY_REC, {**VERIFY, "n_requests": 0, "target": 0}) == 0


@pytest.mark.parametrize("rows", [0, 1, 16, 17, 256, 257, 4096, 1 << 17, (1 << 17) + 3, (1 << 31) - 1])
def test_adapter_workspace_holds_a_partial_of_every_row_worked_at_once(lib, rows):
    got = spanq.adapter_workspace(rows, 4096, 24, (64, 64))
    cols = 2 * 32  # two parts, rank 24 in blocks of 16
    # at most 16 partials and their sum, and eight bytes for a row's place in the order by adapter
    assert min(rows, 1 << 16) * cols * 4 <= got <= min(rows, 1 << 16) * (cols * 4 * 17 + 8)


def test_workspaces_serve_smaller_calls():
    sizes = [0, 1, 7, 14, 15, 28, 29, 57, 64, 65, 113, 128, 129, 192, 200, 256, 257, 300, 520, 1024, 1030, 2048, 4096,
             4160, 9000, 16384, 16448, 65536, 65537, 65736, 70000, 131072, 1 << 20]
    for args in ((4096, 16, (4096,)), (4096, 128, (16384, 8192, 512)), (14336, 64, (4096,)), (8, 8, (8,))):
        need = [spanq.adapter_workspace(n, *args) for n in sizes]
        assert need == sorted(need)
    for args in ((0, 1000), (4, 1000), (4, 32768), (8, 50257), (64, 65536), (7, 128256), (0, 1 << 24)):
        need = [spanq.verify_workspace(n, *args) for n in sizes]
        assert need == sorted(need)


def test_workspaces_refuse_sizes_of_no_call():
    for args in ((4, 60, 16, (8,)), (4, 64, 16, (12,)), (-1, 64, 16, (8,)), (4, 64, 130, (8,)), (4, 64, 16, ())):
        with pytest.raises(spanq.SpanError):
            spanq.adapter_workspace(*args)
    for args in ((1, 65, 100), (-1, 4, 100), (1, 4, 0)):
        with pytest.raises(spanq.SpanError):
            spanq.verify_workspace(*args)


def test_tensors_on_the_host_are_refused():
    torch = pytest.importorskip("torch")
    x = torch.zeros(2, 64, dtype=torch.bfloat16)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(spanq.SpanError) as e:
        spanq.adapter_apply(x, x, i, torch.zeros(1, 1, 8, 64, dtype=torch.bfloat16),
                            torch.zeros(1, 64, 8, dtype=torch.bfloat16), None, x)
    assert e.value.code == -1
    h = torch.zeros(2, 1, 64)
    with pytest.raises(spanq.SpanError):
        spanq.qk_norm_rope(h, None, None, None, None, 1e-5, h, None, None)
    with pytest.raises(spanq.SpanError):
        spanq.qk_norm_rope(None, None, None, None, None, 1e-5, None, None, None)
    with pytest.raises(spanq.SpanError):
        spanq.verify_drafts(torch.zeros(2, 9), None, None, torch.zeros(2), None, i, i[:, None])


def test_what_is_no_tensor_on_a_gpu_is_refused_before_anything_else(lib):
    torch = pytest.importorskip("torch")
    x, i = torch.zeros(2, 64, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    h, u = torch.zeros(2, 3, 64), torch.zeros(2)
    a, b = torch.zeros(1, 1, 8, 64, dtype=torch.bfloat16), torch.zeros(1, 64, 8, dtype=torch.bfloat16)
    for call in (lambda: spanq.qk_norm_rope(h, None, None, None, None, 1e-5, h, None, None),
                 lambda: spanq.qk_norm_rope(None, None, None, None, None, 1e-5, None, None, None),
                 lambda: spanq.qk_norm_rope(h.to_sparse(), None, None, None, None, 1e-5, h, None, None),
                 lambda: spanq.qk_norm_rope([1.0], None, None, None, None, 1e-5, [1.0], None, None),
                 lambda: spanq.adapter_apply(x, x, i, a, b, None, x), lambda: spanq.adapter_apply(None, x, i, a, b, None, x),
                 lambda: spanq.adapter_apply(x, None, i, a, b, None, None),
                 lambda: spanq.verify_drafts(u[None], None, None, u, None, i, i[:, None]),
                 lambda: spanq.verify_drafts(u[None], None, None, u, None, i, None)):
        with pytest.raises(spanq.SpanError) as e:
            call()
        assert e.value.code == -1
