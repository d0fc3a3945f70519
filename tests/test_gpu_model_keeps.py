"""Norms and adapters that a model was given stay alive and as they are, whatever the caller does with the lists."""
import gc
import weakref

import pytest

import workloads as W
from tests.helpers import StackRun

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
spanq = pytest.importorskip("paper_2511_02749_amd")


def test_weights_live_as_long_as_the_model_has_them():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    swl = W.stack_small()
    run, sw, bf = StackRun(swl), swl.weights, torch.bfloat16
    L, H, F = sw.n_layers, sw.hidden, sw.ffn
    gains = [torch.ones(sw.head_dim, dtype=bf, device="cuda") for _ in range(L)]
    a = [torch.zeros(2, 1, 8, F, dtype=bf, device="cuda") for _ in range(L)]
    b = [torch.zeros(2, H, 8, dtype=bf, device="cuda") for _ in range(L)]
    run.model.set_qk_norm(gains, gains)
    run.model.set_adapters(2, 8, down=(a, b))
    seen = [weakref.ref(t) for t in gains + a + b]
    for t in (gains, a, b):
        t.clear()
    gc.collect()
    assert all(r() is not None for r in seen)
    run.model.set_qk_norm()
    run.model.set_adapters()
    gc.collect()
    assert all(r() is None for r in seen)
    run.close()
