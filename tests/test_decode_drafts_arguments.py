"""What Model.decode_drafts refuses on the host, before the library is called."""
from types import SimpleNamespace

import numpy as np
import pytest

spanq = pytest.importorskip("paper_2511_02749_amd")


class _Plan:
    n_queries, _h, _stream = 3, None, None


def _model(monkeypatch):
    """A model without a library behind it: what reaches the library is recorded."""
    from paper_2511_02749_amd import _lib
    calls = []

    class Lib:
        def span_model_decode_drafts(self, *args):
            sampling = args[6]._obj
            calls.append(([sampling.u_accept[i] for i in range(6)], [sampling.u_sample[i] for i in range(3)]))
            return 0

    monkeypatch.setattr(_lib, "load", lambda: Lib())
    m = spanq.Model.__new__(spanq.Model)
    m._h, m.cfg = None, SimpleNamespace(vocab=100)
    m.pool = SimpleNamespace(cfg=SimpleNamespace(device=0))
    return m, calls


GOOD = dict(tokens=[1, 2, 3], drafts=[[4], [], [5, 6]], u_accept=[[0.5], [], [0.5, 0.5]], u_sample=[0.1, 0.2, 0.3],
            temperature=[1.0, 0.0, 0.5])


@pytest.mark.parametrize("change", [
    dict(u_accept=[[0.5], []]), dict(u_accept=[[0.5], [], [0.5, 0.5], []]), dict(u_accept=[]),
    dict(u_accept=[[0.5], [], [0.5]]), dict(u_sample=[0.1]), dict(u_sample=[0.1] * 4), dict(temperature=[1.0]),
    dict(temperature=[1.0] * 4), dict(u_sample=None), dict(u_accept=None), dict(drafts=[[4], []]), dict(tokens=[1, 2])])
def test_lists_of_other_lengths_are_refused(monkeypatch, change):
    model, calls = _model(monkeypatch)
    with pytest.raises(spanq.SpanError) as e:
        model.decode_drafts(_Plan(), **{**GOOD, **change})
    assert e.value.code == -1 and not calls


def test_an_entry_for_each_query_goes_to_the_library(monkeypatch):
    model, calls = _model(monkeypatch)
    for change in ({}, dict(temperature=0.7), dict(u_accept=[[0.5, 0.9], [0.1], [0.5, 0.5]])):
        assert model.decode_drafts(_Plan(), **{**GOOD, **change}) == [[], [], []]
    accept, sample = calls[0]
    assert accept == [0.5, 0.0, 0.0, 0.0, 0.5, 0.5] and np.allclose(sample, [0.1, 0.2, 0.3]) and len(calls) == 3
