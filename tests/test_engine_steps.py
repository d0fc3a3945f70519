"""Steps of the generation engine with drafts and sampling, on the CPU with a model that is told its answers."""
import pytest

from paper_2511_02749_amd import SpanError
from paper_2511_02749_amd import spanquery as sq
from paper_2511_02749_amd.engine import Engine


class _Told:
    """A pool, its plan and its model in one; `steps`: what each decode step answers for its queries."""

    def __init__(self, first, steps=()):
        self.first, self.steps = first, list(steps)
        self.committed = self.destroyed = False
        self.fed, self.drafts = [], []

    def plan(self, queries, stream):
        return self

    def forward(self, plan, rows, stream=None):
        return list(self.first)

    def decode_drafts(self, plan, tokens, drafts, **_):
        self.fed.append(list(tokens))
        self.drafts.append([list(d) for d in drafts])
        step = self.steps.pop(0)
        if isinstance(step, Exception):
            raise step
        return step

    def stats(self):
        return dict(pages_hit=0, tokens_hit=0, tokens_new=0, decode_steps=len(self.fed))

    def commit(self):
        self.committed = True

    def destroy(self):
        self.destroyed = True


def _spans(n):
    return [sq.Spans(prefix=[], fragments=[], cross=[1, 2]) for _ in range(n)]


@pytest.mark.parametrize("first,steps,max_tokens", [
    ([7], [[[-1]]], 2),                                     # the last token asked for
    ([7, 8], [[[5], [6]], [[5], [-1]]], 3),                 # one of two queries, in the last step
    ([7, 8], [[[5, 6], [9]], [[], [-1]]], 3),               # the other one has finished
    ([7], [[[3, -1]]], 3),                                  # after a kept draft
    ([7], [[[3]], [[-1]]], 9)])
def test_no_token_of_no_weight_is_returned_or_committed(first, steps, max_tokens):
    told = _Told(first, steps)
    engine = Engine(told, told, n_drafts=2)
    with pytest.raises(RuntimeError, match="weight"):
        engine.generate_many(_spans(len(first)), max_tokens)
    assert told.destroyed and not told.committed and not engine.calls


@pytest.mark.parametrize("first", [[-1], [5, -1]])
def test_a_first_sampled_token_of_no_weight_ends_the_call(first, monkeypatch):
    told = _Told(first)
    engine = Engine(told, told, temperature=1.0)
    monkeypatch.setattr(engine, "_sample_first", lambda plan, rows, n: list(first))
    with pytest.raises(RuntimeError, match="weight"):
        engine.generate_many(_spans(len(first)), 1)
    assert told.destroyed and not told.committed


def test_a_first_greedy_token_of_no_weight_ends_a_call_with_drafts():
    told = _Told([5, -1])
    with pytest.raises(RuntimeError, match="weight"):
        Engine(told, told, n_drafts=3).generate_many(_spans(2), 4)
    assert told.destroyed and not told.fed


def test_finished_queries_feed_nothing_and_the_others_go_on():
    told = _Told([7, 8], [[[5, 6], [9]], [[], [4]]])
    assert Engine(told, told, n_drafts=2).generate_many(_spans(2), 3) == [[7, 5, 6], [8, 9, 4]]
    assert told.committed and told.fed == [[7, 8], [-1, 9]]


def test_drafts_that_the_pool_has_no_pages_for_are_left_out():
    spans = [sq.Spans(prefix=[], fragments=[], cross=[7, 3, 4, 5, 7])]
    told = _Told([3], [SpanError(-2, "pages"), [[4]], [[5, 7]]])
    assert Engine(told, told, n_drafts=4).generate_many(spans, 4) == [[3, 4, 5, 7]]
    assert told.drafts == [[[4, 5]], [[]], [[5]]] and told.committed
    for error, steps in ((SpanError(-2, "pages"), 2), (SpanError(-3, "runtime"), 1)):
        told = _Told([3], [error] * steps)
        with pytest.raises(SpanError):
            Engine(told, told, n_drafts=4).generate_many(spans, 4)
        assert not told.steps and told.destroyed and not told.committed


@pytest.mark.parametrize("n", [-1, 65, 1000])
def test_numbers_of_drafts_that_no_step_takes_are_refused_at_once(n):
    with pytest.raises(ValueError, match="n_drafts"):
        Engine(None, None, n_drafts=n)
    assert Engine(None, None, n_drafts=64).n_drafts == 64
