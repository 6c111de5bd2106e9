"""The tag head's own checks, with the operators replaced: what they are given has been checked elsewhere."""
import pytest
import torch

from paper_1502_03409_amd import taghead
from paper_1502_03409_amd.taghead import TagHead


@pytest.fixture
def head(monkeypatch):
    called = []
    for name in ("glu_fwd", "glu_bwd", "xent_fwd", "xent_fwd_bwd", "logp_fwd", "logp_bwd", "grad_clip"):
        monkeypatch.setattr(taghead.H, name, lambda *a, name=name, **k: called.append(name))
    h = TagHead(8, 8, 16, 6, tags=3, likeliest=2, device="cpu")
    h.called = called
    return h


X, TAGS, TARGET = torch.zeros(6, 8), torch.zeros(6, 3, dtype=torch.int64), torch.zeros(6, dtype=torch.int64)
GIVEN = torch.zeros(6, 3)


def gradients(head, n=6, T=3):
    head.gradients_of(X[:n], TAGS[:n, :T] if T else None, GIVEN[:n, :T] if T else None, torch.zeros(n))


def test_gradients_follow_an_answer_that_is_learned_from(head):
    head.answer(X, TAGS, learn=True)
    gradients(head)
    gradients(head)              # for other given gradients: nothing that they need has changed
    head.answer(X[:2], None, likeliest=2, learn=True)
    gradients(head, 2, 0)
    assert head.called.count("logp_bwd") == head.called.count("glu_bwd") == 3


BETWEEN = {
    "an answer not learned from": lambda h: h.answer(X, TAGS),
    "an answer refused": lambda h: pytest.raises(ValueError, h.answer, X, TAGS.repeat(1, 2), learn=True),
    "other gradients": lambda h: h.gradients(X, TARGET),
    "an evaluation": lambda h: h.evaluate(X, TARGET),
    "a step": lambda h: h.update(0.1),
    "another batch": lambda h: h.answer(X[:4], TAGS[:4], learn=True),
    "other tags": lambda h: h.answer(X, TAGS[:, :2], learn=True),
    "no tags": lambda h: h.answer(X, learn=True),
}


@pytest.mark.parametrize("between", BETWEEN, ids=lambda k: k.replace(" ", "_"))
def test_gradients_of_anything_else_are_refused(head, between):
    """The hidden layer, its gates, the softmax's sums or the weights are others by then."""
    head.answer(X, TAGS, learn=True)
    BETWEEN[between](head)
    with pytest.raises(ValueError, match="learn=True"):
        gradients(head)
    assert "logp_bwd" not in head.called


def test_gradients_without_an_answer_are_refused(head):
    with pytest.raises(ValueError, match="learn=True"):
        gradients(head)
    head.answer(X, TAGS)
    with pytest.raises(ValueError, match="learn=True"):
        gradients(head)
