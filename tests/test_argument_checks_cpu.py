"""A tensor that stands in the place of another one has to have that one's shape, also where it is the queries themselves (no GPU: the launch
is a stub, and nothing may reach it)."""
import pytest
import torch

import paper_2609_02846_b200.autograd as A
import paper_2609_02846_b200.binding as B

BF = torch.bfloat16


@pytest.fixture
def launches(monkeypatch):
    seen = []
    monkeypatch.setattr(B, "_call", lambda fn, where, x, *args: seen.append(where))
    return seen


def _t(*shape):
    return torch.zeros(*shape, dtype=BF)


Q, LONG, MORE_HEADS, FEWER_HEADS = (1, 4, 2, 64), (1, 400, 2, 64), (1, 4, 8, 64), (1, 4, 1, 64)


@pytest.mark.parametrize("sinks", [0, 4])
@pytest.mark.parametrize("other", [LONG, FEWER_HEADS])
def test_queries_in_the_place_of_values(launches, other, sinks):
    q, k, o, lse = _t(*Q), _t(*other), _t(*Q), torch.zeros(1, 2, 4)
    for f in (lambda: B.attention(q, k, q, sinks=sinks), lambda: A.attention(q, k, q, sinks=sinks), lambda: B.attention(q, k, q, window_left=3, sinks=sinks),
              lambda: B.attention_backward(o, q, k, q, o, lse, sinks=sinks)):
        with pytest.raises(ValueError, match="expected a tensor like"):
            f()
    assert not launches


def test_queries_in_the_place_of_a_gradient(launches):
    q, k, o, lse = _t(*Q), _t(*LONG), _t(*Q), torch.zeros(1, 2, 4)
    for out in ((o, q, k), (o, k, q)):
        with pytest.raises(ValueError, match="expected a tensor like"):
            B.attention_backward(o, q, k, k, o, lse, out=out)
    assert not launches


@pytest.mark.parametrize("other", [MORE_HEADS, FEWER_HEADS])
def test_queries_in_the_place_of_what_belongs_to_the_keys(launches, other):
    q, k, x, f = _t(*Q), _t(*other), _t(*Q), torch.zeros(32, dtype=torch.float64)
    for g in (lambda: B.rotary(q, k, f, out=(x, q)), lambda: B.qk_norm_rotary(q, k, None, None, f, out=(x, q)),
              lambda: B.qk_norm_rotary_backward(x, q, q, k, None, None, f), lambda: B.qk_norm_rotary_backward(x, k, q, k, None, None, f, out=(x, q))):
        with pytest.raises(ValueError, match="expected a tensor like"):
            g()
    assert not launches


def test_queries_in_any_place_of_their_own_shape(launches):
    """What was right stays: q, k and v as one tensor, outputs and upstream gradients in the queries' place."""
    q, lse, f = _t(*Q), torch.zeros(1, 2, 4), torch.zeros(32, dtype=torch.float64)
    B.attention(q, q, q)
    B.attention(q, q, q, out=q)
    B.attention_backward(q, q, q, q, q, lse)
    B.rotary(q, q, f)
    B.rotary(q, None, f, out=(q, None))
    B.qk_norm_rotary_backward(q, q, q, q, None, None, f)
    assert len(launches) == 6
