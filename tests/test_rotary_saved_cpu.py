"""What the backward pass of the rotary functions reads again is under torch's check of versions (no GPU: stubs in the library's place)."""
import pytest
import torch

import paper_2609_02846_b200.autograd as A


@pytest.fixture(autouse=True)
def stubs(monkeypatch):
    seen = []
    monkeypatch.setattr(A.B, "rotary", lambda q, k, *args: seen.append(args) or (q.clone(), None if k is None else k.clone()))
    monkeypatch.setattr(A.B, "qk_norm_rotary", lambda q, k, wq, wk, *args: seen.append(args) or (q.clone(), None if k is None else k.clone()))
    monkeypatch.setattr(A.B, "qk_norm_rotary_backward", lambda dq, dk, q, k, wq, wk, *args, want_weights: seen.append(args) or (dq, dk, None, None))
    return seen


CALLS = [lambda q, f, at: A.rotary(q, None, f, at, True, 1.5), lambda q, f, at: A.qk_norm_rotary(q, None, None, None, f, at, True, 1.5, 1e-3)]


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("changed", ["positions", "frequencies"])
def test_positions_and_frequencies_that_change_before_the_backward_pass(call, changed):
    q, f, at = torch.ones(1, 3, 2, 8, requires_grad=True), torch.ones(4, dtype=torch.float64), torch.arange(3)
    y = call(q, f, at)[0]
    (at if changed == "positions" else f).add_(1)
    with pytest.raises(RuntimeError, match="inplace operation"):
        y.sum().backward()
    call(q, f, at)[0].sum().backward()                     # unchanged: as ever


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("at", [None, 7, torch.arange(3)])
def test_both_passes_get_the_same_arguments(call, at, stubs):
    q, f = torch.ones(1, 3, 2, 8, requires_grad=True), torch.ones(4, dtype=torch.float64)
    call(q, f, at)[0].sum().backward()
    there, back = stubs
    assert torch.equal(back[0], f)
    assert back[1] == at if not torch.is_tensor(at) else torch.equal(back[1], at)
    assert there[2:4] == back[2:4] == (True, 1.5)


@pytest.mark.parametrize("call", CALLS)
def test_tensors_of_inference_mode(call, stubs):
    """They have no version to check, as those that a module takes to another device in an evaluation have none: they are used as they are."""
    with torch.inference_mode():
        f, at = torch.ones(4, dtype=torch.float64), torch.arange(3)
    q = torch.ones(1, 3, 2, 8, requires_grad=True)
    call(q, f, at)[0].sum().backward()
    assert stubs[1][0] is f and stubs[1][1] is at and q.grad is not None
