"""The optimizer's count of its steps (no GPU: a stub that may refuse stands in the library's place)."""
import copy

import pytest
import torch

import paper_2609_02846_b200.optimizer as O


@pytest.fixture
def steps(monkeypatch):
    """Numbers of the steps that reach the library.  With a clock the stub counts as the device does: not the steps that are left out."""
    seen = []

    def adamw(ps, gs, m, v, step, clock=None, grad_scale=None, **kw):
        if any(g.dtype not in (torch.float32, torch.bfloat16) for g in gs):
            raise TypeError("refused")
        if clock is None:
            seen.append(step)
        elif grad_scale is None or bool(grad_scale.isfinite()):
            clock[0] += 1
            seen.append(int(clock[0]))
    monkeypatch.setattr(O.B, "adamw", adamw)
    return seen


def _params(n=2):
    ps = [torch.nn.Parameter(torch.ones(4)) for _ in range(n)]
    for p in ps:
        p.grad = torch.ones_like(p)
    return ps


@pytest.mark.parametrize("capturable", [False, True])
def test_a_step_that_is_refused_is_not_counted(steps, capturable):
    a, b = _params()
    opt = O.AdamW([{"params": [a]}, {"params": [b]}], capturable=capturable)
    opt.step()
    b.grad = None
    a.grad = torch.ones(4)
    opt.step()                                             # a: 2, b: 1
    refused = torch.nn.Parameter(torch.ones(4, dtype=torch.float16))
    refused.grad = torch.ones_like(refused)
    opt.add_param_group({"params": [refused]})
    b.grad = torch.ones(4)
    with pytest.raises(TypeError):
        opt.step()                                         # a and b take theirs before the third is refused
    assert [opt.state[p]["step"] for p in (a, b, refused)] == [3, 2, 0]
    refused.grad = None
    opt.step()
    assert steps == [1, 1, 2, 3, 2, 4, 3]


def _numbers(opt):
    return [s["step"] for s in opt.state_dict()["state"].values()]


def _taken(n, **kw):
    opt = O.AdamW(_params(), **kw)
    for _ in range(n):
        opt.step()
    return opt


def test_a_count_on_the_device_that_is_no_longer_kept(steps):
    """A capturable optimizer that loads a state which is not: what it counts on the host from there on stays."""
    opt, other = _taken(2, capturable=True), _taken(5)
    opt.load_state_dict(copy.deepcopy(other.state_dict()))
    assert not opt.param_groups[0]["capturable"]
    del steps[:]
    for number in (6, 7):
        opt.step()
        assert _numbers(opt) == [number] * 2
    opt.param_groups[0]["capturable"] = True               # and on the device again
    opt.step()
    assert _numbers(opt) == [8] * 2
    opt.param_groups[0]["capturable"] = False
    assert _numbers(opt) == [8] * 2
    opt.step()
    assert steps == [6, 7, 8, 9] and _numbers(opt) == [9] * 2


def test_replays_are_counted_when_the_count_moves_to_the_host(steps):
    opt = _taken(2, capturable=True)
    opt.param_groups[0]["clocks"][torch.device("cpu")][0] += 3          # what replays of a captured step do
    opt.param_groups[0]["capturable"] = False
    opt.step()
    assert steps[-1] == 6 and _numbers(opt) == [6] * 2


def test_what_is_saved_names_no_counter_of_the_device(steps):
    opt = _taken(2, capturable=True)
    saved = opt.state_dict()
    assert all(not torch.is_tensor(x) and not isinstance(x, dict) for group in saved["param_groups"] for x in group.values())
    new = O.AdamW(_params(), capturable=True)
    new.load_state_dict(copy.deepcopy(saved))
    new.step()
    assert steps == [1, 2, 3] and _numbers(new) == [3] * 2


def test_a_count_on_the_device_begins_at_the_most_that_a_parameter_has(steps):
    a, b = _params()
    opt = O.AdamW([a, b])
    opt.step()
    a.grad, g = None, a.grad
    opt.step()
    a.grad = g
    opt.param_groups[0]["capturable"] = True
    opt.step()
    assert steps == [1, 2, 3] and _numbers(opt) == [3] * 2


@pytest.mark.parametrize("capturable", [False, True])
def test_steps_that_are_left_out_are_not_counted(steps, capturable):
    """In both modes: the bias corrections and the draws of 8-bit moments go by the steps that were taken."""
    opt = O.AdamW(_params(), capturable=capturable)
    for scale in (1.0, float("nan"), 0.5, float("inf"), -float("inf")):
        opt.step(grad_scale=torch.tensor([scale]))
    opt.step()
    assert _numbers(opt) == [3] * 2
    opt.step(grad_scale=torch.tensor([float("nan")]))
    assert _numbers(opt) == [3] * 2                        # what is saved knows it already
    assert _numbers(copy.deepcopy(opt)) == [3] * 2
    assert steps == ([1, 2, 3] if capturable else [1, 2, 2, 3, 3, 3, 4])          # (the device leaves them out by itself)


def test_a_step_that_is_left_out_is_taken_back_from_those_that_took_part(steps):
    a, b = _params()
    opt = O.AdamW([a, b])
    opt.step()
    b.grad, g = None, b.grad
    opt.step(grad_scale=torch.tensor([float("inf")]))
    b.grad = g
    opt.step()
    assert _numbers(opt) == [2, 2]
    opt.step(grad_scale=torch.tensor([float("inf")]))
    opt.load_state_dict(_taken(7).state_dict())            # states that know nothing of it
    assert _numbers(opt) == [7, 7]
