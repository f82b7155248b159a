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
