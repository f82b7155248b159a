"""The optimizer's count of its steps on the GPU."""
import math

import pytest
import torch

from paper_2609_02846_b200.optimizer import AdamW

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _params():
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    ps = [torch.nn.Parameter(torch.randn(s, generator=g, device=DEV).to(t)) for s, t in (((300, 70), torch.bfloat16), ((500,), torch.float32))]
    for p in ps:
        p.grad = torch.randn(p.shape, generator=g, device=DEV).to(p.dtype)
    return ps


def _same(a, b, oa, ob):
    for p, q in zip(a, b):
        assert torch.equal(p, q)
        assert all(torch.equal(oa.state[p][k], ob.state[q][k]) for k in oa.state[p] if torch.is_tensor(oa.state[p][k]))


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_that_are_left_out_leave_no_trace_in_either_mode(bits):
    """The same weights, moments and numbers as without them: corrections and draws go by the steps that were taken."""
    sets = [_params() for _ in range(3)]
    opts = [AdamW(sets[0], state_bits=bits), AdamW(sets[1], state_bits=bits, capturable=True), AdamW(sets[2], state_bits=bits)]
    for scale in (1.0, math.nan, 0.5, math.inf, 0.25):
        value = torch.tensor([scale], device=DEV)
        for i, opt in enumerate(opts):
            if i < 2 or math.isfinite(scale):
                opt.step(grad_scale=value)
    for opt in opts:
        assert [s["step"] for s in opt.state_dict()["state"].values()] == [3, 3]
    _same(sets[0], sets[2], opts[0], opts[2])
    _same(sets[1], sets[2], opts[1], opts[2])


@pytest.mark.parametrize("bits", [32, 8])
def test_the_count_moves_between_device_and_host(bits):
    """Replays of a captured step, then steps on the host, then the device again: as steps in a row."""
    a, b = _params(), _params()
    oa, ob = AdamW(a, state_bits=bits, capturable=True), AdamW(b, state_bits=bits)
    oa.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        oa.step()
    graph.replay()
    graph.replay()
    oa.param_groups[0]["capturable"] = False
    oa.step()
    oa.param_groups[0]["capturable"] = True
    with pytest.raises(RuntimeError, match="before the capture"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            oa.step()
    oa.step()
    graph.replay()
    for _ in range(6):
        ob.step()
    _same(a, b, oa, ob)
    assert [s["step"] for s in oa.state_dict()["state"].values()] == [6, 6]
