"""What the transformer block makes of its arguments (no GPU: only what it builds is looked at)."""
import pytest
import torch

import paper_2609_02846_b200.block as block


@pytest.fixture
def turns(monkeypatch):
    seen = []

    class Turn(torch.nn.Module):
        def __init__(self, head_dim, **kw):
            super().__init__()
            seen.append((head_dim, kw))
    monkeypatch.setattr(block, "QKNormRotary", Turn)
    monkeypatch.setattr(block, "LayerNorm", lambda n: torch.nn.Identity())
    return seen


@pytest.mark.parametrize("rotary,qk_norm,want", [(False, False, None), (None, False, None), (True, False, dict(norm=False)), ({}, False, dict(norm=False)),
                                                 ({}, True, dict(norm=True)), (dict(base=500.0), True, dict(norm=True, base=500.0))])
def test_rotary(turns, rotary, qk_norm, want):
    b = block.TransformerBlock(256, 4, 2, 512, linear=lambda i, o: torch.nn.Identity(), rotary=rotary, qk_norm=qk_norm)
    assert turns == ([] if want is None else [(64, want)])
    assert (b.turn is None) == (want is None)


@pytest.mark.parametrize("rotary", [False, None])
def test_norms_want_positions(turns, rotary):
    with pytest.raises(ValueError, match="rotary"):
        block.TransformerBlock(256, 4, 2, 512, linear=lambda i, o: torch.nn.Identity(), rotary=rotary, qk_norm=True)
