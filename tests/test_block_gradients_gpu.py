"""Gradients of the differentiable wrappers where types and shapes of their inputs differ."""
import pytest
import torch

import paper_2609_02846_b200 as lib
from paper_2609_02846_b200 import autograd as A
from paper_2609_02846_b200.block import TransformerBlock
from block_reference import assert_within, layer_norm_backward
from test_layer_norm_gpu import make

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dt,bdt", [(BF, F), (F, BF), (BF, BF), (F, F)])
@pytest.mark.parametrize("cols", [256, 333])
def test_gradient_of_a_bias_without_a_weight_has_the_bias_type(cols, dt, bdt):
    """Held to the bound of the bias's own type: a binary32 sum is not rounded to the activations' BF16 on its way."""
    x, _, b, dy = make(500, cols, dt, bdt, seed=cols)
    _, mean, rstd = lib.layer_norm(x, None, b)
    want = layer_norm_backward(dy, x, None, mean, rstd)
    dx, dw, db = lib.layer_norm_backward(dy, x, None, mean, rstd, bias_dtype=bdt)
    assert dw is None and db.dtype == bdt
    assert_within(db, *want[2], "db")
    assert_within(dx, *want[0], "dx")
    xx, bb = x.clone().requires_grad_(), b.clone().requires_grad_()
    A.layer_norm(xx, None, bb).backward(dy)
    assert bb.grad.dtype == bdt and torch.equal(bb.grad, db) and torch.equal(xx.grad, dx)
    assert lib.layer_norm_backward(dy, x, None, mean, rstd)[2].dtype == dt           # nothing asked for: x's type
    w = torch.ones(cols, dtype=bdt, device=DEV)
    assert lib.layer_norm_backward(dy, x, w, mean, rstd, bias_dtype=bdt)[2].dtype == bdt
    with pytest.raises(ValueError):
        lib.layer_norm_backward(dy, x, w, mean, rstd, bias_dtype=F if bdt == BF else BF)       # two types of parameters
    with pytest.raises(TypeError):
        lib.layer_norm_backward(dy, x, None, mean, rstd, bias_dtype=torch.float16)


@pytest.mark.parametrize("dt", [BF, F])
@pytest.mark.parametrize("rows,cols", [(700, 33), (3000, 1023), (300, 1537), (900, 4607), (300, 8191), (40, 12001), (30, 16385), (3000, 1024), (60, 16384)])
def test_layer_norm_in_place(rows, cols, dt):
    """y over x, dx over dy and dx over x: aligned rows and rows at every offset from 16 bytes, all kernels."""
    x, w, b, dy = make(rows, cols, dt, F, seed=cols)
    y, mean, rstd = lib.layer_norm(x, w, b)
    want = lib.layer_norm_backward(dy, x, w, mean, rstd)
    z = x.clone()
    assert all(torch.equal(a, c) for a, c in zip(lib.layer_norm(z, w, b, out=z), (y, mean, rstd)))
    z = dy.clone()
    assert all(torch.equal(a, c) for a, c in zip(lib.layer_norm_backward(z, x, w, mean, rstd, out=z), want))
    z = x.clone()
    assert all(torch.equal(a, c) for a, c in zip(lib.layer_norm_backward(dy, z, w, mean, rstd, out=z), want))


def test_micro_batches_of_a_step_draw_masks_of_their_own():
    """Accumulated gradients: next_micro_batch() moves the dropout layers alone, so the linears keep the step (and with it the schedule of
    their tensor references), and a micro-batch that is computed again before it meets its own masks again."""
    block = TransformerBlock(256, 4, 2, 512, 0.5)
    x = torch.randn(1, 128, 256, device=DEV, dtype=BF)
    zeros = lambda drop: drop(torch.ones(64, 256, device=DEV)) == 0
    seen = []
    for micro in range(3):
        masks = [zeros(block.drop1), zeros(block.drop2)]
        assert torch.equal(masks[0], zeros(block.drop1))
        y = block(x)
        assert torch.equal(y, block(x))
        for mask in masks:
            assert all(abs(float((mask == other).float().mean()) - 0.5) < 0.05 for other in seen)
            seen.append(mask)
        block.next_micro_batch()
    assert block.qkv.step == block.down.step == 0
    block.advance()
    assert block.qkv.step == 1 and block.drop1.step == block.drop2.step == 4
