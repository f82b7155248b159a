"""The operators between the linears through autograd, and the block that runs them together."""
import math

import pytest
import torch

import paper_2609_02846_b200 as lib
from paper_2609_02846_b200 import autograd as A
from paper_2609_02846_b200.block import TransformerBlock
from block_reference import allowed, draws

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _rel(a, b):
    a, b = a.detach().double(), b.detach().double()
    return float((a - b).norm() / b.norm())


def test_functions_match_the_calls_they_wrap():
    g = torch.Generator(device=DEV)
    g.manual_seed(0)
    n = lambda *s: torch.randn(*s, generator=g, device=DEV).to(torch.bfloat16)
    x, w, b, dy = n(3, 50, 256), torch.rand(256, device=DEV, requires_grad=True), torch.rand(256, device=DEV, requires_grad=True), n(3, 50, 256)
    x.requires_grad_()
    y = A.layer_norm(x, w, b)
    y.backward(dy)
    wy, mean, rstd = lib.layer_norm(x.detach().view(-1, 256), w.detach(), b.detach())
    want = lib.layer_norm_backward(dy.view(-1, 256), x.detach().view(-1, 256), w.detach(), mean, rstd)
    assert torch.equal(y.view(-1, 256), wy) and torch.equal(x.grad.view(-1, 256), want[0]) and torch.equal(w.grad, want[1]) and torch.equal(b.grad, want[2])
    x.grad = None
    r = n(3, 50, 256).requires_grad_()
    z = A.dropout_add(x, 0.3, 11, r)
    z.backward(dy)
    assert torch.equal(x.grad.view(-1, 256), lib.dropout_add(dy.view(-1, 256), 0.3, 11)) and torch.equal(r.grad, dy)
    q, k, v, do = (n(2, 96, h, 64) for h in (4, 2, 2, 4))
    for t in (q, k, v):
        t.requires_grad_()
    o = A.attention(q, k, v, causal=True)
    o.backward(do)
    wo, lse = lib.attention(q.detach(), k.detach(), v.detach(), causal=True)
    assert torch.equal(o, wo)
    for t, want in zip((q, k, v), lib.attention_backward(do, q.detach(), k.detach(), v.detach(), wo, lse, causal=True)):
        assert torch.equal(t.grad, want)


def test_gradients_that_arrive_expanded():
    """sum() hands back a gradient with zero strides: the wrappers copy it, the bare calls refuse it."""
    x = torch.randn(32, 64, device=DEV, requires_grad=True)
    A.dropout_add(A.layer_norm(x), 0.1, 3).sum().backward()
    assert bool(x.grad.isfinite().all())
    q = torch.randn(1, 32, 2, 64, device=DEV).to(torch.bfloat16).requires_grad_()
    A.attention(q, q, q).sum().backward()
    assert bool(q.grad.isfinite().all())


def test_dropout_module_draws_by_layer_and_step_and_rests_in_evaluation():
    x = torch.ones(64, 256, device=DEV)
    a, b = A.DropoutAdd(0.5), A.DropoutAdd(0.5)
    first = a(x)
    assert torch.equal(first, a(x)) and not torch.equal(first, b(x))
    a.advance()
    assert not torch.equal(first, a(x))
    a.eval()
    assert torch.equal(a(x, x), 2 * x)


def _plain_block(block, x, p, masks):
    """The block in 64 bits with torch's own differentiation; `masks` are the dropout masks of the two residual additions."""
    B, L, hidden = x.shape
    H, Hk, D = block.heads, block.kv_heads, block.head_dim
    P = {n: t.detach().double().requires_grad_() for n, t in block.named_parameters()}
    norm = lambda t, i: (t - t.mean(-1, keepdim=True)) / torch.sqrt(t.var(-1, keepdim=True, unbiased=False) + 1e-5) * P[f"norm{i}.weight"] + P[f"norm{i}.bias"]
    x = x.detach().double().requires_grad_()
    r = x
    qkv = (norm(r, 1) @ P["qkv.weight"].T).view(B, L, H + 2 * Hk, D).permute(0, 2, 1, 3)
    q, k, v = qkv[:, :H], qkv[:, H:H + Hk].repeat_interleave(H // Hk, 1), qkv[:, H + Hk:].repeat_interleave(H // Hk, 1)
    s = (q @ k.transpose(-1, -2) / math.sqrt(D)).masked_fill(~allowed(L, L, True, -1, L, x.device), -math.inf)
    o = (s.softmax(-1) @ v).permute(0, 2, 1, 3).reshape(B, L, hidden)
    t = int(p * 65536 + 0.5)
    drop = lambda y, m: torch.where(m.view_as(y), y * 65536 / (65536 - t), torch.zeros((), dtype=torch.float64, device=y.device))
    r = r + drop(o @ P["proj.weight"].T, masks[0])
    h = torch.relu(norm(r, 2) @ P["up.weight"].T)
    return r + drop((h * h) @ P["down.weight"].T, masks[1]), x, P


def test_block_with_plain_linears_against_64_bits():
    """BF16 block (torch's linears, the library's operators) against the same block in 64 bits: every stored activation is rounded
    to BF16 (2^-8), about ten of them follow one another in each direction: 2-norm of the difference below 10 * 2^-8."""
    torch.manual_seed(1)
    B, L, hidden, H, Hk, ffn, p = 2, 200, 256, 4, 2, 512, 0.1
    linear = lambda i, o: torch.nn.Linear(i, o, bias=False, device=DEV, dtype=torch.bfloat16)
    block = TransformerBlock(hidden, H, Hk, ffn, p, linear=linear)
    x = torch.randn(B, L, hidden, device=DEV, dtype=torch.bfloat16).requires_grad_()
    dy = torch.randn(B, L, hidden, device=DEV, dtype=torch.bfloat16)
    y = block(x)
    y.backward(dy)
    n, t = B * L * hidden, int(p * 65536 + 0.5)
    masks = [torch.from_numpy(draws(n, A.sr_stream_seed(d.seed, d.rank, d.step)) >= t).to(DEV) for d in (block.drop1, block.drop2)]
    wy, wx, P = _plain_block(block, x, p, masks)
    wy.backward(dy.double())
    assert _rel(y, wy) < 10 * 2.0 ** -8
    assert _rel(x.grad, wx.grad) < 10 * 2.0 ** -8
    for name, t in block.named_parameters():
        assert _rel(t.grad, P[name].grad) < 10 * 2.0 ** -8, name
    assert lib.last_device_status() == 0


def test_block_of_fp4_linears_points_the_same_way():
    """Forward and backward of the whole block with UE5M3-FP4 linears against the same weights with torch's linears.  E2M1 with
    16-element blocks is off by about 0.1 of a value in the mean square (up to 0.2 with stochastic rounding), so a product of two
    rounded operands by 0.15 to 0.25 and two such products in a row by 0.35 at most: the cosine stays above 1 / sqrt(1 + 0.35^2) = 0.94;
    0.9 is asked for."""
    torch.manual_seed(2)
    cos = lambda a, b: float((a.detach().double() * b.detach().double()).sum() / a.detach().double().norm() / b.detach().double().norm())
    fp4 = TransformerBlock(256, 4, 2, 512, 0.05)
    plain = TransformerBlock(256, 4, 2, 512, 0.05, linear=lambda i, o: torch.nn.Linear(i, o, bias=False, device=DEV, dtype=torch.bfloat16))
    plain.load_state_dict(fp4.state_dict())
    plain.drop1.seed, plain.drop2.seed = fp4.drop1.seed, fp4.drop2.seed
    x = torch.randn(2, 256, 256, device=DEV, dtype=torch.bfloat16)
    dy = torch.randn_like(x)
    got = []
    for block in (fp4, plain):
        xx = x.clone().requires_grad_()
        y = block(xx, torch.tensor([256, 100], dtype=torch.int32, device=DEV))
        y.backward(dy)
        got.append((y - x, xx.grad - dy, {n: t.grad for n, t in block.named_parameters()}))
    assert cos(got[0][0], got[1][0]) > 0.9 and cos(got[0][1], got[1][1]) > 0.9
    for name, grad in got[0][2].items():
        assert cos(grad, got[1][2][name]) > 0.9, name
    fp4.advance()
    assert fp4.qkv.step == fp4.drop1.step == fp4.drop2.step == 1
    assert lib.last_device_status() == 0
