"""Rotary positions, norms of queries and keys, window, sinks and the optimizer together, in the block that calls them."""
import math

import numpy as np
import pytest
import torch

import adamw_reference as adam
import paper_2609_02846_b200 as lib
import rotary_reference as rot
from block_reference import allowed, assert_within, draws
from paper_2609_02846_b200 import autograd as A
from paper_2609_02846_b200.block import TransformerBlock
from paper_2609_02846_b200.optimizer import AdamW

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _rel(a, b):
    a, b = a.detach().double(), b.detach().double()
    return float((a - b).norm() / b.norm())


def _plain_linear(i, o):
    return torch.nn.Linear(i, o, bias=False, device=DEV, dtype=torch.bfloat16)


def _plain_block(block, x, masks, p, positions, left, sinks):
    """The block in 64 bits with torch's own differentiation."""
    B, L, hidden = x.shape
    H, Hk, D = block.heads, block.kv_heads, block.head_dim
    P = {n: t.detach().double().requires_grad_() for n, t in block.named_parameters()}
    norm = lambda t, i: (t - t.mean(-1, keepdim=True)) / torch.sqrt(t.var(-1, keepdim=True, unbiased=False) + 1e-5) * P[f"norm{i}.weight"] + P[f"norm{i}.bias"]
    x = x.detach().double().requires_grad_()
    qkv = (norm(x, 1) @ P["qkv.weight"].T).view(B, L, H + 2 * Hk, D)
    q, k, v = qkv.split((H, Hk, Hk), 2)
    turn = block.turn

    def turned(t, weight):
        if turn.norm:
            t = t / torch.sqrt((t * t).mean(-1, keepdim=True) + turn.eps) * P[weight]
        at = positions.double()[..., None] * turn.frequencies
        c, s = (f(at)[:, :, None] * turn.amplitude for f in (torch.cos, torch.sin))
        h = turn.frequencies.numel()
        a, b, rest = t[..., :h], t[..., h:2 * h], t[..., 2 * h:]
        return torch.cat([a * c - b * s, a * s + b * c, rest], -1)
    q, k = turned(q, "turn.q_weight"), turned(k, "turn.k_weight")
    first = lambda t, n: t.permute(0, 2, 1, 3).repeat_interleave(n, 1)
    see = allowed(L, L, True, left, L, DEV) | (allowed(L, L, True, -1, L, DEV) & (torch.arange(L, device=DEV) < sinks))
    s = (first(q, 1) @ first(k, H // Hk).transpose(-1, -2) / math.sqrt(D)).masked_fill(~see, -math.inf)
    o = (s.softmax(-1) @ first(v, H // Hk)).permute(0, 2, 1, 3).reshape(B, L, hidden)
    t = int(p * 65536 + 0.5)
    drop = lambda y, m: torch.where(m.view_as(y), y * 65536 / (65536 - t), torch.zeros((), dtype=torch.float64, device=DEV))
    r = x + drop(o @ P["proj.weight"].T, masks[0])
    h = torch.relu(norm(r, 2) @ P["up.weight"].T)
    return r + drop((h * h) @ P["down.weight"].T, masks[1]), x, P


@pytest.mark.parametrize("qk_norm,rotary", [(True, True), (False, dict(rotary_dim=32, scaling="linear", factor=4))])
def test_block_against_64_bits(qk_norm, rotary):
    """As the plain block's test: every stored activation is rounded to BF16 (2^-8), about eleven of them follow one another in each direction."""
    torch.manual_seed(1)
    B, L, hidden, H, Hk, ffn, p, left, sinks = 2, 300, 256, 4, 2, 512, 0.1, 50, 3
    block = TransformerBlock(hidden, H, Hk, ffn, p, left, _plain_linear, sinks, rotary, qk_norm)
    if qk_norm:
        with torch.no_grad():
            block.turn.q_weight.uniform_(0.5, 1.5)
            block.turn.k_weight.uniform_(0.5, 1.5)
    x = torch.randn(B, L, hidden, device=DEV, dtype=torch.bfloat16).requires_grad_()
    dy = torch.randn(B, L, hidden, device=DEV, dtype=torch.bfloat16)
    positions = torch.stack([torch.arange(L), 5000 + torch.arange(L)]).to(DEV)
    y = block(x, positions=positions)
    y.backward(dy)
    masks = [torch.from_numpy(draws(B * L * hidden, A.sr_stream_seed(d.seed, d.rank, d.step)) >= int(p * 65536 + 0.5)).to(DEV) for d in (block.drop1, block.drop2)]
    wy, wx, P = _plain_block(block, x, masks, p, positions, left, sinks)
    wy.backward(dy.double())
    assert _rel(y, wy) < 11 * 2.0 ** -8
    assert _rel(x.grad, wx.grad) < 11 * 2.0 ** -8
    for name, t in block.named_parameters():
        assert _rel(t.grad, P[name].grad) < 11 * 2.0 ** -8, name
    assert lib.last_device_status() == 0


def test_positions_move_with_the_window():
    """Rotation is relative: the same tokens at other positions give the same outputs up to the rounding of q and k (2^-8 each, of scores of size 1 and their
    probabilities) and of o."""
    torch.manual_seed(3)
    block = TransformerBlock(256, 4, 2, 512, 0.0, 64, _plain_linear, 2, True, True)
    x = torch.randn(1, 200, 256, device=DEV, dtype=torch.bfloat16)
    with torch.no_grad():
        assert _rel(block(x, positions=1 << 19), block(x)) < 4 * 2.0 ** -8


@pytest.mark.parametrize("bits", [32, 8])
def test_fp4_block_takes_steps(bits):
    """The whole of it with FP4 linears: weights move by what the gradients say, masters and weights stay together."""
    torch.manual_seed(2)
    block = TransformerBlock(256, 4, 2, 512, 0.05, 100, sinks=4, rotary=True, qk_norm=True)
    lr, betas, eps, decay = 1e-3, (0.9, 0.99), 1e-8, 0.1
    opt = AdamW(block.parameters(), lr=lr, betas=betas, eps=eps, weight_decay=decay, state_bits=bits, seed=5)
    x = torch.randn(2, 256, 256, device=DEV, dtype=torch.bfloat16)
    for step in range(1, 4):
        block(x).float().square().mean().backward()
        before = {n: (opt.state[p].get("master", p) if opt.state[p] else p).detach().double().clone() for n, p in block.named_parameters()}
        opt.step()
        if step == 1:                                      # m = (1 - b1) g, v = (1 - b2) g^2 in every way of keeping them
            for n, p in block.named_parameters():
                g = p.grad.float().reshape(-1).cpu().numpy()
                m, v = adam.moments(np.zeros_like(g), np.zeros_like(g), g, betas)
                want, bound = adam.weights(before[n].reshape(-1).cpu().numpy(), m, v, 1, lr, betas, eps, decay)
                got = opt.state[p].get("master", p)
                assert_within(got.reshape(-1), torch.from_numpy(want), torch.from_numpy(bound), n)
        for n, p in block.named_parameters():
            assert bool(p.grad.isfinite().all()) and bool(p.isfinite().all()), n
            if "master" in opt.state[p]:
                assert torch.equal(p, opt.state[p]["master"].to(p.dtype))
        opt.zero_grad()
        block.advance()
    assert lib.last_device_status() == 0


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_optimizer_steps(bits):
    """Replays of a captured step go on counting; states that are loaded land in the graph's tensors."""
    def make():
        torch.manual_seed(4)
        ps = [torch.nn.Parameter(torch.randn(s, device=DEV).to(t)) for s, t in (((300, 70), torch.bfloat16), ((500,), torch.float32))]
        for p in ps:
            p.grad = torch.randn_like(p)
        return ps
    a, b = make(), make()
    oa, ob = AdamW(a, state_bits=bits, capturable=True), AdamW(b, state_bits=bits)
    fresh = AdamW(make(), capturable=True)
    with pytest.raises(RuntimeError, match="before the capture"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            fresh.step()
    oa.step()
    saved = oa.state_dict()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        oa.step()
    for _ in range(3):
        graph.replay()
    for _ in range(4):
        ob.step()
    for p, q in zip(a, b):
        assert torch.equal(p, q)
        assert all(torch.equal(oa.state[p][k], ob.state[q][k]) for k in oa.state[p] if torch.is_tensor(oa.state[p][k]))
    d = oa.state_dict()
    assert [s["step"] for s in d["state"].values()] == [4, 4] and [s["step"] for s in saved["state"].values()] == [1, 1]
    oa.load_state_dict(ob.state_dict())
    graph.replay()
    ob.step()
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    with pytest.raises(RuntimeError, match="capturable"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            ob.step()


def test_wrappers_match_the_calls_they_wrap():
    g = torch.Generator(device=DEV)
    g.manual_seed(0)
    n = lambda *s: torch.randn(*s, generator=g, device=DEV).to(torch.bfloat16)
    q, k, dq, dk = (n(2, 40, h, 64) for h in (4, 2, 4, 2))
    w = [torch.rand(64, generator=g, device=DEV).requires_grad_() for _ in range(2)]
    f, _ = lib.rotary_frequencies(64)
    q.requires_grad_()
    k.requires_grad_()
    torch.autograd.backward(A.rotary(q, k, f, 7), (dq, dk))
    want = lib.rotary(dq, dk, f, 7, inverse=True)
    assert torch.equal(q.grad, want[0]) and torch.equal(k.grad, want[1])
    q.grad = k.grad = None
    torch.autograd.backward(A.qk_norm_rotary(q, k, *w, f, 7), (dq, dk))
    want = lib.qk_norm_rotary_backward(dq, dk, q.detach(), k.detach(), *(t.detach() for t in w), f, 7)
    assert all(torch.equal(t.grad, x) for t, x in zip((q, k, *w), want))
    q.grad = None
    A.qk_norm_rotary(q, None, None, None, f)[0].sum().backward()           # an expanded gradient, no keys, no weights
    assert bool(q.grad.isfinite().all())
    v, do = n(2, 40, 2, 64), n(2, 40, 4, 64)
    kw = dict(causal=True, window_left=9, sinks=3)
    A.attention(q, k, v, **kw).backward(do)
    o, lse = lib.attention(q.detach(), k.detach(), v, **kw)
    assert bool(lse.isfinite().all())
    q.grad = None
    A.attention(q, k, v, **kw).backward(do)
    assert torch.equal(q.grad, lib.attention_backward(do, q.detach(), k.detach(), v, o, lse, **kw)[0])
