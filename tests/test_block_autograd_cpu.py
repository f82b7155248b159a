"""The differentiable wrappers' own rules, with plain arithmetic in place of the library's calls (no GPU)."""
import pytest
import torch

import paper_2609_02846_b200.autograd as A


def _norm(x, w=None, b=None, eps=1e-5):
    mean = x.float().mean(1)
    rstd = 1 / torch.sqrt(((x.float() - mean[:, None]) ** 2).mean(1) + eps)
    y = (x.float() - mean[:, None]) * rstd[:, None] * (1 if w is None else w) + (0 if b is None else b)
    return y.to(x.dtype), mean, rstd


def _norm_backward(dy, x, w, mean, rstd, want_weight=True, want_bias=True, **kw):
    xh = (x.float() - mean[:, None]) * rstd[:, None]
    g = dy.float() * (1 if w is None else w)
    dx = rstd[:, None] * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return dx.to(x.dtype), (dy * xh).sum(0) if want_weight and w is not None else None, dy.sum(0) if want_bias else None


def _keep(n):
    return (torch.arange(n) * 7 % 5 != 0).float() * 1.25


def _dropout(x, p, seed, residual=None, out=None):
    y = x * _keep(x.numel()).view_as(x)
    return y if residual is None else y + residual


def _attention(q, k, v, *args):
    p = torch.einsum("bihd,bjhd->bhij", q, k).softmax(-1)
    return torch.einsum("bhij,bjhd->bihd", p, v), torch.zeros(q.shape[0], q.shape[2], q.shape[1])


def _attention_backward(do, q, k, v, o, lse, *args):
    with torch.enable_grad():
        ins = [t.detach().requires_grad_() for t in (q, k, v)]
        return torch.autograd.grad(_attention(*ins)[0], ins, do.detach())


@pytest.fixture
def calls(monkeypatch):
    for name, fn in dict(layer_norm=_norm, layer_norm_backward=_norm_backward, dropout_add=_dropout, attention=_attention,
                         attention_backward=_attention_backward).items():
        def call(*a, _fn=fn, **kw):
            with torch.no_grad():                         # as the library: outputs without a history
                return _fn(*a, **kw)
        monkeypatch.setattr(A.B, name, call)


def _penalised(f, x):
    """A loss with a gradient penalty whose upstream gradient needs no gradient itself."""
    y = (f(x) * torch.linspace(-1, 1, x.numel()).view_as(x)).sum()
    g, = torch.autograd.grad(y, x, create_graph=True)
    return y + (g ** 2).sum()


def test_second_derivatives_are_refused_where_there_are_none(calls):
    """Without a refusal the penalty's own gradient is dropped in silence, since the loss has another path to x."""
    x = torch.randn(4, 8, requires_grad=True)
    w = torch.randn(8, requires_grad=True)
    for source in (x, w):
        with pytest.raises(RuntimeError, match="second derivative"):
            torch.autograd.grad(_penalised(lambda t: A.layer_norm(t, w), x), source)
    q, k, v = (torch.randn(1, 5, 2, 8, requires_grad=True) for _ in range(3))
    loss = _penalised(lambda t: A.attention(t, k, v), q)
    for source in (q, k, v):
        with pytest.raises(RuntimeError, match="second derivative"):
            torch.autograd.grad(loss, source, retain_graph=True)


def test_linear_refuses_a_second_derivative(monkeypatch):
    monkeypatch.setattr(A.B, "linear_forward", lambda x, w, *a, **kw: ((x.detach() @ w.detach().T), None, w.detach()))
    monkeypatch.setattr(A.B, "linear_backward", lambda dy, x, qw, *a, **kw: (dy.detach() @ qw, dy.detach().T @ x.detach()))
    layer = A.Ue5m3Linear(128, 128, device="cpu", dtype=torch.float32)
    for scale in (layer.scale_x, layer.scale_w, layer.scale_dy):
        monkeypatch.setattr(scale, "get", lambda t, step: None)
    x = torch.randn(128, 128, requires_grad=True)
    for source in (x, layer.weight):
        with pytest.raises(RuntimeError, match="second derivative"):
            torch.autograd.grad(_penalised(layer, x), source)


def test_a_gradient_asked_for_with_its_graph_is_still_a_gradient(calls):
    """create_graph alone changes no value and refuses nothing."""
    x, w, b = torch.randn(4, 8, requires_grad=True), torch.randn(8, requires_grad=True), torch.randn(8, requires_grad=True)
    for ins, f in (((x, w, b), lambda: A.layer_norm(x, w, b)), ((x,), lambda: A.layer_norm(x)), ((x,), lambda: A.dropout_add(x, 0.2, 1))):
        plain = torch.autograd.grad(f().square().sum(), ins)
        graph = torch.autograd.grad(f().square().sum(), ins, create_graph=True)
        assert all(torch.equal(a, c) for a, c in zip(plain, graph))


def test_dropout_has_a_second_derivative(calls):
    """y = keep x: with t = linspace the penalty is sum (keep t)^2, and a second factor x makes it depend on x."""
    x = torch.randn(4, 8, requires_grad=True)
    keep = _keep(32).view(4, 8)
    got, = torch.autograd.grad(_penalised(lambda t: A.dropout_add(t * t, 0.2, 1), x), x)
    t = torch.linspace(-1, 1, 32).view(4, 8)
    want = 2 * keep * t * x.detach() + 8 * (keep * t) ** 2 * x.detach()
    assert torch.allclose(got, want, rtol=1e-5, atol=1e-6)
    # ... also with regard to the upstream gradient alone
    u = torch.randn(4, 8, requires_grad=True)
    g, = torch.autograd.grad(A.dropout_add(x, 0.2, 1), x, u, create_graph=True)
    assert torch.equal(torch.autograd.grad(g.sum(), u)[0], keep)


def test_residual_of_another_shape_gets_a_gradient_of_its_own(calls):
    """The call adds rows to rows, so a residual may come flattened: its gradient has its shape."""
    x, r = torch.randn(2, 3, 8, requires_grad=True), torch.randn(6, 8, requires_grad=True)
    dy = torch.randn(2, 3, 8)
    A.dropout_add(x, 0.2, 1, r).backward(dy)
    assert torch.equal(r.grad, dy.view(6, 8)) and torch.equal(x.grad, dy * _keep(48).view(2, 3, 8))


@pytest.mark.parametrize("shape", [(3, 0), (2, 3, 0), (0, 8), (0, 3, 8), (2, 0, 8)])
def test_empty_tensors(calls, shape):
    """No rows and rows of no columns are matrices like any other."""
    x, r = torch.randn(shape, requires_grad=True), torch.randn(shape, requires_grad=True)
    y = A.dropout_add(x, 0.2, 1, r)
    assert y.shape == shape
    y.sum().backward()
    assert x.grad.shape == r.grad.shape == shape
