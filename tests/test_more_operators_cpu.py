"""Host-side rules of rotary positions, norms of queries and keys, attention with sinks and the AdamW step: refusals, workspaces, frequencies, the
optimizer's bookkeeping (no GPU)."""
import copy
import ctypes as C
import math

import pytest
import torch

import paper_2609_02846_b200.autograd as A
import paper_2609_02846_b200.binding as B
import paper_2609_02846_b200.optimizer as O
from paper_2609_02846_b200.build import build_library

OK, INVALID, SHAPE, ALIGN, UNSUPPORTED = 0, 1, 2, 3, 4
P = 1 << 20


@pytest.fixture(scope="module")
def lib():
    build_library()
    return B._load()


def _turn(batch=2, tokens=8, heads=4, kv_heads=2, dim=64, rot=64, frequencies=P, positions=None, stride=0, bytes_=0, interleaved=0, amplitude=1.0,
          dtype=B.BF16):
    return B._RotaryShape(batch, tokens, heads, kv_heads, dim, rot, frequencies, positions, stride, 0, bytes_, interleaved, amplitude, dtype)


def _tensors(dim=64, heads=4, kv_heads=2, tokens=8, at=1 << 20, gap=1 << 16):
    """q, k, q_out, k_out, far from one another."""
    t = lambda i, h: B._Heads(at + i * gap, tokens * h * dim, h * dim, dim)
    return t(0, heads), t(1, kv_heads), t(2, heads), t(3, kv_heads)


@pytest.mark.parametrize("bad,status", [
    (dict(rot=65), SHAPE), (dict(rot=66), SHAPE), (dict(rot=0), INVALID), (dict(dim=63, rot=62), SHAPE), (dict(dim=258), UNSUPPORTED), (dict(heads=0), INVALID),
    (dict(kv_heads=-1), INVALID), (dict(batch=-1), INVALID), (dict(frequencies=None), INVALID), (dict(frequencies=P + 4), ALIGN),
    (dict(positions=P, bytes_=2), INVALID), (dict(positions=P + 4, bytes_=8), ALIGN), (dict(interleaved=2), INVALID),
    (dict(amplitude=float("nan")), INVALID), (dict(amplitude=float("inf")), INVALID), (dict(dtype=5), INVALID)])
def test_rotary_shapes_that_are_refused(lib, bad, status):
    s, (q, k, qo, ko) = _turn(**bad), _tensors()
    assert lib.ue5m3_rotary(s, 0, q, k, qo, ko, None) == status
    assert lib.ue5m3_qk_norm_rotary(s, q, k, None, None, B.F32, 1e-6, qo, ko, None) == status
    assert lib.ue5m3_qk_norm_rotary_backward(s, qo, ko, q, k, None, None, B.F32, 1e-6, q, k, None, None, None, None) == status
    assert lib.ue5m3_qk_norm_rotary_backward_workspace_bytes(s) == 0


def test_rotary_calls_refuse_before_they_look_for_a_device(lib):
    s, (q, k, qo, ko) = _turn(), _tensors()
    f = lambda **kw: lib.ue5m3_rotary(kw.get("s", s), kw.get("inverse", 0), kw.get("q", q), kw.get("k", k), kw.get("qo", qo), kw.get("ko", ko), None)
    assert f(inverse=2) == INVALID and f(q=None) == INVALID and f(ko=None) == INVALID
    assert f(q=B._Heads(P + 1, 2048, 256, 64)) == ALIGN and f(q=B._Heads(None, 2048, 256, 64)) == INVALID
    assert f(q=B._Heads(P, 0, 256, 64)) == ALIGN and f(q=B._Heads(P, 2048, -256, 64)) == ALIGN
    # outputs over what is still to be read
    assert f(qo=k) == INVALID and f(ko=q) == INVALID and f(ko=qo) == INVALID
    assert f(qo=B._Heads(P + 2 * 64, 2048, 256, 64)) == INVALID                      # a head further
    g = lambda **kw: lib.ue5m3_qk_norm_rotary(s, q, k, kw.get("w", P), P, kw.get("wd", B.F32), kw.get("eps", 1e-6), qo, ko, None)
    assert g(w=P + 2) == ALIGN and g(wd=3) == INVALID and g(eps=-1.0) == INVALID and g(eps=float("nan")) == INVALID
    b = lambda **kw: lib.ue5m3_qk_norm_rotary_backward(s, kw.get("dq", qo), ko, q, k, P, P, B.F32, 1e-6, q, k, kw.get("dw", P), P, kw.get("ws", P), None)
    assert b(ws=None) == INVALID and b(ws=P + 8) == ALIGN and b(dq=None) == INVALID and b(dw=P + 1) == ALIGN
    assert lib.ue5m3_qk_norm_rotary_backward_workspace_bytes(s) == 148 * 4 * 2 * 64 * 4


def test_rotary_in_place_views_of_one_projection_are_no_overlap(lib):
    """Where the check of overlaps passes, the next refusal is the missing device (or, with one, nothing): never INVALID."""
    s = _turn(heads=4, kv_heads=2)
    view = lambda h0: B._Heads(P + h0 * 64 * 2, 8 * 8 * 64, 8 * 64, 64)
    if torch.cuda.is_available():
        pytest.skip("would run")
    assert lib.ue5m3_rotary(s, 0, view(0), view(4), view(0), view(4), None) not in (INVALID, SHAPE, ALIGN)
    assert lib.ue5m3_rotary(s, 0, view(0), view(4), view(1), view(5), None) == INVALID


def test_binding_checks_of_rotary():
    q, k, f = torch.zeros(2, 3, 4, 8), torch.zeros(2, 3, 2, 8), torch.zeros(4, dtype=torch.float64)
    for bad in (dict(q=q[0]), dict(k=k[:, :2]), dict(f=f.float()), dict(f=f[::2]), dict(pos=torch.zeros(3)), dict(pos=torch.zeros(4, dtype=torch.int64)),
                dict(pos=torch.zeros(3, 3, dtype=torch.int64)), dict(pos=torch.zeros(2, 6, dtype=torch.int32)[:, ::2])):
        with pytest.raises(ValueError):
            B._rotary_shape(bad.get("q", q), bad.get("k", k), bad.get("f", f), bad.get("pos"), False, 1.0)
    s = B._rotary_shape(q, k, f, torch.zeros(2, 3, dtype=torch.int32), True, 1.5)
    assert (s.position_stride, s.position_bytes, s.interleaved, s.rotary_dim, s.kv_heads) == (3, 4, 1, 8, 2)
    s = B._rotary_shape(q, None, f, 77, False, 1.0)
    assert (s.first_position, s.position_bytes, s.kv_heads) == (77, 0, 0)
    assert B._rotary_shape(q, k, f, torch.zeros(1, 3, dtype=torch.int64).expand(2, 3), False, 1.0).position_stride == 0
    with pytest.raises(ValueError, match="device tensors"):
        B.rotary(q, k, f)


def test_frequencies():
    f, a = B.rotary_frequencies(8, base=100.0, device="cpu")
    assert f.dtype == torch.float64 and a == 1.0 and torch.allclose(f, torch.tensor([1.0, 100 ** -0.25, 0.1, 100 ** -0.75], dtype=torch.float64), rtol=1e-15)
    g, _ = B.rotary_frequencies(8, base=100.0, scaling="linear", factor=4, device="cpu")
    assert torch.equal(g, f / 4)
    g, _ = B.rotary_frequencies(8, base=100.0, scaling="base", factor=4, device="cpu")
    assert g[0] == 1.0 and math.isclose(g[3], f[3] / 4, rel_tol=1e-14)
    g, a = B.rotary_frequencies(64, scaling="parts", factor=8, trained_length=4096, device="cpu")
    f, _ = B.rotary_frequencies(64, device="cpu")
    turns = 4096 * f / (2 * math.pi)
    assert torch.equal(g[turns >= 32], f[turns >= 32]) and torch.allclose(g[turns <= 1], f[turns <= 1] / 8, rtol=1e-15)
    assert bool(((g <= f) & (g >= f / 8 * (1 - 1e-15))).all()) and math.isclose(a, 0.1 * math.log(8) + 1)
    for bad in (dict(rotary_dim=7), dict(rotary_dim=0), dict(rotary_dim=8, base=0.0), dict(rotary_dim=8, scaling="x"), dict(rotary_dim=8, factor=0.5),
                dict(rotary_dim=8, scaling="parts", factor=2), dict(rotary_dim=8, scaling="parts", factor=2, trained_length=9, fast=1, slow=1)):
        with pytest.raises(ValueError):
            B.rotary_frequencies(device="cpu", **bad)


# ---- attention with sinks -----------------------------------------------------------------------
def _shape(batch, q_len, k_len, heads, kv_heads, dim, left=-1):
    return B._AttentionShape(batch, q_len, k_len, heads, kv_heads, dim, left, None, 0.1, B.BF16, 1)


def test_sinks_workspace(lib):
    f, plain = lib.ue5m3_attention_sinks_backward_workspace_bytes, lib.ue5m3_attention_backward_workspace_bytes
    s = _shape(2, 4096, 4096, 32, 8, 128, 1023)
    assert f(s, 0) == plain(s) and f(s, -1) == 0 and f(s, 129) == 0
    # 32 query tiles see the first keys; half of an SM's share is 32 * 16 * 9 / 296 = 15: three parts of binary32 dk and dv of 128 keys
    assert f(s, 4) - plain(s) == 3 * 16 * 2 * 128 * 128 * 4
    assert f(_shape(2, 4096, 4096, 32, 8, 128), 4) == plain(_shape(2, 4096, 4096, 32, 8, 128))          # no window: no sinks
    assert f(_shape(1, 300, 300, 2, 2, 64, 299), 4) == plain(_shape(1, 300, 300, 2, 2, 64))
    assert f(_shape(0, 300, 300, 2, 2, 64, 9), 4) == plain(_shape(0, 300, 300, 2, 2, 64, 9))


def test_sinks_are_refused_out_of_range(lib):
    t = B._Heads(P, 1024, 128, 64)
    for sinks, status in ((-1, INVALID), (129, UNSUPPORTED)):
        assert lib.ue5m3_attention_sinks(_shape(2, 8, 8, 2, 2, 64, 3), sinks, t, t, t, t, P, None, None) == status
        assert lib.ue5m3_attention_sinks_backward(_shape(2, 8, 8, 2, 2, 64, 3), sinks, t, t, t, t, t, P, t, t, t, P, None) == status


# ---- AdamW --------------------------------------------------------------------------------------
class _Tensor(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("param", "grad", "master", "m", "v", "m_scale", "v_scale")] + \
        [("n", C.c_int64), ("stream", C.c_uint32), ("param_dtype", C.c_uint8), ("grad_dtype", C.c_uint8), ("reserved", C.c_uint16)]


def test_adamw_refusals(lib):
    assert C.sizeof(_Tensor) == 72

    def call(tensor=None, count=1, **step):
        t = _Tensor(**{**dict(param=P, grad=P, m=P, v=P, m_scale=P, v_scale=P, n=5, param_dtype=B.F32, grad_dtype=B.BF16), **(tensor or {})})
        s = B._AdamwStep(*[{**dict(step=1, lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1, grad_scale=None, clock=None, seed=0, state_bits=32), **step}[n]
                           for n, _ in B._AdamwStep._fields_])
        return lib.ue5m3_adamw(C.addressof(t) if count else None, count, s, None)
    for bad in (dict(step=0), dict(lr=-1.0), dict(lr=math.nan), dict(lr=math.inf), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1e-8), dict(weight_decay=math.nan),
                dict(state_bits=16), dict(state_bits=8, eps=0.0), dict(count=-1)):
        assert call(**bad) == INVALID, bad
    assert call(grad_scale=P + 2) == ALIGN and call(clock=P + 4) == ALIGN
    for bad in (dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(n=-1), dict(param_dtype=2), dict(grad_dtype=9)):
        assert call(bad) == INVALID, bad
    assert call(dict(m_scale=None), state_bits=8) == INVALID and call(dict(v_scale=P + 2), state_bits=8) == ALIGN
    for bad in (dict(param=P + 2), dict(grad=P + 1), dict(master=P + 2), dict(m=P + 1), dict(v=P + 3)):
        assert call(bad) == ALIGN, bad
    assert call(dict(n=(1 << 35) + 1)) == UNSUPPORTED
    assert lib.ue5m3_adamw(None, 0, None, None) == INVALID


def test_adamw_binding_checks():
    x = lambda n=6, dtype=torch.float32: torch.zeros(n, dtype=dtype)
    B.adamw([], [], [], [])
    for bad in (dict(g=[]), dict(g=[x(5)]), dict(m=[x(5)]), dict(m=[x(6, torch.bfloat16)]), dict(master=[x(6, torch.bfloat16)]), dict(master=[]),
                dict(m_scale=[x(1)]), dict(p=[x(12)[::2]]), dict(streams=[1, 2])):
        with pytest.raises(ValueError):
            B.adamw(bad.pop("p", [x()]), bad.pop("g", [x()]), bad.pop("m", [x()]), [x()], **bad)
    p = x()
    with pytest.raises(ValueError, match="twice"):
        B.adamw([p, p], [x(), x()], [x(), x()], [x(), x()])
    with pytest.raises(ValueError):
        B.adamw([p], [x()], [x(6, torch.uint8)], [x(6, torch.uint8)], m_scale=[x(2)], v_scale=[x(1)])
    with pytest.raises(TypeError):
        B.adamw([x(6, torch.float16)], [x(6, torch.float16)], [x()], [x()])
    with pytest.raises(ValueError, match="device tensors"):
        B.adamw([p], [x()], [x()], [x()])


@pytest.fixture
def steps(monkeypatch):
    """Calls that reach the library, with a step that adds the gradient in its place."""
    seen = []

    def adamw(ps, gs, m, v, step, **kw):
        seen.append(dict(n=len(ps), step=step, **kw))
        for i, (p, g) in enumerate(zip(ps, gs)):
            m[i].add_(1)
            w = p if kw["master"] is None or kw["master"][i] is None else kw["master"][i]
            w.add_(g, alpha=-kw["lr"])
            p.copy_(w)
    monkeypatch.setattr(O.B, "adamw", adamw)
    return seen


def _params():
    return [torch.nn.Parameter(torch.ones(300)), torch.nn.Parameter(torch.ones(4, 4, dtype=torch.bfloat16)), torch.nn.Parameter(torch.ones(2))]


def test_optimizer_groups_parameters_by_their_step(steps):
    ps = _params()
    opt = O.AdamW([{"params": ps[:2]}, {"params": ps[2:], "lr": 0.5}], lr=0.1, state_bits=8)
    for p in ps:
        p.grad = torch.ones_like(p)
    ps[1].grad = None
    opt.step()
    ps[1].grad = torch.ones_like(ps[1])
    version = ps[0]._version
    opt.step()
    assert [(s["n"], s["step"], s["lr"], s["streams"]) for s in steps] == [(1, 1, 0.1, (0,)), (1, 1, 0.5, (2,)), (1, 2, 0.1, (0,)), (1, 1, 0.1, (1,)), (1, 2, 0.5, (2,))]
    assert opt.state[ps[0]]["m"].dtype == torch.uint8 and opt.state[ps[0]]["m_scale"].numel() == 2 and "master" not in opt.state[ps[0]]
    assert opt.state[ps[1]]["master"].dtype == torch.float32 and ps[0]._version > version + 1


def test_optimizer_state_keeps_its_types(steps):
    ps = _params()
    opt = O.AdamW(ps, state_bits=8)
    for p in ps:
        p.grad = torch.ones_like(p)
    opt.step()
    saved = copy.deepcopy(opt.state_dict())
    other = [torch.nn.Parameter(p.detach().clone()) for p in ps]
    new = O.AdamW(other, state_bits=8, lr=7.0)
    new.load_state_dict(saved)
    for p, q in zip(ps, other):
        assert opt.state[p].keys() == new.state[q].keys() and new.state[q]["step"] == 1
        for key, value in opt.state[p].items():
            if torch.is_tensor(value):
                assert torch.equal(value, new.state[q][key]) and value.dtype == new.state[q][key].dtype and value.data_ptr() != new.state[q][key].data_ptr()
    assert new.param_groups[0]["lr"] == 1e-3
    there = opt.state[ps[0]]["m"]
    for p in ps:
        p.grad = torch.ones_like(p)
    opt.step()
    opt.load_state_dict(saved)
    assert opt.state[ps[0]]["m"] is there and int(there[0]) == 1 and opt.state[ps[0]]["step"] == 1          # written in place
    with torch.no_grad():
        ps[1].fill_(3.0)
    opt.take_over_weights()
    assert bool((opt.state[ps[1]]["master"] == 3).all())


def test_optimizer_refuses(steps):
    for bad in (dict(state_bits=16), dict(lr=-1.0), dict(betas=(1.0, 0.9)), dict(eps=0.0, state_bits=8), dict(weight_decay=-1.0), dict(lr=math.nan)):
        with pytest.raises(ValueError):
            O.AdamW(_params(), **bad)
    p = torch.nn.Parameter(torch.ones(4, 6).t())
    p.grad = torch.ones_like(p)
    with pytest.raises(ValueError, match="contiguous"):
        O.AdamW([p]).step()
    assert O.AdamW(_params()).step(lambda: 5) == 5 and not steps


# ---- the differentiable wrappers, with plain arithmetic in place of the library ------------------
def _plain_rotary(q, k, f, positions=None, interleaved=False, amplitude=1.0, inverse=False, out=None):
    def one(x):
        if x is None:
            return None
        t = torch.arange(x.shape[1])[:, None] * f.float() * (-1 if inverse else 1)
        c, s = t.cos()[:, None] * amplitude, t.sin()[:, None] * amplitude
        h = f.numel()
        a, b = x[..., :h], x[..., h:2 * h]
        return torch.cat([a * c - b * s, a * s + b * c, x[..., 2 * h:]], -1)
    with torch.no_grad():
        return one(q), one(k)


def _plain_norm_backward(dq, dk, q, k, wq, wk, *args, want_weights=True):
    with torch.enable_grad():
        outs, grads = [], []
        for x, d, w in ((q, dq, wq), (k, dk, wk)):
            ins = [x.detach().requires_grad_()] + ([w.detach().requires_grad_()] if w is not None else [])
            y = ins[0] * torch.rsqrt((ins[0] ** 2).mean(-1, keepdim=True) + args[-1]) * (ins[1] if w is not None else 1)
            back = _plain_rotary(d.detach(), None, *args[:-1], True)[0]
            got = torch.autograd.grad(y, ins, back)
            outs.append(got[0])
            grads.append(got[1] if w is not None and want_weights else None)
        return *outs, *grads


def _plain_norm(q, k, wq, wk, f, positions, interleaved, amplitude, eps):
    n = lambda x, w: x * torch.rsqrt((x ** 2).mean(-1, keepdim=True) + eps) * (1 if w is None else w)
    with torch.no_grad():
        return _plain_rotary(n(q, wq), n(k, wk), f, positions, interleaved, amplitude)


def test_wrappers_of_rotary(monkeypatch):
    for name, fn in dict(rotary=_plain_rotary, qk_norm_rotary=_plain_norm, qk_norm_rotary_backward=_plain_norm_backward).items():
        monkeypatch.setattr(A.B, name, fn)
    f, _ = B.rotary_frequencies(4, device="cpu")
    torch.manual_seed(0)
    q, k, wq, wk = (torch.randn(s, dtype=torch.float64, requires_grad=True) for s in ((1, 3, 2, 6), (1, 3, 1, 6), (6,), (6,)))
    f = f.double()
    monkeypatch.setattr(torch.Tensor, "float", lambda t: t.double())        # differences in 64 bits
    assert torch.autograd.gradcheck(lambda a, b: A.rotary(a, b, f, amplitude=1.2), (q, k))
    assert torch.autograd.gradgradcheck(lambda a, b: A.rotary(a, b, f, amplitude=1.2), (q, k))
    assert torch.autograd.gradcheck(lambda a, b, u, v: A.qk_norm_rotary(a, b, u, v, f), (q, k, wq, wk))
    y, z = A.qk_norm_rotary(q, k, wq, wk, f)
    g, = torch.autograd.grad((y.sum() + z.sum()), q, create_graph=True)
    with pytest.raises(RuntimeError, match="no second derivative"):
        (g ** 2).sum().backward()
    y, z = A.qk_norm_rotary(q, k, None, wk, f)                  # one side's output used alone; an expanded gradient
    y.sum().backward()
    assert q.grad.shape == q.shape and not k.grad.any() and wq.grad is None
