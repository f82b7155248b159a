"""ue5m3_layer_norm and its backward pass against the formulas in 64 bits."""
import pytest
import torch

import paper_2609_02846_b200 as lib
from block_reference import assert_within, layer_norm, layer_norm_backward

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F = torch.bfloat16, torch.float32


def make(rows, cols, dt, wdt, seed=0, mean=0.5):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device=DEV)
    x = (n(rows, cols) * torch.exp(n(cols)) + mean).to(dt)
    return x, (1 + 0.2 * n(cols)).to(wdt), n(cols).to(wdt), n(rows, cols).to(dt)


def check(x, w, b, dy, eps=1e-5):
    y, mean, rstd = lib.layer_norm(x, w, b, eps)
    dx, dw, db = lib.layer_norm_backward(dy, x, w, mean, rstd, want_bias=b is not None)
    torch.cuda.synchronize()
    wy, wm, wr, by = layer_norm(x, w, b, eps)
    size = x.double().abs().amax(1)
    assert_within(y, wy, by, "y")
    assert_within(mean, wm, 2.0 ** -21 * size, "mean")
    assert_within(rstd, wr, 2.0 ** -20 * wr * (1 + size * wr), "rstd")
    want = layer_norm_backward(dy, x, w, mean, rstd)
    for name, got, (v, bound) in zip(("dx", "dw", "db"), (dx, dw, db), want):
        if got is None:
            assert (name == "dw" and w is None) or (name == "db" and b is None)
        else:
            assert_within(got, v, bound, name)
    return y, mean, rstd, dx, dw, db


@pytest.mark.parametrize("dt,wdt", [(BF, BF), (BF, F), (F, F), (F, BF)])
@pytest.mark.parametrize("cols", [1, 3, 8, 31, 64, 512, 1000, 1537, 4096, 5000, 8192])
def test_widths_and_types(cols, dt, wdt):
    check(*make(37, cols, dt, wdt, seed=cols))


@pytest.mark.parametrize("dt", [BF, F])
@pytest.mark.parametrize("cols", [8200, 8201, 16384, 16385, 20000])
def test_long_rows(cols, dt):
    check(*make(9, cols, dt, F, seed=cols))


@pytest.mark.parametrize("rows", [1, 2, 147, 148, 149, 1000, 5000])
def test_row_counts(rows):
    check(*make(rows, 256, BF, F, seed=rows))
    check(*make(rows, 1030, F, F, seed=rows))


def test_optional_parameters():
    x, w, b, dy = make(50, 768, BF, F)
    for ww, bb in ((None, None), (w, None), (None, b)):
        if ww is None and bb is not None:
            y, mean, rstd = lib.layer_norm(x, None, bb)
            wy, _, _, by = layer_norm(x, None, bb, 1e-5)
            assert_within(y, wy, by, "y")
        else:
            check(x, ww, bb, dy)
    y, mean, rstd = lib.layer_norm(x, w, b)
    full = lib.layer_norm_backward(dy, x, w, mean, rstd)
    assert lib.layer_norm_backward(dy, x, w, mean, rstd, want_weight=False, want_bias=False)[1:] == (None, None)
    only_b = lib.layer_norm_backward(dy, x, w, mean, rstd, want_weight=False)
    assert only_b[1] is None and torch.equal(only_b[2], full[2]) and torch.equal(only_b[0], full[0])
    only_w = lib.layer_norm_backward(dy, x, w, mean, rstd, want_bias=False)
    assert only_w[2] is None and torch.equal(only_w[1], full[1])


def test_a_large_mean_and_constant_rows():
    """Variance from centred values: rows around 1000 with deviation 1e-2; rows without variance give the bias."""
    x, w, b, dy = make(40, 4096, F, F)
    check(1000.0 + 1e-2 * x, w, b, dy)
    y, mean, rstd = lib.layer_norm(torch.full((4, 1024), 3.0, dtype=BF, device=DEV), w[:1024].contiguous(), b[:1024].contiguous(), 1e-5)
    assert torch.equal(y, b[:1024].to(BF).expand(4, 1024)) and bool((mean == 3.0).all())


def test_strides_and_alignment():
    """Leading dimensions, element-aligned starts, in-place output: the values are those of the contiguous tensors."""
    x, w, b, dy = make(60, 640, BF, BF)
    y, mean, rstd = lib.layer_norm(x, w, b)
    dx, dw, db = lib.layer_norm_backward(dy, x, w, mean, rstd)
    for pad, start in ((8, 0), (8, 8), (3, 1), (640, 7)):
        cut = lambda t: torch.zeros(60, 640 + pad + start, dtype=BF, device=DEV)[:, start:start + 640].copy_(t)
        xs, dys = cut(x), cut(dy)
        ys, ms, rs = lib.layer_norm(xs, w, b, out=cut(x))
        assert_within(ys, *[layer_norm(x, w, b, 1e-5)[i] for i in (0, 3)], "y")
        dxs, dws, dbs = lib.layer_norm_backward(dys, xs, w, mean, rstd, out=cut(x))
        for got, (v, bound) in zip((dxs, dws, dbs), layer_norm_backward(dy, x, w, mean, rstd)):
            assert_within(got, v, bound)
    z = x.clone()
    lib.layer_norm(z, w, b, out=z)
    assert torch.equal(z, y)
    z = dy.clone()
    lib.layer_norm_backward(z, x, w, mean, rstd, out=z)
    assert torch.equal(z, dx)


def test_infinities_stay_in_their_row():
    x, w, b, dy = make(30, 512, BF, F)
    y0, m0, r0 = lib.layer_norm(x, w, b)
    x2 = x.clone()
    x2[7, 100] = float("inf")
    x2[8, 3] = float("nan")
    y, _, _ = lib.layer_norm(x2, w, b)
    keep = [i for i in range(30) if i not in (7, 8)]
    assert torch.equal(y[keep], y0[keep]) and bool(y[8].isnan().all()) and bool(y[7].isnan().any())


def test_no_rows():
    x, w, b, dy = make(4, 96, BF, F)
    y, mean, rstd = lib.layer_norm(x[:0], w, b)
    dx, dw, db = lib.layer_norm_backward(dy[:0], x[:0], w, mean, rstd)
    assert y.shape == dx.shape == (0, 96) and bool((dw == 0).all()) and bool((db == 0).all())


def test_same_result_every_time_and_on_other_streams():
    x, w, b, dy = make(3000, 4096, BF, F)
    first = check(x, w, b, dy)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(s):
            y, mean, rstd = lib.layer_norm(x, w, b)
            again = (y, mean, rstd, *lib.layer_norm_backward(dy, x, w, mean, rstd))
        s.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(first, again))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y, mean, rstd = lib.layer_norm(x, w, b)
        again = (y, mean, rstd, *lib.layer_norm_backward(dy, x, w, mean, rstd))
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(first, again))


def test_gradients_against_differences():
    x, w, b, dy = make(6, 200, F, F, seed=3)
    _, mean, rstd = lib.layer_norm(x, w, b)
    grads = lib.layer_norm_backward(dy, x, w, mean, rstd)
    ins = [t.double() for t in (x, w, b)]
    f = lambda a, c, d: (layer_norm(a, c, d, 1e-5)[0] * dy.double()).sum()
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    for i in range(3):
        u = torch.randn(ins[i].shape, generator=g, device=DEV, dtype=torch.float64)
        e = 1e-5
        at = lambda s: f(*[t + s * e * u if j == i else t for j, t in enumerate(ins)])
        want, got = (at(1) - at(-1)) / (2 * e), (grads[i].double() * u).sum()
        assert abs(float(got - want)) <= 1e-5 * float((grads[i].double().abs() * u.abs()).sum()) + 1e-6


def test_refusals():
    x, w, b, dy = make(8, 64, BF, F)
    _, mean, rstd = lib.layer_norm(x, w, b)
    for bad in (w[:63], w[None], torch.ones(128, device=DEV)[::2], w.cpu()):
        with pytest.raises(ValueError):
            lib.layer_norm(x, bad, None)
    with pytest.raises(ValueError):
        lib.layer_norm(x, w, b.to(BF))                       # two types of parameters
    with pytest.raises(TypeError):
        lib.layer_norm(x.half(), None, None)
    with pytest.raises(ValueError):
        lib.layer_norm(x.t(), None, None)
    with pytest.raises(ValueError):
        lib.layer_norm(x.cpu(), None, None)
    for eps in (-1e-5, float("nan"), float("inf")):
        with pytest.raises(lib.Ue5m3Error, match="INVALID_ARG"):
            lib.layer_norm(x, w, b, eps)
    with pytest.raises(lib.Ue5m3Error, match="INVALID_ARG"):
        lib.layer_norm(x[:1].expand(8, 64), w, b)            # rows that lie on one another
    with pytest.raises(lib.Ue5m3Error, match="INVALID_ARG"):
        lib.layer_norm(x[:, :0], None, None)
    with pytest.raises(ValueError):
        lib.layer_norm_backward(dy.float(), x, w, mean, rstd)
    with pytest.raises(ValueError):
        lib.layer_norm_backward(dy[:7], x, w, mean, rstd)
    with pytest.raises(ValueError):
        lib.layer_norm_backward(dy, x, w, mean[:7], rstd)


@pytest.mark.parametrize("dt", [BF, F])
@pytest.mark.parametrize("rows,cols", [(700, 33), (700, 1023), (300, 1024), (300, 1025), (900, 2047), (300, 4607), (300, 4608), (300, 4609), (301, 8192)])
def test_rows_without_alignment(rows, cols, dt):
    """Widths around the limits of the columns a thread holds, every row at another offset from 16 bytes."""
    x, w, b, dy = make(rows, cols, dt, F, seed=cols)
    def odd(t):
        wide = torch.zeros(rows, cols + 3 + cols % 2, dtype=t.dtype, device=DEV)
        return wide[:, 1:cols + 1].copy_(t)
    check(odd(x), w, b, odd(dy))
