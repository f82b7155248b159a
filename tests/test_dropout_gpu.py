"""ue5m3_dropout_add against the generator's definition (masks equal, values within one rounding)."""
import pytest
import torch

import paper_2609_02846_b200 as lib
from block_reference import assert_within, draws, dropout_add

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F = torch.bfloat16, torch.float32
SEED = 0x1234_5678_9ABC_DEF0


def make(rows, cols, dt, seed=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(rows, cols, generator=g, device=DEV).to(dt), (3 * torch.randn(rows, cols, generator=g, device=DEV)).to(dt)


def check(x, res, p, seed=SEED, out=None):
    y = lib.dropout_add(x, p, seed, res, out=out)
    torch.cuda.synchronize()
    want, keep = dropout_add(x, p, seed, res)
    # one product and one sum in binary32
    bound = 2.0 ** -23 * (want.abs() + (0 if res is None else 2 * res.double().abs()))
    assert_within(y, want, bound, "y")
    base = torch.zeros_like(x) if res is None else res
    assert torch.equal(y[~keep], base[~keep])                # exactly nothing is added where an element is dropped
    return y, keep


@pytest.mark.parametrize("dt", [BF, F])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (3, 8), (5, 9), (77, 129), (64, 4096), (1000, 333), (513, 1024)])
@pytest.mark.parametrize("residual", [False, True])
def test_sizes(rows, cols, dt, residual):
    x, res = make(rows, cols, dt, rows)
    check(x, res if residual else None, 0.1)


@pytest.mark.parametrize("p", [0.0, 1e-6, 1.0 / 65536, 0.25, 0.5, 0.9, 1.0 - 2.0 ** -16, 1.0])
def test_probabilities(p):
    x, res = make(50, 264, BF)
    x[3, 5], x[4, 6], x[5, 7] = float("nan"), float("inf"), -float("inf")
    y = lib.dropout_add(x, p, SEED, res)
    want, keep = dropout_add(x, p, SEED, res)
    assert bool((y.isnan() == want.isnan()).all()) and torch.equal(y[~keep], res[~keep])
    fine = want.isfinite()
    assert_within(y[fine], want[fine], 2.0 ** -22 * (want.abs() + res.double().abs())[fine])
    t = int(p * 65536 + 0.5)
    n = keep.numel()
    sigma = (n * (t / 65536) * (1 - t / 65536)) ** 0.5
    assert abs(int((~keep).sum()) - n * t / 65536) <= 6 * sigma + 1e-9


def test_backward_is_the_same_call_without_a_residual():
    """The mask of dy is the mask of x: with p and seed alike both are zero at the same elements and scaled alike."""
    x, res = make(200, 520, F)
    dy = torch.randn(200, 520, device=DEV)
    ones = lib.dropout_add(torch.ones_like(x), 0.3, 99)
    assert torch.allclose(lib.dropout_add(x, 0.3, 99, res), x * ones + res, atol=1e-5)
    assert torch.equal(lib.dropout_add(dy, 0.3, 99), dy * ones)
    # differences: the call is linear in x
    u = torch.randn_like(x)
    d = (lib.dropout_add(x + u, 0.3, 99, res).double() - lib.dropout_add(x - u, 0.3, 99, res).double()) / 2
    assert abs(float((d * dy).sum() - (lib.dropout_add(dy, 0.3, 99).double() * u).sum())) < 1e-3 * float((dy.double() * u).norm())


def test_draws_depend_on_seed_and_index_only():
    x, res = make(96, 1024, BF)
    y, keep = check(x, res, 0.5, 7)
    assert torch.equal(lib.dropout_add(x.view(192, 512), 0.5, 7, res.view(192, 512)).view(96, 1024), y)
    _, other = check(x, res, 0.5, 8)
    share = float((keep == other).float().mean())
    assert abs(share - 0.5) < 0.01
    assert not (draws(4096, 7) == draws(4096, 7 + (1 << 40))).all()


@pytest.mark.parametrize("pad,start", [(8, 0), (16, 8), (1, 0), (3, 5)])
@pytest.mark.parametrize("cols", [256, 100, 33])
def test_strides_and_alignment(pad, start, cols):
    x, res = make(40, cols, BF)
    cut = lambda t: torch.zeros(40, cols + pad + start, dtype=BF, device=DEV)[:, start:start + cols].copy_(t)
    want, _ = check(x, res, 0.2)
    for xs, rs in ((cut(x), cut(res)), (x, cut(res)), (cut(x), res)):
        holder = torch.full((40, cols + pad + start), 9.0, dtype=BF, device=DEV)
        out = holder[:, start:start + cols]
        assert torch.equal(lib.dropout_add(xs, 0.2, SEED, rs, out=out), want)
        assert bool((holder[:, start + cols:] == 9.0).all()) and bool((holder[:, :start] == 9.0).all())
    z = res.clone()
    lib.dropout_add(x, 0.2, SEED, z, out=z)
    assert torch.equal(z, want)


def test_indexes_over_32_bits():
    """A tall strided view: element offsets pass 2^32 while the logical index stays small."""
    big = torch.zeros((1 << 32) + 4096, dtype=torch.bfloat16, device=DEV)
    ld = 1 << 30
    x = big.as_strided((5, 64), (ld, 1))
    src, _ = make(5, 64, BF)
    x.copy_(src)
    assert torch.equal(lib.dropout_add(x, 0.5, 3), lib.dropout_add(src, 0.5, 3))
    w = torch.ones(64, device=DEV)
    assert torch.equal(lib.layer_norm(x, w)[0], lib.layer_norm(src, w)[0])


def test_empty_and_refusals():
    x, res = make(8, 64, BF)
    assert lib.dropout_add(x[:0], 0.1, 1).shape == (0, 64) and lib.dropout_add(x[:, :0], 0.1, 1).shape == (8, 0)
    for p in (-0.1, 1.1, float("nan")):
        with pytest.raises(lib.Ue5m3Error, match="INVALID_ARG"):
            lib.dropout_add(x, p, 1)
    for bad in (res[:7], res.float(), res.cpu()):
        with pytest.raises(ValueError):
            lib.dropout_add(x, 0.1, 1, bad)
    with pytest.raises(TypeError):
        lib.dropout_add(x.half(), 0.1, 1)
    with pytest.raises(ValueError):
        lib.dropout_add(x.t(), 0.1, 1)
    with pytest.raises(lib.Ue5m3Error, match="INVALID_ARG"):
        lib.dropout_add(x[:1].expand(8, 64), 0.1, 1)
