"""Rotary positions of queries and keys, alone and behind the norm of every head's row, against 64 bits."""
import math

import pytest
import torch

import paper_2609_02846_b200 as lib
from block_reference import assert_within
import rotary_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F = torch.bfloat16, torch.float32


def _gen(seed=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _inputs(B, L, H, Hk, D, dtype, seed=0, fused=True):
    """q and k as views of a fused projection (with a value part), or on their own."""
    g = _gen(seed)
    if fused:
        qkv = torch.randn(B, L, H + 2 * Hk, D, generator=g, device=DEV).to(dtype)
        return qkv[:, :, :H], qkv[:, :, H:H + Hk]
    return torch.randn(B, L, H, D, generator=g, device=DEV).to(dtype), torch.randn(B, L, Hk, D, generator=g, device=DEV).to(dtype)


def _positions(kind, B, L, seed=1):
    """(what the call takes, [B, L] positions)"""
    g = _gen(seed)
    if kind is None:
        return None, torch.arange(L, device=DEV)[None].expand(B, L)
    if kind == "start":
        return 12345, 12345 + torch.arange(L, device=DEV)[None].expand(B, L)
    if kind == "row":
        p = torch.randint(0, 1 << 20, (L,), generator=g, device=DEV)
        return p, p[None].expand(B, L)
    p = torch.randint(-5, 1 << 30 if kind == "far" else 4096, (B, L), generator=g, device=DEV)
    if kind == "int32":
        return p.int(), p
    if kind == "strided":
        wide = torch.zeros(B, L + 3, dtype=torch.int64, device=DEV)
        wide[:, :L] = p
        return wide[:, :L], p
    return p, p


# B, L, H, Hk, D, R, neighbours, dtype, positions: the vector widths (16, 8, 4 and 2 bytes), whole and partial rotation, lanes left over
CASES = [
    (2, 37, 32, 8, 128, 128, False, BF, None), (16, 1, 32, 8, 128, 128, False, BF, "far"), (1, 1, 1, 1, 2, 2, True, BF, "start"),
    (3, 19, 5, 5, 80, 80, False, BF, "row"), (2, 9, 6, 2, 72, 72, False, BF, "int32"), (2, 9, 6, 2, 72, 36, False, BF, "strided"),
    (2, 9, 3, 1, 64, 46, False, BF, "far"), (2, 9, 3, 1, 64, 46, True, BF, "far"), (1, 33, 4, 4, 256, 64, True, BF, None),
    (1, 33, 4, 4, 256, 256, False, BF, None), (1, 7, 3, 3, 250, 10, False, BF, None), (1, 7, 3, 3, 250, 250, True, BF, None),
    (2, 37, 32, 8, 128, 128, False, F, "far"), (3, 21, 16, 4, 80, 40, True, F, "row"), (2, 9, 3, 1, 66, 34, False, F, None),
    (2, 9, 3, 3, 256, 254, False, F, None), (2, 9, 3, 1, 100, 100, True, F, "start"), (1, 2500, 4, 1, 64, 64, False, BF, None),
]


@pytest.mark.parametrize("B,L,H,Hk,D,R,neighbours,dtype,positions", CASES)
def test_rotary_forwards_and_back(B, L, H, Hk, D, R, neighbours, dtype, positions):
    q, k = _inputs(B, L, H, Hk, D, dtype)
    f, _ = lib.rotary_frequencies(R)
    at, pos = _positions(positions, B, L)
    for inverse, amplitude in ((False, 1.0), (True, 1.25)):
        out = lib.rotary(q, k, f, at, interleaved=neighbours, amplitude=amplitude, inverse=inverse)
        for got, x, name in zip(out, (q, k), "qk"):
            want, bound = ref.rotary(x, f, pos, neighbours, amplitude, inverse)
            assert_within(got, want, bound, name)
            assert torch.equal(got[..., R:], x[..., R:])


@pytest.mark.parametrize("wdtype", [F, BF, None])
@pytest.mark.parametrize("B,L,H,Hk,D,R,neighbours,dtype,positions", CASES)
def test_norm_and_rotary(B, L, H, Hk, D, R, neighbours, dtype, positions, wdtype):
    if wdtype == BF and dtype == F:
        pytest.skip("a float32 model has float32 weights")
    q, k = _inputs(B, L, H, Hk, D, dtype)
    g = _gen(2)
    wq, wk = (None, None) if wdtype is None else ((1 + 0.3 * torch.randn(D, generator=g, device=DEV)).to(wdtype) for _ in range(2))
    f, _ = lib.rotary_frequencies(R)
    at, pos = _positions(positions, B, L)
    out = lib.qk_norm_rotary(q, k, wq, wk, f, at, interleaved=neighbours, amplitude=0.75, eps=1e-5)
    for got, x, w, name in zip(out, (q, k), (wq, wk), "qk"):
        want, bound = ref.qk_norm_rotary(x, w, f, pos, neighbours, 0.75, 1e-5)
        assert_within(got, want, bound, name)


def _chain(B, L, H):
    """Most values that one sum of a weight's gradient takes one after the other: the heads of a warp's tokens, then lanes, warps and CTAs."""
    return H * math.ceil(B * L / 500) + 5 + 4 + 64


@pytest.mark.parametrize("wdtype", [F, BF])
@pytest.mark.parametrize("B,L,H,Hk,D,R,neighbours,dtype,positions", CASES)
def test_backward(B, L, H, Hk, D, R, neighbours, dtype, positions, wdtype):
    if wdtype == BF and dtype == F:
        pytest.skip("a float32 model has float32 weights")
    q, k = _inputs(B, L, H, Hk, D, dtype)
    dq, dk = _inputs(B, L, H, Hk, D, dtype, seed=5, fused=False)
    g = _gen(2)
    wq, wk = ((1 + 0.3 * torch.randn(D, generator=g, device=DEV)).to(wdtype) for _ in range(2))
    f, _ = lib.rotary_frequencies(R)
    at, pos = _positions(positions, B, L)
    out = lib.qk_norm_rotary_backward(dq, dk, q, k, wq, wk, f, at, interleaved=neighbours, amplitude=0.75, eps=1e-5)
    for i, (x, dy, w, name) in enumerate(((q, dq, wq, "q"), (k, dk, wk, "k"))):
        (dx, bound), (dw, bound_dw) = ref.qk_norm_rotary_backward(dy, x, w, f, pos, neighbours, 0.75, 1e-5, _chain(B, L, max(H, Hk)))
        assert_within(out[i], dx, bound, "d" + name)
        assert_within(out[2 + i], dw, bound_dw, "weight of " + name)
    again = lib.qk_norm_rotary_backward(dq, dk, q, k, wq, wk, f, at, interleaved=neighbours, amplitude=0.75, eps=1e-5)
    assert all(torch.equal(a, b) for a, b in zip(out, again))


@pytest.mark.parametrize("dtype", [BF, F])
def test_many_tokens_and_many_heads(dtype):
    """More tokens than warps at a time, more heads than a warp has side by side in a step."""
    B, L, H, Hk, D = 3, 1500, 13, 7, 64
    q, k = _inputs(B, L, H, Hk, D, dtype)
    dq, dk = _inputs(B, L, H, Hk, D, dtype, seed=5)
    w = 1 + 0.3 * torch.randn(D, generator=_gen(2), device=DEV)
    f, amplitude = lib.rotary_frequencies(D, scaling="parts", factor=8, trained_length=1024)
    pos = torch.arange(L, device=DEV)[None].expand(B, L)
    out = lib.qk_norm_rotary_backward(dq, dk, q, k, w, w, f, amplitude=amplitude)
    for i, (x, dy, heads) in enumerate(((q, dq, H), (k, dk, Hk))):
        (dx, bound), (dw, bound_dw) = ref.qk_norm_rotary_backward(dy, x, w, f, pos, False, amplitude, 1e-6, _chain(B, L, heads))
        assert_within(out[i], dx, bound)
        assert_within(out[2 + i], dw, bound_dw)


@pytest.mark.parametrize("offset", [0, 1])
def test_addresses_that_are_not_aligned_and_outputs_over_inputs(offset):
    B, L, H, Hk, D = 2, 11, 6, 2, 64
    flat = torch.randn(B * L * (H + Hk) * D + offset, generator=_gen(), device=DEV).to(BF)
    x = flat[offset:].view(B, L, H + Hk, D)
    q, k = x[:, :, :H], x[:, :, H:]
    f, _ = lib.rotary_frequencies(D)
    want = lib.rotary(q.clone(), k.clone(), f)
    lib.rotary(q, k, f, out=(q, k))
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    dq, dk = _inputs(B, L, H, Hk, D, BF, seed=3)
    w = torch.rand(D, generator=_gen(4), device=DEV)
    want = lib.qk_norm_rotary_backward(dq, dk, q, k, w, w, f)
    got = lib.qk_norm_rotary_backward(dq, dk, q, k, w, w, f, out=(dq, dk))
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and got[0] is dq


def test_queries_alone_and_weights_that_nobody_wants():
    q, _ = _inputs(2, 5, 4, 1, 64, BF, fused=False)
    dq, _ = _inputs(2, 5, 4, 1, 64, BF, seed=3, fused=False)
    f, _ = lib.rotary_frequencies(64)
    w = torch.rand(64, generator=_gen(4), device=DEV)
    assert lib.rotary(q, None, f)[1] is None
    both = lib.rotary(q, q, f)
    assert torch.equal(lib.rotary(q, None, f)[0], both[0]) and torch.equal(both[0], both[1])
    a = lib.qk_norm_rotary_backward(dq, None, q, None, w, None, f)
    b = lib.qk_norm_rotary_backward(dq, dq, q, q, w, w, f)
    c = lib.qk_norm_rotary_backward(dq, dq, q, q, w, w, f, want_weights=False)
    assert torch.equal(a[0], b[0]) and a[1] is None and a[3] is None
    # with and without keys the warps share the rows out differently: two orders of one sum
    _, (dw, bound) = ref.qk_norm_rotary_backward(dq, q, w, f, torch.arange(5, device=DEV)[None].expand(2, 5), False, 1.0, 1e-6, _chain(2, 5, 4))
    for x in (a[2], b[2], b[3]):
        assert_within(x, dw, bound)
    assert torch.equal(c[0], b[0]) and c[2] is None


def test_no_tokens_and_rows_of_zeros():
    f, _ = lib.rotary_frequencies(64)
    w = torch.ones(64, device=DEV)
    for shape in ((0, 5, 4, 64), (2, 0, 4, 64)):
        e = torch.empty(shape, device=DEV, dtype=BF)
        assert lib.rotary(e, e, f)[0].shape == e.shape
        out = lib.qk_norm_rotary_backward(e, e, e, e, w, w, f)
        assert not out[2].any() and not out[3].any()
    z = torch.zeros(1, 3, 2, 64, device=DEV)
    assert not lib.qk_norm_rotary(z, z, w, w, f)[0].any()
    out = lib.qk_norm_rotary_backward(torch.ones_like(z), torch.ones_like(z), z, z, w, w, f, eps=1e-6)
    assert bool(out[0].isfinite().all()) and not out[2].any()


@pytest.mark.parametrize("dtype", [BF, F])
def test_an_eps_of_zero_with_heads_left_over(dtype):
    """Places in a warp that no head takes hold zeros: their root is zero, and nothing of them reaches the weights' gradients."""
    B, L, H, Hk, D = 2, 9, 5, 3, 64
    q, k = _inputs(B, L, H, Hk, D, dtype)
    dq, dk = _inputs(B, L, H, Hk, D, dtype, seed=5)
    w = 1 + 0.3 * torch.randn(D, generator=_gen(2), device=DEV)
    f, _ = lib.rotary_frequencies(D)
    pos = torch.arange(L, device=DEV)[None].expand(B, L)
    out = lib.qk_norm_rotary_backward(dq, dk, q, k, w, w, f, eps=0.0)
    for i, (x, dy, heads) in enumerate(((q, dq, H), (k, dk, Hk))):
        (dx, bound), (dw, bound_dw) = ref.qk_norm_rotary_backward(dy, x, w, f, pos, False, 1.0, 0.0, _chain(B, L, heads))
        assert_within(out[i], dx, bound)
        assert_within(out[2 + i], dw, bound_dw)


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("R", [64, 40])
def test_what_is_not_turned_is_kept_as_it_is(neighbours, R):
    q = torch.randn(1, 4, 2, 128, generator=_gen(), device=DEV).to(BF)
    q[..., R] = math.inf
    q[..., 127] = math.nan
    f, _ = lib.rotary_frequencies(R)
    y, _ = lib.rotary(q, None, f, 100, interleaved=neighbours)
    assert bool(y[..., :R].isfinite().all()) and torch.equal(y[..., R:127], q[..., R:127]) and bool(y[..., 127].isnan().all())


def test_gradients_against_differences():
    """Along a direction, of a loss in 64 bits made of the call's own outputs: the third-order rest of a central difference of step h over values of
    size 1 is h^2, the outputs' binary32 error over 2 h is 2^-21 / h: both below 1e-3 of the gradient at h = 2^-7."""
    B, L, H, D = 2, 7, 4, 64
    g = _gen(1)
    n = lambda *s: torch.randn(*s, generator=g, device=DEV)
    q, w, dy = n(B, L, H, D), 1 + 0.1 * n(D), n(B, L, H, D)
    f, _ = lib.rotary_frequencies(32)
    loss = lambda x, u: (lib.qk_norm_rotary(x, None, u, None, f, 50)[0].double() * dy.double()).sum()
    dq, _, dw, _ = lib.qk_norm_rotary_backward(dy, None, q, None, w, None, f, 50)
    h = 2.0 ** -7
    along_q = dq / dq.norm() * math.sqrt(q.numel()) * 0.1
    along_w = dw / dw.norm() * math.sqrt(D) * 0.1
    for slope, want in (((loss(q + h * along_q, w) - loss(q - h * along_q, w)) / (2 * h), (dq.double() * along_q.double()).sum()),
                        ((loss(q, w + h * along_w) - loss(q, w - h * along_w)) / (2 * h), (dw.double() * along_w.double()).sum())):
        assert abs(float(slope / want) - 1) < 1e-2


def test_very_many_heads():
    """More of them than fit any batch, shared out among warps."""
    q, k = _inputs(1, 2, 700, 1, 32, BF, fused=False)
    f, _ = lib.rotary_frequencies(32)
    pos = torch.arange(2, device=DEV)[None]
    for got, x in zip(lib.rotary(q, k, f), (q, k)):
        assert_within(got, *ref.rotary(x, f, pos))


def test_graphs_and_other_streams():
    q, k = _inputs(2, 33, 8, 2, 128, BF)
    f, _ = lib.rotary_frequencies(128)
    w = torch.rand(128, generator=_gen(4), device=DEV)
    pos = torch.arange(33, device=DEV)
    want = lib.qk_norm_rotary_backward(q, k, q, k, w, w, f, pos)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = lib.qk_norm_rotary_backward(q, k, q, k, w, w, f, pos)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = lib.qk_norm_rotary_backward(q, k, q, k, w, w, f, pos)
    pos += 7
    graph.replay()
    want = lib.qk_norm_rotary_backward(q, k, q, k, w, w, f, pos)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
