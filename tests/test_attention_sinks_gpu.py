"""Attention with a sliding window and first keys that stay visible behind it, against the formulas in 64 bits."""
import math

import pytest
import torch

import paper_2609_02846_b200 as lib
import sinks_reference as ref
import test_attention_edges_gpu as edges
from block_reference import assert_within
from test_attention_gpu import make

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _lens(lens):
    return None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)


def _call(q, k, v, do, **kw):
    o, lse = lib.attention(q, k, v, **kw)
    return o, lse, *lib.attention_backward(do, q, k, v, o, lse, **kw)


def check(q, k, v, do, left, sinks, causal=True, lens=None, scale=None):
    o, lse, *grads = _call(q, k, v, do, causal=causal, window_left=left, k_lens=lens, scale=scale, sinks=sinks)
    torch.cuda.synchronize()
    assert lib.last_device_status() == 0
    wo, wl, bo, bl = ref.attention(sinks, q, k, v, causal, left, lens, scale)
    assert_within(o, wo, bo, "o")
    assert_within(lse, wl, bl, "lse")
    for name, got, (want, bound) in zip(("dq", "dk", "dv"), grads, ref.attention_backward(sinks, do, q, k, v, o, lse, causal, left, lens, scale)):
        assert_within(got, want, bound, name)
    return o, lse, grads


@pytest.mark.parametrize("sinks", [1, 4, 127, 128])
@pytest.mark.parametrize("left", [0, 1, 63, 128, 200])
@pytest.mark.parametrize("causal", [False, True])
def test_windows_and_sinks(left, causal, sinks):
    check(*make(1, 515, 515, 2, 2, 128, seed=left), left, sinks, causal)
    check(*make(1, 300, 700, 2, 1, 64, seed=left + 1), left, sinks, causal)


@pytest.mark.parametrize("Lq,Lk", [(1, 1), (1, 3), (1, 1000), (2, 129), (127, 127), (128, 128), (129, 255), (257, 385), (640, 130), (5, 3), (1000, 1000)])
def test_lengths(Lq, Lk):
    """One token to several tiles; more queries than keys: the first ones see nothing, sinks neither."""
    o, lse, (dq, _, _) = check(*make(1, Lq, Lk, 4, 2, 64, seed=Lq * 1000 + Lk), 40, 3)
    if Lq > Lk:
        assert bool((o[:, :Lq - Lk] == 0).all()) and bool((lse[:, :, :Lq - Lk] == -math.inf).all()) and bool((dq[:, :Lq - Lk] == 0).all())


@pytest.mark.parametrize("H,Hk,D", [(1, 1, 8), (6, 2, 40), (8, 1, 72), (4, 4, 128)])
def test_heads(H, Hk, D):
    check(*make(2, 300, 300, H, Hk, D, seed=D), 50, 5)


@pytest.mark.parametrize("lens", [[500, 0, 3], [1, 260, 499]])
@pytest.mark.parametrize("causal", [False, True])
def test_ragged(lens, causal):
    """Sequences shorter than the sinks, empty ones, and ones that end in front of a query's window: the sinks are all it sees then."""
    o, _, (_, dk, _) = check(*make(3, 500, 500, 2, 1, 64, seed=lens[0]), 100, 4, causal, _lens(lens))
    for b, n in enumerate(lens):
        assert bool((dk[b, n:] == 0).all())
        if n == 0:
            assert bool((o[b] == 0).all())


@pytest.mark.parametrize("B,Lq,Lk,H,Hk,D,left", [(2, 1, 8192, 32, 8, 128, 511), (1, 1, 8192, 8, 2, 64, 5000), (1, 7, 3000, 4, 4, 128, 100), (1, 100, 4000, 4, 1, 64, 2000)])
def test_few_queries_of_a_long_cache(B, Lq, Lk, H, Hk, D, left):
    """The keys are shared out among CTAs, of which the first has the sinks."""
    check(*make(B, Lq, Lk, H, Hk, D, seed=left), left, 4)
    check(*make(B, Lq, Lk, H, Hk, D, seed=left), left, 4, lens=_lens([Lk - left - 200] * B))


@pytest.mark.parametrize("B,L,H,Hk,D,left,sinks", [(1, 2900, 2, 1, 64, 10, 4), (1, 2000, 4, 2, 128, 300, 128), (2, 1500, 2, 2, 80, 0, 1)])
def test_long_sequences_whose_sinks_are_shared_out(B, L, H, Hk, D, left, sinks):
    check(*make(B, L, L, H, Hk, D, seed=L), left, sinks)


def test_without_a_window_and_without_sinks():
    q, k, v, do = make(1, 400, 400, 4, 2, 64)
    same = lambda a, b: all(torch.equal(x, y) for x, y in zip(a, b))
    assert same(_call(q, k, v, do, causal=True, sinks=4), _call(q, k, v, do, causal=True))
    assert same(_call(q, k, v, do, causal=True, window_left=399, sinks=4), _call(q, k, v, do, causal=True))
    assert same(_call(q, k, v, do, causal=True, window_left=50, sinks=0), _call(q, k, v, do, causal=True, window_left=50))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Lq,Lk,left,sinks", [(1, 700, 100, 4), (3, 1000, 300, 128), (130, 900, 65, 1), (128, 4097, 500, 16), (300, 1000, 17, 60)])
def test_garbage_between_the_sinks_and_every_window(Lq, Lk, left, sinks, D):
    q, k, v, do = make(2, Lq, Lk, 4, 2, D, seed=Lk)
    first = Lk - Lq - left
    assert first > sinks
    for kl in (None, _lens([Lk, Lk - 5]), _lens([Lk, 2])):
        kw = dict(causal=True, window_left=left, k_lens=kl, sinks=sinks)
        want = _call(q, k, v, do, **kw)
        assert bool((want[3][:, sinks:first] == 0).all()) and bool((want[4][:, sinks:first] == 0).all())
        k2, v2 = k.clone(), v.clone()
        k2[:, sinks:first], v2[:, sinks:first] = float("nan"), float("inf")
        v2[:, sinks:first:3] = float("nan")
        if kl is not None:
            for b, n in enumerate(kl.tolist()):
                k2[b, n:], v2[b, n:] = float("nan"), float("nan")
        for a, b in zip(want, _call(q, k2, v2, do, **kw)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("Lq,Lk,H,Hk,D,left,sinks", [(200, 200, 4, 2, 128, 40, 4), (150, 300, 2, 1, 64, 20, 30), (1, 260, 8, 2, 128, 60, 2)])
def test_gradients_against_differences_along_them(Lq, Lk, H, Hk, D, left, sinks):
    q, k, v, do = make(1, Lq, Lk, H, Hk, D, seed=Lq + Lk)
    o, lse, *grads = _call(q, k, v, do, causal=True, window_left=left, sinks=sinks)
    with ref.sinks_in(sinks, edges):
        for want, tol, got, *others in edges.along_the_gradient(q, k, v, do, o, lse, grads, True, left, None):
            assert tol < 0.5 * want
            assert abs(got - want) <= tol
            assert all(abs(x - want) > tol for x in others)


def test_graphs_streams_and_views():
    B, L, H, Hk, D = 2, 700, 4, 2, 64
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    qkv = torch.randn(B, L, H + 2 * Hk, D, generator=g, device=DEV).to(torch.bfloat16)
    do = torch.randn(B, L, H, D, generator=g, device=DEV).to(torch.bfloat16)
    q, k, v = qkv.split((H, Hk, Hk), 2)
    kw = dict(causal=True, window_left=90, sinks=4)
    want = _call(q, k, v, do, **kw)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = _call(q, k, v, do, **kw)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _call(q, k, v, do, **kw)
    qkv.mul_(0.5)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(_call(q, k, v, do, **kw), got))
