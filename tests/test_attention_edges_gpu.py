"""ue5m3_attention and its backward pass where inputs, memory and launches meet: workspaces that are used again, garbage in rows that take
no part, outputs that overlap inputs, derivatives."""
import pytest
import torch

import paper_2609_02846_b200 as lib
from block_reference import allowed, attention, attention_backward
from test_attention_gpu import make

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_rows_of_an_earlier_call_are_not_seen():
    """Calls in a row without a synchronisation get the same workspace memory from the allocator: each kernel sees the rows (lse and
    dout . o) that its own call computed, whatever an earlier call left there."""
    sets = []
    for seed, sharp in ((1, 0.2), (2, 8.0), (3, 1.0)):
        q, k, v, do = make(2, 300, 500, 4, 2, 64, seed=seed, sharp=sharp)
        o, lse = lib.attention(q, k, v)
        sets.append((do, q, k, v, o, lse))
    want = []
    for s in sets:
        want.append(lib.attention_backward(*s))
        torch.cuda.synchronize()
    for turn in range(60):
        got = lib.attention_backward(*sets[turn % 3])
        assert all(torch.equal(a, b) for a, b in zip(got, want[turn % 3])), turn


@pytest.mark.parametrize("B,Lq,Lk,H,Hk,D", [(2, 700, 700, 4, 2, 128), (1, 1, 8192, 32, 8, 128), (3, 33, 400, 12, 2, 80), (1, 300, 3000, 2, 2, 64), (40, 65, 513, 6, 2, 128)])
def test_output_in_place_of_the_queries(B, Lq, Lk, H, Hk, D):
    """Whole tiles, keys shared out, heads in one tile (with a partial tile in front of the next group's heads)."""
    q, k, v, do = make(B, Lq, Lk, H, Hk, D, seed=Lq)
    o, lse = lib.attention(q, k, v, causal=True)
    again = q.clone()
    got, got_lse = lib.attention(again, k, v, causal=True, out=again)
    assert got is again and torch.equal(got, o) and torch.equal(got_lse, lse)
    grads = lib.attention_backward(do, q, k, v, o, lse, causal=True)
    over = o.clone()
    for a, b in zip(grads, lib.attention_backward(do, q, k, v, over, lse, causal=True, out=(over, torch.empty_like(k), torch.empty_like(v)))):
        assert torch.equal(a, b)


def test_outputs_over_inputs_are_refused():
    q, k, v, do = make(1, 64, 64, 2, 2, 64)
    o, lse = lib.attention(q, k, v)
    for out in (k, v):
        with pytest.raises(lib.Ue5m3Error, match="INVALID_ARG"):
            lib.attention(q, k, v, out=out)
    fine = [torch.empty_like(t) for t in (q, k, v)]
    for i, out in ((0, q), (0, do), (1, k), (2, v), (1, fine[0]), (2, q)):
        with pytest.raises(lib.Ue5m3Error, match="INVALID_ARG"):
            lib.attention_backward(do, q, k, v, o, lse, out=tuple(out if j == i else t for j, t in enumerate(fine)))


def _call(q, k, v, do, o=None, **kw):
    out, lse = lib.attention(q, k, v, **kw)
    return out, lse, *lib.attention_backward(do, q, k, v, out if o is None else o, lse, **kw)


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Lq,Lk,causal,left,lens", [
    (300, 200, True, -1, None), (700, 130, True, -1, None),                  # the first Lq - Lk queries stand in front of every key
    (515, 515, True, 40, [515, 100, 300]), (400, 400, False, 3, [1, 129, 400]),     # queries whose window begins behind their sequence's end
    (20, 200, True, 10, [200, 130, 175])])
def test_garbage_in_queries_that_see_no_key(Lq, Lk, causal, left, lens, D, value):
    """q and dout of such queries change no output and no gradient, and their own are zero."""
    B = 1 if lens is None else len(lens)
    q, k, v, do = make(B, Lq, Lk, 4, 2, D, seed=Lq + D)
    kl = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    kw = dict(causal=causal, window_left=left, k_lens=kl)
    want = _call(q, k, v, do, **kw)
    at = torch.arange(Lq, device=DEV) + Lk - Lq
    q2, do2 = q.clone(), do.clone()
    some = False
    for b in range(B):
        n = Lk if lens is None else lens[b]
        dead = ((at < 0) if causal else torch.zeros_like(at, dtype=torch.bool)) | ((at - left >= n) if left >= 0 else False)
        some = some or bool(dead.any())
        assert bool((want[2][b, dead] == 0).all())
        q2[b, dead] = value
        do2[b, dead] = -value
    assert some
    for a, b in zip(want, _call(q2, k, v, do2, **kw)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Lq,Lk,left", [(1, 700, 100), (3, 1000, 300), (130, 900, 65), (300, 700, 17), (128, 4097, 500)])
def test_garbage_in_keys_in_front_of_every_window(Lq, Lk, left, D):
    """Keys and values that no query's window reaches, as a cache that is written round holds them."""
    q, k, v, do = make(2, Lq, Lk, 4, 2, D, seed=Lk)
    first = Lk - Lq - left
    assert first > 0
    for kl in (None, torch.tensor([Lk, Lk - 5], dtype=torch.int32, device=DEV)):
        kw = dict(causal=True, window_left=left, k_lens=kl)
        want = _call(q, k, v, do, **kw)
        assert bool((want[3][:, :first] == 0).all()) and bool((want[4][:, :first] == 0).all())
        k2, v2 = k.clone(), v.clone()
        k2[:, :first], v2[:, :first] = float("nan"), float("inf")
        v2[:, :first:3] = float("nan")
        for a, b in zip(want, _call(q, k2, v2, do, **kw)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("Lq,Lk,H,Hk,D,causal,left,lens", [
    (150, 150, 2, 1, 64, True, -1, None), (200, 200, 4, 2, 128, True, 40, None), (130, 300, 2, 2, 72, False, -1, [250]), (1, 260, 8, 2, 128, True, -1, None)])
def test_gradients_against_differences_along_them(Lq, Lk, H, Hk, D, causal, left, lens):
    """Along u = g / |g| for the gradient g that the formulas give in 64 bits, the difference quotient of sum(o * dout) is |g|, and the
    kernel's gradient projected on u lies within the roundings, element by element: P and dS in BF16 (the reference's bound), o in BF16
    inside dout . o, the gradient's own.  They are below half of |g| here, so that zero, the negated gradient and its double all fail."""
    q, k, v, do = make(1, Lq, Lk, H, Hk, D, seed=Lq + Lk)
    kl = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    kw = dict(causal=causal, window_left=left, k_lens=kl)
    o, lse = lib.attention(q, k, v, **kw)
    grads = lib.attention_backward(do, q, k, v, o, lse, **kw)
    for want, tol, got, *others in along_the_gradient(q, k, v, do, o, lse, grads, causal, left, lens):
        assert tol < 0.5 * want
        assert abs(got - want) <= tol
        assert all(abs(x - want) > tol for x in others)


def along_the_gradient(q, k, v, do, o, lse, grads, causal, left, lens):
    """(difference quotient, tolerance, projection of the gradient, projections of wrong ones) for q, k and v."""
    ins = [t.double() for t in (q, k, v)]
    exact_o, exact_lse, off_o, _ = attention(*ins, causal, left, lens)
    formulas = attention_backward(do, *ins, exact_o, exact_lse, causal, left, lens)
    f = lambda *t: float((attention(*t, causal, left, lens)[0] * do.double()).sum())
    # what the rounding of o changes in D = dout . o, and that in dq and dk (dv does not depend on o)
    off_d = (do.double().abs() * (off_o + 2.0 ** -8 * exact_o.abs())).sum(-1)                                # [1, Lq, H]
    group = q.shape[2] // k.shape[2]
    extra = [torch.zeros_like(t) for t in ins]
    n = k.shape[1] if lens is None else lens[0]
    ok = allowed(q.shape[1], k.shape[1], causal, left, n, q.device)
    for h in range(q.shape[2]):
        qq, kk = ins[0][0, :, h], ins[1][0, :, h // group]
        s = (qq @ kk.T * q.shape[3] ** -0.5).masked_fill(~ok, float("-inf"))
        p = torch.softmax(s, 1) * off_d[0, :, h, None] * q.shape[3] ** -0.5
        extra[0][0, :, h] = p @ kk.abs()
        extra[1][0, :, h // group] += p.T @ qq.abs()
    for i in range(3):
        g, bound = formulas[i]
        u, e = g / g.norm(), 1e-3
        at = lambda s: f(*(t + s * e * u if j == i else t for j, t in enumerate(ins)))
        want = (at(1) - at(-1)) / (2 * e)
        tol = float(((bound + extra[i] + 2.0 ** -8 * g.abs()) * u.abs()).sum()) + 1e-4 * want
        got = float((grads[i].double() * u).sum())
        yield want, tol, got, 0.0, -got, 2 * got
