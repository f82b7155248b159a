"""ue5m3_attention and ue5m3_attention_backward against the formulas in 64 bits: masks, ragged lengths, grouped heads, head
dimensions, strides, empty rows, garbage behind the sequences' ends, streams, refusals and directional differences."""
import math

import pytest
import torch

import paper_2609_02846_b200 as lib
from block_reference import assert_within, attention, attention_backward

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def make(B, Lq, Lk, H, Hk, D, seed=0, sharp=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device=DEV)
    q = (n(B, Lq, H, D) * sharp).to(torch.bfloat16)
    k, v, do = n(B, Lk, Hk, D).to(torch.bfloat16), n(B, Lk, Hk, D).to(torch.bfloat16), n(B, Lq, H, D).to(torch.bfloat16)
    return q, k, v, do


def check(q, k, v, do, causal=False, left=-1, lens=None, scale=None):
    o, lse = lib.attention(q, k, v, causal=causal, window_left=left, k_lens=lens, scale=scale)
    grads = lib.attention_backward(do, q, k, v, o, lse, causal=causal, window_left=left, k_lens=lens, scale=scale)
    torch.cuda.synchronize()
    assert lib.last_device_status() == 0
    wo, wl, bo, bl = attention(q, k, v, causal, left, lens, scale)
    assert_within(o, wo, bo, "o")
    assert_within(lse, wl, bl, "lse")
    for name, got, (want, bound) in zip(("dq", "dk", "dv"), grads, attention_backward(do, q, k, v, o, lse, causal, left, lens, scale)):
        assert_within(got, want, bound, name)
    return o, lse, grads


@pytest.mark.parametrize("D", [8, 40, 64, 80, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_head_dimensions(D, causal):
    check(*make(2, 200, 200, 4, 2, D, seed=D), causal=causal)


@pytest.mark.parametrize("Lq,Lk", [(1, 1), (1, 7), (1, 1000), (2, 129), (127, 127), (128, 128), (129, 255), (256, 256), (257, 385), (640, 130), (5, 3)])
@pytest.mark.parametrize("causal", [False, True])
def test_lengths(Lq, Lk, causal):
    """One token to several tiles, more queries than keys included: with a causal mask the first Lq - Lk queries then see nothing."""
    o, lse, (dq, dk, dv) = check(*make(1, Lq, Lk, 2, 1, 64, seed=Lq * 1000 + Lk), causal=causal)
    if causal and Lq > Lk:
        assert bool((o[:, :Lq - Lk] == 0).all()) and bool((lse[:, :, :Lq - Lk] == -math.inf).all()) and bool((dq[:, :Lq - Lk] == 0).all())


@pytest.mark.parametrize("left", [0, 1, 63, 128, 200, 5000])
@pytest.mark.parametrize("causal", [False, True])
def test_windows(left, causal):
    check(*make(1, 515, 515, 2, 2, 128, seed=left), causal=causal, left=left)
    check(*make(1, 300, 700, 2, 1, 64, seed=left + 1), causal=causal, left=left)


@pytest.mark.parametrize("H,Hk", [(1, 1), (6, 2), (8, 1), (4, 4)])
def test_grouped_heads(H, Hk):
    check(*make(2, 333, 333, H, Hk, 128, seed=H), causal=True)


def test_lengths_of_sequences_and_garbage_behind_them():
    """Whole, partial, one-key and empty sequences; NaN and infinities behind each sequence's end change nothing."""
    B, L = 6, 420
    q, k, v, do = make(B, L, L, 4, 2, 128, seed=5)
    lens = torch.tensor([420, 0, 1, 128, 129, 300], dtype=torch.int32, device=DEV)
    for causal, left in ((False, -1), (True, -1), (True, 50)):
        clean = check(q, k, v, do, causal=causal, left=left, lens=lens)
        k2, v2 = k.clone(), v.clone()
        for b in range(B):
            n = int(lens[b])
            k2[b, n:] = float("nan")
            v2[b, n:] = float("inf")
            v2[b, n + 1::2] = float("nan")
        dirty = check(q, k2, v2, do, causal=causal, left=left, lens=lens)
        for a, b in zip((clean[0], clean[1], *clean[2]), (dirty[0], dirty[1], *dirty[2])):
            assert torch.equal(a, b)
        for g in clean[2][1:]:
            for b in range(B):
                assert bool((g[b, int(lens[b]):] == 0).all())
    # lengths outside 0 .. keys are clamped
    wild = torch.tensor([10 ** 6, -5, 1, 128, 129, 300], dtype=torch.int32, device=DEV)
    for a, b in zip(lib.attention(q, k, v, k_lens=wild), lib.attention(q, k, v, k_lens=lens)):
        assert torch.equal(a, b)


def test_sharp_rows_and_a_maximum_that_keeps_rising():
    """Scores up to hundreds, and keys ordered so that every tile raises the maximum by more than the tolerated factor."""
    check(*make(1, 300, 900, 2, 2, 128, seed=9, sharp=30.0))
    q, k, v, do = make(1, 160, 1024, 1, 1, 64, seed=10)
    ramp = torch.linspace(-6, 6, 1024, device=DEV)[None, :, None, None]
    k = (torch.ones_like(k.float()) * ramp + 0.05 * k.float()).to(torch.bfloat16)
    q = (1.0 + 0.1 * q.float()).abs().to(torch.bfloat16)
    check(q, k, v, do, scale=0.5)
    check(q, -k, v, do, scale=0.5, causal=True)


@pytest.mark.parametrize("scale", [1e-6, 0.03, 2.0])
def test_scales(scale):
    check(*make(1, 130, 260, 2, 2, 64, seed=3), scale=scale)


def test_views_of_a_fused_projection_and_strided_outputs():
    B, L, H, Hk, D = 2, 333, 4, 2, 128
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    qkv = torch.randn(B, L, (H + 2 * Hk) * D + 8, generator=g, device=DEV).to(torch.bfloat16)
    cut = lambda t: (t[:, :, :H * D].unflatten(2, (H, D)), t[:, :, H * D:(H + Hk) * D].unflatten(2, (Hk, D)), t[:, :, (H + Hk) * D:(H + 2 * Hk) * D].unflatten(2, (Hk, D)))
    q, k, v = cut(qkv)
    do = torch.randn(B, H, L, D, generator=g, device=DEV).to(torch.bfloat16).transpose(1, 2)          # heads outside tokens
    o, lse, grads = check(q, k, v, do, causal=True)
    o2 = torch.full((B, H, L, D), 7.0, dtype=torch.bfloat16, device=DEV).transpose(1, 2)
    lib.attention(q, k, v, causal=True, out=o2)
    assert torch.equal(o, o2)
    fused = torch.full_like(qkv, 5.0)
    lib.attention_backward(do, q, k, v, o2, lse, causal=True, out=cut(fused))
    for a, b in zip(grads, cut(fused)):
        assert torch.equal(a, b)
    assert bool((fused[:, :, -8:] == 5.0).all())           # nothing is written between the rows


def test_results_do_not_change_from_call_to_call_or_with_the_batch():
    q, k, v, do = make(3, 700, 700, 4, 2, 128, seed=4)
    a = lib.attention(q, k, v, causal=True)
    ga = lib.attention_backward(do, q, k, v, *a, causal=True)
    for _ in range(3):
        b = lib.attention(q, k, v, causal=True)
        gb = lib.attention_backward(do, q, k, v, *b, causal=True)
        assert all(torch.equal(x, y) for x, y in zip((*a, *ga), (*b, *gb)))
    one = lib.attention(q[1:2], k[1:2], v[1:2], causal=True)
    assert torch.equal(one[0], a[0][1:2]) and torch.equal(one[1], a[1][1:2])


def test_empty_tensors():
    q, k, v, do = make(2, 70, 70, 2, 1, 64)
    o, lse = lib.attention(q, k[:, :0], v[:, :0])
    assert bool((o == 0).all()) and bool((lse == -math.inf).all())
    dq, dk, dv = lib.attention_backward(do, q, k[:, :0], v[:, :0], o, lse)
    assert bool((dq == 0).all()) and dk.numel() == dv.numel() == 0
    o, lse = lib.attention(q[:, :0], k, v)
    assert o.numel() == lse.numel() == 0
    dq, dk, dv = lib.attention_backward(do[:, :0], q[:, :0], k, v, o, lse)
    assert bool((dk == 0).all()) and bool((dv == 0).all())
    assert lib.attention(q[:0], k[:0], v[:0])[0].shape == (0, 70, 2, 64)
    torch.cuda.synchronize()
    assert lib.last_device_status() == 0


def test_gradients_against_differences():
    """<gradient, u> against the central difference of sum(o * do) along u, in 64 bits around the same BF16 inputs."""
    q, k, v, do = make(1, 150, 150, 2, 1, 64, seed=8)
    o, lse = lib.attention(q, k, v, causal=True)
    grads = lib.attention_backward(do, q, k, v, o, lse, causal=True)
    bounds = attention_backward(do, q, k, v, o, lse, True)
    f = lambda a, b, c: (attention(a, b, c, True)[0] * do.double()).sum()
    ins = [t.double() for t in (q, k, v)]
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    for i in range(3):
        u = torch.randn(ins[i].shape, generator=g, device=DEV, dtype=torch.float64)
        e = 1e-4
        at = lambda s: f(*[t + s * e * u if j == i else t for j, t in enumerate(ins)])
        want = (at(1) - at(-1)) / (2 * e)
        got = (grads[i].double() * u).sum()
        # the bound of every element, and what the rounding of the stored o changes in dout . o (2^-8 of it)
        tol = (bounds[i][1] * u.abs()).sum() + 2.0 ** -8 * got.abs() + 1e-4 * want.abs()
        spread = 2.0 ** -8 * (do.double().abs() * o.double().abs()).sum(-1).amax() * (ins[0].abs().amax() + ins[1].abs().amax()) * u.abs().sum() * 64 ** -0.5
        assert abs(float(got - want)) <= float(tol + spread), (i, float(got), float(want))


def test_other_streams_and_graphs():
    q, k, v, do = make(1, 300, 300, 2, 2, 128, seed=6)
    want = lib.attention(q, k, v, causal=True)
    gwant = lib.attention_backward(do, q, k, v, *want, causal=True)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = lib.attention(q, k, v, causal=True)
        ggot = lib.attention_backward(do, q, k, v, *got, causal=True)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((*want, *gwant), (*got, *ggot)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = lib.attention(q, k, v, causal=True)
        ggot = lib.attention_backward(do, q, k, v, *got, causal=True)
    for t in (*got, *ggot):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((*want, *gwant), (*got, *ggot)))


def test_refusals():
    q, k, v, do = make(1, 20, 20, 4, 2, 64)
    o, lse = lib.attention(q, k, v)
    with pytest.raises(TypeError):
        lib.attention(q.half(), k.half(), v.half())
    with pytest.raises(lib.Ue5m3Error, match="UNSUPPORTED"):
        lib.attention(q.float(), k.float(), v.float())
    with pytest.raises(lib.Ue5m3Error, match="UNSUPPORTED"):
        lib.attention(*make(1, 20, 20, 4, 2, 136)[:3])
    with pytest.raises(lib.Ue5m3Error, match="SHAPE"):
        lib.attention(*make(1, 20, 20, 4, 2, 60)[:3])
    with pytest.raises(lib.Ue5m3Error, match="SHAPE"):
        lib.attention(q, *make(1, 20, 20, 4, 3, 64)[1:3])
    for bad in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(lib.Ue5m3Error, match="INVALID_ARG"):
            lib.attention(q, k, v, scale=bad)
    with pytest.raises(lib.Ue5m3Error, match="INVALID_ARG"):
        lib.attention(q, k, v, window_left=-2)
    for bad in (k[:, :19], k[:, :, :1], k.float(), k.cpu()):
        with pytest.raises(ValueError):
            lib.attention(q, k, bad)
    with pytest.raises(ValueError):
        lib.attention(q, k.transpose(2, 3).contiguous().transpose(2, 3), v)                   # last dimension not contiguous
    wide = torch.zeros(1, 20, 4, 68, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(lib.Ue5m3Error, match="ALIGN"):
        lib.attention(wide[..., :64], k, v)                                                   # strides not multiples of 8
    with pytest.raises(lib.Ue5m3Error, match="ALIGN"):
        lib.attention(q[:, :, :1].expand(1, 20, 4, 64), k, v)                                 # a stride of zero
    flat = torch.zeros(20 * 4 * 64 + 8, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(lib.Ue5m3Error, match="ALIGN"):
        lib.attention(flat[4:4 + 20 * 4 * 64].view(1, 20, 4, 64), k, v)                       # base not 16-byte aligned
    with pytest.raises(ValueError):
        lib.attention(q, k, v, k_lens=torch.tensor([20], device=DEV))                         # int64
    with pytest.raises(ValueError):
        lib.attention(q, k, v, k_lens=torch.tensor([20, 20], dtype=torch.int32, device=DEV))
    with pytest.raises(ValueError):
        lib.attention_backward(do, q, k, v, o, lse[:, :, :19])
    with pytest.raises(ValueError):
        lib.attention_backward(do[:, :19], q, k, v, o, lse)
    with pytest.raises(ValueError):
        lib.attention(q.cpu(), k.cpu(), v.cpu())


@pytest.mark.parametrize("Lq,Lk", [(1, 8192), (1, 300), (3, 2000), (130, 4097), (300, 3000)])
@pytest.mark.parametrize("causal", [False, True])
def test_few_queries_for_many_keys(Lq, Lk, causal):
    """The keys are shared out among CTAs and joined: one head and several, empty and short sequences, windows that leave parts
    without a key, any strides of the output."""
    check(*make(1, Lq, Lk, 1, 1, 128, seed=Lk), causal=causal)
    q, k, v, do = make(3, Lq, Lk, 4, 2, 72, seed=Lk + 1)
    lens = torch.tensor([Lk, 0, Lk // 3], dtype=torch.int32, device=DEV)
    o, lse, _ = check(q, k, v, do, causal=causal, lens=lens)
    out = torch.full((3, 4, Lq, 72), 3.0, dtype=torch.bfloat16, device=DEV).transpose(1, 2)
    again = lib.attention(q, k, v, causal=causal, k_lens=lens, out=out)
    assert torch.equal(again[0], o) and torch.equal(again[1], lse)
    check(q, k, v, do, causal=True, left=200)
    v2 = v.clone()
    v2[2, Lk // 3:] = float("nan")
    assert torch.equal(lib.attention(q, k, v2, causal=causal, k_lens=lens)[0], o)


def test_offsets_over_32_bits():
    """Tokens 2^30 elements apart: offsets pass 2^32 elements and bytes in every tensor, read and written."""
    big = torch.zeros((1 << 32) + 8192, dtype=torch.bfloat16, device=DEV)
    far = lambda at: big[at:].as_strided((1, 5, 2, 64), (8, 1 << 30, 64, 1))
    src = make(1, 5, 5, 2, 2, 64, seed=12)
    q, k, v, do = (far(128 * i).copy_(t) for i, t in enumerate(src))
    o, lse = lib.attention(q, k, v, causal=True, out=far(512))
    grads = lib.attention_backward(do, q, k, v, o, lse, causal=True, out=(far(640), far(768), far(896)))
    want = lib.attention(*src[:3], causal=True)
    gwant = lib.attention_backward(src[3], *src[:3], *want, causal=True)
    assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
    for a, b in zip(grads, gwant):
        assert torch.equal(a, b)


def test_one_key_per_query():
    """With a single key the probability is 1: o is v, dv the sum of do over the group, dq and dk vanish."""
    q, k, v, do = make(3, 4, 1, 4, 2, 64, seed=13)
    o, lse = lib.attention(q, k, v)
    assert torch.equal(o, v.repeat_interleave(2, 2).expand(3, 4, 4, 64))
    dq, dk, dv = lib.attention_backward(do, q, k, v, o, lse)
    size = float(do.abs().max() * v.abs().max() * 64) * float(torch.maximum(q.abs().max(), k.abs().max())) * 4
    assert float(dq.abs().max()) <= 2.0 ** -20 * size and float(dk.abs().max()) <= 2.0 ** -20 * size


@pytest.mark.parametrize("B,Lq,Lk,H,Hk,D", [(1, 1, 700, 4, 1, 64), (2, 1, 1500, 32, 8, 128), (16, 1, 300, 20, 10, 128), (3, 33, 400, 12, 2, 80), (1, 40, 900, 4, 1, 128),
                                            (2, 43, 300, 7, 1, 64), (1, 64, 100, 10, 2, 64), (1, 9, 4500, 28, 2, 128), (1, 1, 9000, 200, 1, 64), (2, 65, 513, 6, 2, 128),
                                            (1, 128, 384, 6, 2, 128), (1, 127, 130, 3, 1, 16)])
def test_few_queries_of_grouped_heads(B, Lq, Lk, H, Hk, D):
    """Queries of several heads in one tile: whole, partial and several tiles to a group, on keys that are shared out or not; the
    next group's head behind a partial tile; no mask, causal, a window, lengths."""
    q, k, v, do = make(B, Lq, Lk, H, Hk, D, seed=Lq + H)
    lens = torch.tensor([(Lk * (3 * b + 1)) // (3 * B) for b in range(B)], dtype=torch.int32, device=DEV)
    for causal, left, l in ((False, -1, None), (True, -1, None), (True, 70, None), (True, -1, lens)):
        o, lse, _ = check(q, k, v, do, causal=causal, left=left, lens=l)
        out = torch.full((B, H, Lq, D), 7.0, dtype=torch.bfloat16, device=DEV).transpose(1, 2)
        lib.attention(q, k, v, causal=causal, window_left=left, k_lens=l, out=out)
        assert torch.equal(o, out)
