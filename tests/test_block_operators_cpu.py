"""Host-side rules of the operators between the linears: workspace sizes and the splits behind them (no GPU)."""
import ctypes as C

import pytest

import paper_2609_02846_b200.binding as B
from paper_2609_02846_b200.build import build_library


@pytest.fixture(scope="module")
def lib():
    build_library()
    return B._load()


def _shape(batch, q_len, k_len, heads, kv_heads, dim, left=-1, scale=0.1, dtype=B.BF16, causal=0):
    return B._AttentionShape(batch, q_len, k_len, heads, kv_heads, dim, left, None, scale, dtype, causal)


def test_layer_norm_workspace(lib):
    f = lib.ue5m3_layer_norm_backward_workspace_bytes
    assert f(1, 100) == 2 * 100 * 4 and f(148, 64) == f(10 ** 6, 64) == 148 * 2 * 64 * 4
    assert f(0, 64) > 0 and f(-1, 64) == 0 and f(5, 0) == 0


def test_attention_workspace_is_asked_for_only_when_keys_are_shared_out(lib):
    f = lib.ue5m3_attention_workspace_bytes
    assert f(_shape(2, 4096, 4096, 32, 8, 128)) == 0                 # enough query tiles
    assert f(_shape(1, 1, 200, 8, 2, 64)) == 0                       # two key tiles: nothing to share out
    # eight tiles, each of the four heads that share keys; 64 key tiles: 18 parts of binary32 o and lse
    assert f(_shape(1, 1, 8192, 32, 8, 128)) == 18 * 32 * (128 + 4) * 4
    assert f(_shape(1, 100, 512, 32, 8, 128)) == 0                   # four key tiles: sharing out costs more than it saves
    assert f(_shape(1, 0, 8192, 32, 8, 128)) == f(_shape(0, 1, 8192, 32, 8, 128)) == f(_shape(1, 1, 0, 32, 8, 128)) == 0


def test_attention_backward_workspace(lib):
    f = lib.ue5m3_attention_backward_workspace_bytes
    rows = lambda batch, heads, q_len: batch * heads * ((q_len + 127) // 128 * 128) * 2 * 4
    assert f(_shape(2, 200, 200, 8, 8, 64)) == rows(2, 8, 200)
    assert f(_shape(1, 1, 8192, 32, 8, 128)) == rows(1, 32, 1) + 4 * 32 * 128 * 4
    assert f(_shape(1, 0, 8192, 32, 8, 128)) == 0


@pytest.mark.parametrize("bad", [dict(dim=60), dict(dim=136), dict(heads=6, kv_heads=4), dict(scale=0.0), dict(scale=float("nan")), dict(left=-2),
                                 dict(dtype=7), dict(causal=2), dict(q_len=-1), dict(kv_heads=0)])
def test_shapes_that_no_call_takes_have_no_workspace(lib, bad):
    args = dict(batch=1, q_len=1, k_len=8192, heads=32, kv_heads=8, dim=128)
    args.update(bad)
    s = _shape(**args)
    assert lib.ue5m3_attention_workspace_bytes(s) == 0 and lib.ue5m3_attention_backward_workspace_bytes(s) == 0


def test_calls_refuse_before_they_look_for_a_device(lib):
    """Argument errors come first, so they are the same with and without a GPU."""
    invalid, shape, align = 1, 2, 3
    p = C.c_void_p(1 << 20)
    assert lib.ue5m3_dropout_add(p, 8, None, 0, B.BF16, 4, 8, 1.5, 0, p, 8, None) == invalid
    assert lib.ue5m3_dropout_add(p, 7, None, 0, B.BF16, 4, 8, 0.5, 0, p, 8, None) == invalid
    assert lib.ue5m3_dropout_add(C.c_void_p((1 << 20) + 1), 8, None, 0, B.BF16, 4, 8, 0.5, 0, p, 8, None) == align
    assert lib.ue5m3_layer_norm(p, B.BF16, 4, 0, 8, p, p, B.F32, 1e-5, p, 8, p, p, None) == invalid
    assert lib.ue5m3_layer_norm(p, B.BF16, 4, 8, 8, C.c_void_p((1 << 20) + 2), p, B.F32, 1e-5, p, 8, p, p, None) == align
    assert lib.ue5m3_layer_norm_backward(p, 8, p, B.F32, 4, 8, 8, p, B.F32, p, p, p, 8, p, p, None, None) == invalid     # sums without a workspace
    t = B._Heads(1 << 20, 1024, 128, 64)
    odd = B._Heads(1 << 20, 1024, 132, 64)
    assert lib.ue5m3_attention(_shape(2, 8, 8, 2, 2, 60), t, t, t, t, p, None, None) == shape
    assert lib.ue5m3_attention(_shape(2, 8, 8, 2, 2, 64), odd, t, t, t, p, None, None) == align
    assert lib.ue5m3_attention(_shape(2, 8, 8, 2, 2, 64), t, t, t, t, None, None, None) == invalid


# ---- outputs that share memory with inputs ------------------------------------------------------
def _elements(t, sizes, dim):
    """The 16-byte units that a tensor [batch, tokens, heads, dim] covers."""
    out = set()
    for b in range(sizes[0]):
        for i in range(sizes[1]):
            for h in range(sizes[2]):
                at = t.data // 16 + (b * t.batch_stride + i * t.token_stride + h * t.head_stride) // 8
                out.update(range(at, at + dim // 8))
    return out


# An lse pointer that is not aligned is refused (3) behind the check of overlaps (1): no call reaches a device.
ODD = C.c_void_p((1 << 20) + 1)


def _forward_status(lib, s, q, k, v, o):
    return lib.ue5m3_attention(s, q, k, v, o, ODD, None, None)


def _backward_status(lib, s, dout, q, k, v, o, dq, dk, dv):
    return lib.ue5m3_attention_backward(s, dout, q, k, v, o, ODD, dq, dk, dv, C.c_void_p(1 << 20), None)


def test_attention_refuses_an_output_over_its_inputs(lib):
    overlap, none = 1, 3
    s = _shape(2, 40, 40, 4, 4, 64)
    at = lambda n: B._Heads((1 << 20) + n * (1 << 16), 40 * 256, 256, 64)
    q, k, v, o = (at(n) for n in range(4))
    assert _forward_status(lib, s, q, k, v, o) == none
    assert _forward_status(lib, s, q, k, v, q) == none                      # o in place of q
    assert _forward_status(lib, s, q, k, v, k) == overlap and _forward_status(lib, s, q, k, v, v) == overlap
    later = B._Heads(q.data + 256 * 2, 40 * 256, 256, 64)                   # q from its second token on
    assert _forward_status(lib, s, q, k, v, later) == overlap
    ins, outs = [at(n) for n in (4, 0, 1, 2, 3)], [at(n) for n in (5, 6, 7)]
    assert _backward_status(lib, s, *ins, *outs) == none
    assert _backward_status(lib, s, *ins, ins[4], *outs[1:]) == none         # dq in place of o
    for i in range(3):
        for other in ins[:4] + [t for j, t in enumerate(outs) if j != i]:
            assert _backward_status(lib, s, *ins, *(other if j == i else t for j, t in enumerate(outs))) == overlap


def test_attention_takes_interleaved_views_and_refuses_what_meets(lib):
    """Random layouts, against the sets of elements: views of one buffer interleave without an element in common, or with one."""
    import random
    rng = random.Random(5)
    seen = {1: 0, 3: 0}
    for _ in range(3000):
        batch, tokens, heads, dim = rng.randint(1, 3), rng.randint(1, 4), rng.randint(1, 3), 8 * rng.randint(1, 3)
        sizes = (batch, tokens, heads)

        def tensor(width):
            order = rng.choice([(2, 1, 0), (1, 2, 0), (2, 0, 1)])           # which dimension is innermost
            strides, step = [8, 8, 8], width
            for i in order:
                strides[i] = step
                step *= sizes[i] + rng.choice([0, 0, 1])
            return B._Heads((1 << 20) + 16 * rng.randint(0, 12), *strides)
        width = dim + 8 * rng.randint(0, 3)
        q, o = tensor(width), tensor(rng.choice([width, dim + 8 * rng.randint(0, 3)]))
        far = B._Heads(1 << 30, *([8 * 64] * 3))
        s = _shape(batch, tokens, tokens, heads, heads, dim)
        same = all(getattr(q, n) == getattr(o, n) for n, size in (("data", 0), ("batch_stride", batch), ("token_stride", tokens), ("head_stride", heads))
                   if n == "data" or size > 1)
        want = 1 if not same and _elements(q, sizes, dim) & _elements(o, sizes, dim) else 3
        assert _forward_status(lib, s, q, far, far, o) == want
        seen[want] += 1
    assert min(seen.values()) > 300
