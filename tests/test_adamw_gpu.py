"""The AdamW step over many tensors: moments and codes to the bit, weights within the roundings of their update."""
import numpy as np
import pytest
import torch

import paper_2609_02846_b200 as lib
from block_reference import assert_within
import adamw_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F = torch.bfloat16, torch.float32
ARGS = dict(lr=2e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)
# lengths around the vector, the block and a CTA's share
SIZES = [(1,), (7,), (8,), (9,), (255,), (256,), (257,), (33, 31), (2047,), (2048,), (2049,), (300, 128), (0,), (5000,)]


class Case:
    def __init__(self, sizes, pdtype, gdtype, master, bits, seed=0, offset=0, scale=1e-2):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        n = lambda s: torch.randn(s, generator=g, device=DEV)

        def place(x, dtype):                               # `offset` elements behind an aligned address
            flat = torch.zeros(x.numel() + offset, dtype=dtype, device=DEV)[offset:]
            return flat.copy_(x.reshape(-1)).view(x.shape)
        self.bits = bits
        w = [0.1 * n(s) for s in sizes]
        self.master = [place(x, F) for x in w] if master else None
        self.p = [place(x, pdtype) for x in w]
        self.g = [place(scale * n(s) * torch.exp(2 * n(s)), gdtype) for s in sizes]
        m, v = [scale * n(s) for s in sizes], [scale ** 2 * n(s) ** 2 for s in sizes]
        if bits == 32:
            self.m, self.v, self.ms, self.vs = [place(x, F) for x in m], [place(x, F) for x in v], None, None
        else:
            self.m, self.v, self.ms, self.vs = [], [], [], []
            for x, codes, scales, fmt in [(x, self.m, self.ms, ref.E4M3) for x in m] + [(x, self.v, self.vs, ref.UE5M3) for x in v]:
                flat = x.reshape(-1).cpu().numpy()
                c, s = ref.encode(flat, np.full(flat.size, 1 << 15, np.uint32), fmt)
                codes.append(place(torch.from_numpy(c).to(DEV).view(x.shape), torch.uint8))
                scales.append(torch.from_numpy(s).to(DEV))

    def numpy(self):
        """Everything as it is now, flat; moments as binary32 values."""
        a = lambda ts: None if ts is None else [t.reshape(-1).float().cpu().numpy() for t in ts]
        out = dict(p=a(self.p), g=a(self.g), master=a(self.master))
        if self.bits == 32:
            out.update(m=a(self.m), v=a(self.v))
        else:
            for key, codes, scales, fmt in (("m", self.m, self.ms, ref.E4M3), ("v", self.v, self.vs, ref.UE5M3)):
                out[key] = [ref.decode(c.reshape(-1).cpu().numpy(), s.cpu().numpy(), fmt) for c, s in zip(codes, scales)]
        return out

    def call(self, step=7, **kw):
        lib.adamw(self.p, self.g, self.m, self.v, step, master=self.master, m_scale=self.ms, v_scale=self.vs, **{**ARGS, **kw})


def _check(case, before, step, seed=0, grad_scale=None, streams=None):
    for i, g in enumerate(before["g"]):
        if g.size == 0:
            continue
        m, v = ref.moments(before["m"][i], before["v"][i], g, ARGS["betas"], grad_scale)
        if case.bits == 32:
            assert np.array_equal(case.m[i].reshape(-1).cpu().numpy(), m) and np.array_equal(case.v[i].reshape(-1).cpu().numpy(), v)
        else:
            r = ref.draws(g.size, seed, i if streams is None else streams[i], step)
            turned = ((r & 0xFF) << 8) | (r >> 8)
            for x, bits, codes, scales, fmt in ((m, turned, case.m, case.ms, ref.E4M3), (v, r, case.v, case.vs, ref.UE5M3)):
                c, s = ref.encode(x, bits, fmt)
                assert np.array_equal(scales[i].cpu().numpy(), s), i
                assert np.array_equal(codes[i].reshape(-1).cpu().numpy(), c), i
        w = before["p"][i] if before["master"] is None else before["master"][i]
        want, bound = ref.weights(w, m, v, step, ARGS["lr"], ARGS["betas"], ARGS["eps"], ARGS["weight_decay"])
        want, bound = torch.from_numpy(want).view(case.p[i].shape), torch.from_numpy(bound).view(case.p[i].shape)
        assert_within(case.p[i], want, bound, f"param {i}")
        if case.master is not None:
            assert_within(case.master[i], want, bound, f"master {i}")
            assert torch.equal(case.p[i], case.master[i].to(case.p[i].dtype))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("pdtype,gdtype,master", [(F, F, False), (BF, BF, True), (BF, F, False), (F, BF, False)])
@pytest.mark.parametrize("offset", [0, 1])
def test_a_step(pdtype, gdtype, master, bits, offset):
    case = Case(SIZES, pdtype, gdtype, master, bits, offset=offset)
    before = case.numpy()
    case.call(step=7, seed=2 ** 63 + 12345)
    _check(case, before, 7, 2 ** 63 + 12345)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("count", [1, 40, 41, 400, 405])
def test_many_tensors(count, bits):
    """Both sizes of the launch's parameters, and more tensors than a launch takes."""
    case = Case([((37 * i) % 300 + 1,) for i in range(count)], F, F, False, bits)
    before = case.numpy()
    streams = [i * 7 + 3 for i in range(count)]
    case.call(step=1, seed=5, streams=streams)
    _check(case, before, 1, 5, streams=streams)


@pytest.mark.parametrize("bits", [32, 8])
def test_gradient_scale_and_steps_that_are_left_out(bits):
    case = Case([(700,), (3,)], BF, BF, True, bits)
    before = case.numpy()
    case.call(step=3, grad_scale=torch.tensor([0.25], device=DEV))
    _check(case, before, 3, grad_scale=0.25)
    before = case.numpy()
    for bad in (float("nan"), float("inf")):
        case.call(step=4, grad_scale=torch.tensor([bad], device=DEV))
    after = case.numpy()
    assert all(np.array_equal(a, b) for k in before for a, b in zip(before[k], after[k]))


@pytest.mark.parametrize("scale", [1e-19, 1e-14, 1e-3, 1e15])
def test_moments_of_8_bits_over_the_range_of_gradients(scale):
    """Down to second moments that are not stored any more, up to where squares end."""
    case = Case([(3000,)], F, F, False, 8, scale=scale)
    before = case.numpy()
    case.call(step=2, seed=9)
    _check(case, before, 2, 9)


def test_8_bits_keep_blocks_of_zeros_and_of_what_is_not_finite():
    case = Case([(1024,)], F, F, False, 8)
    for t in (case.m[0], case.v[0], case.ms[0], case.vs[0]):
        t.zero_()
    case.g[0][:256] = 0
    case.g[0][300] = float("nan")
    case.g[0][600] = float("inf")
    p = case.p[0].clone()
    case.call(step=1, weight_decay=0.0)
    assert not case.ms[0][0] and not case.vs[0][0] and torch.equal(case.p[0][:256], p[:256])
    assert bool(case.ms[0][1:3].isnan().all()) and bool(case.vs[0][1:3].isnan().all()) and bool(case.ms[0][3].isfinite())
    gone = case.p[0].isnan()
    assert gone.nonzero().flatten().tolist() == [300, 600]              # in this step the element alone


def test_8_bit_moments_follow_their_gradients_on_average():
    """Constant gradients from zero states: m and v of 32 bits are reached to the noise of the rounding.  A code is off by at most one step, 1/8 of the
    value; the rounding errors of 200 steps with b2 = 0.99 add up with weights 0.99^k: 1/8 / sqrt(1 - 0.99^2) = 0.9 of a value for a single element at
    the very most (uniform errors: half), and over 2^16 elements the mean is off by less than 0.9 / 2^8 * 4."""
    n = 1 << 16
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    grad = torch.exp(0.5 * torch.randn(n, generator=g, device=DEV)) * 1e-3
    p = [torch.zeros(n, device=DEV)]
    m, v = [torch.zeros(n, dtype=torch.uint8, device=DEV)], [torch.zeros(n, dtype=torch.uint8, device=DEV)]
    ms, vs = [torch.zeros(n // 256, device=DEV)], [torch.zeros(n // 256, device=DEV)]
    for t in range(200):
        lib.adamw(p, [grad], m, v, t + 1, lr=1e-3, betas=(0.9, 0.99), m_scale=ms, v_scale=vs, seed=3)
    d = lambda c, s, fmt: torch.from_numpy(ref.decode(c[0].cpu().numpy(), s[0].cpu().numpy(), fmt)).to(DEV).double()
    x = grad.double()
    got_m, got_v = d(m, ms, ref.E4M3) / (x * (1 - 0.9 ** 200)), d(v, vs, ref.UE5M3) / (x * x * (1 - 0.99 ** 200))
    assert abs(float(got_m.mean()) - 1) < 0.014 and abs(float(got_v.mean()) - 1) < 0.014
    assert float((got_m - 1).abs().max()) < 1.0                 # no element has come to a stop far away


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_in_a_graph_go_on_counting(bits):
    a, b = (Case([(700,), (2500,)], BF, BF, True, bits) for _ in range(2))
    clock = torch.zeros(4, dtype=torch.int64, device=DEV)
    a.call(clock=clock, seed=4)                            # outside: step 1
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.call(clock=clock, seed=4)
    for _ in range(3):
        graph.replay()
    for t in range(4):
        b.call(step=t + 1, seed=4)
    assert int(clock[0]) == 4
    for x, y in zip(a.p + a.m + a.v + a.master, b.p + b.m + b.v + b.master):
        assert torch.equal(x, y)
    a.call(clock=clock, grad_scale=torch.tensor([float("nan")], device=DEV))
    assert int(clock[0]) == 4


def test_other_streams():
    a, b = (Case([(700,), (2500,)], F, F, False, 8) for _ in range(2))
    torch.cuda.synchronize()
    a.call(step=2)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        b.call(step=2)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a.p + a.m + a.v, b.p + b.m + b.v))
