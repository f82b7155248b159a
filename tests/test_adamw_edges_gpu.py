"""The AdamW step where its numbers or its shares of the work end."""
import numpy as np
import pytest
import torch

import paper_2609_02846_b200 as lib
from block_reference import assert_within
import adamw_reference as ref
import test_adamw_gpu as small

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F, BF = torch.float32, torch.bfloat16


@pytest.mark.parametrize("bits,eps", [(32, 0.0), (32, 2.0 ** -126), (32, 2.0 ** -70), (8, 2.0 ** -50)])
def test_second_moments_below_the_normal_numbers(bits, eps):
    """Gradients of 0.5e-19 to 2e-19: v = 0.01 g^2 is subnormal, and the first step is lr all the same where eps does not stand above it.  On top of the
    reference's bound the product of v with the bias correction (100) may be subnormal: it is off by 2^-150, the root by half of that relative to
    it.  (m has no place in the rounding: it is an input of the quotient.)"""
    n, lr, betas = 4000, 1e-3, (0.9, 0.99)
    g = torch.Generator(device=DEV)
    g.manual_seed(0)
    grad = 1e-19 * 2 ** (2 * torch.rand(n, generator=g, device=DEV) - 1) * (torch.randint(0, 2, (n,), generator=g, device=DEV) * 2 - 1)
    if eps > 0:
        grad[::7] = 0                                      # m = v = 0: nothing moves
    p = torch.randn(n, generator=g, device=DEV)
    before = p.cpu().numpy()
    if bits == 32:
        m, v, kw = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV), {}
    else:
        m, v = (torch.zeros(n, dtype=torch.uint8, device=DEV) for _ in range(2))
        kw = {k: [torch.zeros(-(-n // 256), device=DEV)] for k in ("m_scale", "v_scale")}
    lib.adamw([p], [grad], [m], [v], 1, lr=lr, betas=betas, eps=eps, weight_decay=0.0, **kw)
    x = grad.cpu().numpy()
    m1, v1 = ref.moments(np.zeros(n, np.float32), np.zeros(n, np.float32), x, betas)
    assert bool((v1[x != 0] > 0).all()) and bool((v1 < 2.0 ** -126).all())
    with np.errstate(all="ignore"):
        want, bound = ref.weights(before, m1, v1, 1, lr, betas, eps, 0.0)
        update = np.abs(before - want)
        bound = bound + np.where(v1 > 0, update * 0.5 * 2.0 ** -150 / (v1.astype(np.float64) * 100), 0)
    assert_within(p, torch.from_numpy(want), torch.from_numpy(bound))
    if eps == 0:
        assert abs(float(np.abs(before - want).mean()) / lr - 1) < 1e-3            # a step of lr, as for any gradient


@pytest.mark.parametrize("pdtype,gdtype,master,offset", [(F, F, False, 0), (BF, BF, True, 0), (BF, F, True, 1), (F, BF, False, 1)])
def test_8_bits_in_shares_of_several_chunks(pdtype, gdtype, master, offset):
    """From 9.7 million elements on a CTA takes four chunks of 512 in a row, of which it loads each under the one before.  Lengths that leave its last
    share one to four chunks, whole ones and ones that end inside a vector, a block and a chunk; addresses that allow vectors and that do not."""
    ends = [1, 2, 3, 4]
    sizes = [(3 * 2048 + 512 * c - d,) for c in ends for d in (0, 3, 256, 300, 511)] + [(1,), (9_700_003,), (2049,), (0,), (511,)]
    assert sum(-(-s[0] // 512) for s in sizes) >= 148 * 16 * 2 * 4          # shares of several chunks
    case = small.Case(sizes, pdtype, gdtype, master, 8, seed=11, offset=offset)
    before = case.numpy()
    case.call(step=3, seed=77)
    small._check(case, before, 3, 77)


def test_8_bits_in_shares_of_several_chunks_beside_small_launches():
    """The rule looks at each launch of 400 tensors: the first takes shares of several chunks, the second does not."""
    case = small.Case([(9_700_003,)] + [((53 * i) % 700 + 1,) for i in range(404)], F, F, False, 8, seed=12)
    before = case.numpy()
    case.call(step=9, seed=1)
    small._check(case, before, 9, 1)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("offset", [0, 1])
def test_a_float32_param_as_its_own_copy(bits, offset):
    a, b = (small.Case([(700,), (2500,)], F, BF, False, bits, seed=13, offset=offset) for _ in range(2))
    a.master = a.p
    a.call(step=5, seed=3)
    b.call(step=5, seed=3)
    assert all(torch.equal(x, y) for x, y in zip(a.p + a.m + a.v, b.p + b.m + b.v))
