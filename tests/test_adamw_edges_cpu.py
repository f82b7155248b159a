"""Refusals of the AdamW step (no GPU)."""
import ctypes as C

import pytest

import paper_2609_02846_b200.binding as B
import paper_2609_02846_b200.optimizer as O
import torch
from paper_2609_02846_b200.build import build_library

INVALID = 1
BASE = 1 << 30


@pytest.fixture(scope="module")
def lib():
    build_library()
    return B._load()


class Tensor(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("param", "grad", "master", "m", "v", "m_scale", "v_scale")] + \
        [("n", C.c_int64), ("stream", C.c_uint32), ("param_dtype", C.c_uint8), ("grad_dtype", C.c_uint8), ("reserved", C.c_uint16)]


def tensor(at, n=1000, gap=1 << 16, **kw):
    """A descriptor whose arrays lie `gap` bytes apart from `at` on, without a master copy."""
    names = ("param", "grad", "m", "v", "m_scale", "v_scale")
    return Tensor(**{**{name: at + i * gap for i, name in enumerate(names)}, "n": n, "param_dtype": B.F32, "grad_dtype": B.F32, **kw})


def call(lib, *tensors, bits=32, eps=1e-8, **kw):
    s = dict(step=1, lr=1e-3, beta1=0.9, beta2=0.99, eps=eps, weight_decay=0.1, grad_scale=None, clock=None, seed=0, state_bits=bits)
    s.update(kw)
    return lib.ue5m3_adamw(C.addressof((Tensor * len(tensors))(*tensors)), len(tensors), B._AdamwStep(*[s[n] for n, _ in B._AdamwStep._fields_]), None)


def passes(status):
    """Behind the checks of arguments there is no device here, and with one nothing of this would be called."""
    return status not in (0, 1, 2, 3, 4)


no_device = pytest.mark.skipif(torch.cuda.is_available(), reason="calls that pass the checks would run")


@no_device
@pytest.mark.parametrize("bits,eps,good", [(32, 0.0, True), (32, 2.0 ** -126, True), (32, 2.0 ** -127, False), (32, 1e-50, False), (32, 5e-324, False),
                                           (8, 2.0 ** -50, True), (8, 2.0 ** -51, False), (8, 1e-30, False), (8, 1e-45, False), (8, 1e-15, True), (8, 1e-8, True)])
def test_an_eps_that_would_not_hold_the_quotient(lib, bits, eps, good):
    status = call(lib, tensor(BASE), bits=bits, eps=eps)
    assert passes(status) if good else status == INVALID
    make = lambda: O.AdamW([torch.nn.Parameter(torch.ones(2))], eps=eps, state_bits=bits)
    if good:
        make()
    else:
        with pytest.raises(ValueError, match="eps"):
            make()
