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
    array = (Tensor * len(tensors))(*tensors)
    return lib.ue5m3_adamw(C.addressof(array), len(tensors), B._AdamwStep(*[s[n] for n, _ in B._AdamwStep._fields_]), None)


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


NAMES = ("param", "grad", "m", "v", "m_scale", "v_scale")


@no_device
@pytest.mark.parametrize("bits", [32, 8])
def test_memory_that_two_arrays_share(lib, bits):
    """Outputs may have nothing in common with anything else; gradients may be shared among themselves."""
    a, far = BASE, BASE + (1 << 28)
    size = {n: 4000 if bits == 32 else 1000 for n in ("m", "v")} | {n: 4000 for n in ("param", "grad", "master")} | {n: 16 for n in ("m_scale", "v_scale")}
    used = NAMES if bits == 8 else NAMES[:4]
    place = {n: a + i * (1 << 16) for i, n in enumerate(NAMES)}
    assert passes(call(lib, tensor(a), tensor(far), bits=bits))
    for name in used:
        for other in used:                                 # another tensor's array, whole, by its first and by its last bytes
            for at in (place[other], place[other] + size[other] // 4 * 4 - 4, place[other] - size[name] // 4 * 4 + 4):
                if bits == 8 and "m" in (name, other) and at % 4:
                    continue
                status = call(lib, tensor(a), tensor(far, **{name: at}), bits=bits)
                if name == other == "grad":
                    assert passes(status)
                else:
                    assert status == INVALID, (name, other, at - place[other])
            # next to it: nothing in common
            for at in (place[other] + size[other], place[other] - size[name]):
                assert passes(call(lib, tensor(a), tensor(far, **{name: at}), bits=bits)), (name, other)
            if name != other:                              # two arrays of one tensor
                assert call(lib, tensor(far), tensor(a, **{name: place[other]}), bits=bits) == INVALID
    # a float32 param may be its own copy: every thread writes what it has read
    assert passes(call(lib, tensor(a, master=place["param"]), bits=bits)) and call(lib, tensor(a, master=place["param"] + 4), bits=bits) == INVALID
    assert call(lib, tensor(a, master=place["param"], param_dtype=B.BF16), bits=bits) == INVALID
    assert passes(call(lib, tensor(a, master=far), bits=bits))
    # the same tensor twice, wherever it stands; what has no elements has no memory
    many = [tensor(far + i * (1 << 20)) for i in range(500)]
    assert passes(call(lib, *many, bits=bits)) and call(lib, *many, tensor(far + 77 * (1 << 20)), bits=bits) == INVALID
    assert passes(call(lib, tensor(a), tensor(a, n=0), bits=bits))
    # what the step itself reads and writes
    for name in used:
        assert call(lib, tensor(a), bits=bits, clock=place[name]) == INVALID
        assert (call(lib, tensor(a), bits=bits, grad_scale=place[name]) == INVALID) == (name != "grad")
    assert passes(call(lib, tensor(a), bits=bits, clock=far, grad_scale=far + 32)) and call(lib, tensor(a), bits=bits, clock=far, grad_scale=far + 28) == INVALID


@no_device
def test_32_bits_look_at_no_scales(lib):
    """Their addresses may be anything: nothing is read there."""
    assert passes(call(lib, tensor(BASE, m_scale=BASE, v_scale=BASE)))
