"""Failure detection of the operators between the linears without a GPU fault: the self-test switches the copies off, so that every
wait for one runs out after about a millisecond.  The kernels return by themselves, report UE5M3_ERR_TIMEOUT once and leave the
context fit for the next, normal call."""
import pytest
import torch

import paper_2609_02846_b200 as lib
import test_layer_norm_gpu as norm
from test_attention_gpu import check, make

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ERR_TIMEOUT = 6
BYTES = 4 << 20


@pytest.mark.parametrize("which", [0, 1, 2, 3, 4])
def test_waits_run_out_and_are_reported_once(which):
    buffer = torch.full((BYTES // 2,), 3.0, dtype=torch.bfloat16, device=DEV)
    torch.cuda.synchronize()
    assert lib.last_device_status() == 0
    start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    lib.block_stall_selftest(which, buffer, wait_limit_cycles=2_000_000)
    stop.record()
    torch.cuda.synchronize()
    assert start.elapsed_time(stop) < 500.0
    assert lib.last_device_status() == ERR_TIMEOUT
    assert lib.last_device_status() == 0
    if which == 0:
        assert bool((buffer[:300 * 2 * 64] == 3.0).all())
    check(*make(1, 300, 300, 2, 1, 64, seed=which))
    check(*make(1, 1, 4096, 4, 1, 64, seed=which))
    norm.check(*norm.make(600, 512, torch.bfloat16, torch.float32, seed=which))


def test_selftest_rejects_bad_arguments():
    buffer = torch.zeros(BYTES, dtype=torch.uint8, device=DEV)
    for which, b, limit in ((-1, buffer, 10 ** 6), (99, buffer, 10 ** 6), (0, buffer[:-1], 10 ** 6), (0, buffer, 10)):
        with pytest.raises(lib.Ue5m3Error, match="INVALID_ARG"):
            lib.block_stall_selftest(which, b, limit)
    with pytest.raises(ValueError):
        lib.block_stall_selftest(0, buffer.cpu())
    torch.cuda.synchronize()
    assert lib.last_device_status() == 0
