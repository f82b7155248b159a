"""ue5m3_attention and its backward pass where inputs, memory and launches meet: workspaces that are used again, garbage in rows that take
no part, outputs that overlap inputs, derivatives."""
import pytest
import torch

import paper_2609_02846_b200 as lib
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
