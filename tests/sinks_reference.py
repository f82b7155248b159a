"""The 64-bit forms of attention (block_reference.py) where the first keys stay visible behind the window."""
import contextlib

import torch

import block_reference


@contextlib.contextmanager
def sinks_in(sinks, *modules):
    """`allowed` of block_reference, and of modules that took it from there, with `sinks` first keys that no window hides."""
    plain = block_reference.allowed

    def allowed(q_len, k_len, causal, left, n_keys, device):
        j = torch.arange(k_len, device=device)[None, :]
        return plain(q_len, k_len, causal, left, n_keys, device) | (plain(q_len, k_len, causal, -1, n_keys, device) & (j < sinks))
    for m in (block_reference, *modules):
        m.allowed = allowed
    try:
        yield
    finally:
        for m in (block_reference, *modules):
            m.allowed = plain


def attention(sinks, *args, **kw):
    with sinks_in(sinks):
        return block_reference.attention(*args, **kw)


def attention_backward(sinks, *args, **kw):
    with sinks_in(sinks):
        return block_reference.attention_backward(*args, **kw)
