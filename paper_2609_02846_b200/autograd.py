"""The library's calls as torch.autograd.Functions and modules: the linear layer whose three GEMMs run in UE5M3-FP4, and what
stands between such linears in a transformer block (layer norm, norms and rotary positions of queries and keys, attention, dropout added
to the residual).

Nothing is computed here: forward and backward only call `quantize`, `gemm` and `sample_amax` of the C ABI in
the order the recipe prescribes (X and W rounded to nearest even, the upstream gradient rounded stochastically
once per backward GEMM, one sample-and-hold tensor reference per quantized operand).  With a process group the
freshly sampled maxima are MAX-all-reduced on refresh steps, so that all data-parallel ranks scale by the same
reference; this is the only exchange the path has, one float per operand every `interval` steps.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as B


def reduce_amax_(amax: torch.Tensor, group=None) -> torch.Tensor:
    """In-place MAX all-reduce of a sampled tensor maximum over a process group (no-op without one)."""
    if group is not None and torch.distributed.is_initialized() and torch.distributed.get_world_size(group) > 1:
        torch.distributed.all_reduce(amax, op=torch.distributed.ReduceOp.MAX, group=group)
    return amax


class OperandScale:
    """Sample-and-hold reference of one quantized operand, optionally agreed across ranks on refresh steps."""

    def __init__(self, interval: int = 50, group=None):
        self.cache = B.AmaxCache(interval)
        self.group = group

    def get(self, x: torch.Tensor, step: int) -> torch.Tensor:
        refresh = self.cache.refreshes_at(step)
        held = self.cache.get(x, step)
        if refresh:
            reduce_amax_(held, self.group)
        return held


_layer_counter = 0            # layers built so far in this process: the default stream id of a new layer


def sr_stream_seed(layer_seed: int, rank: int, step: int) -> int:
    """Base seed of one backward pass.  Eq. "sr" wants independent draws: two layers of the same shape, two
    data-parallel ranks and two steps must not share a draw stream (the draw depends only on the seed and the element
    index), otherwise their rounding errors are correlated and do not average out in the gradient all-reduce.
    The three fields sit in disjoint bit ranges (step: 24 bits, rank: 14 bits, layer: 24 bits) of a 62-bit value,
    since `linear_backward` uses 4 * seed and 4 * seed + 1 for its two quantizations."""
    return ((int(layer_seed) & 0xFFFFFF) << 38) | ((int(rank) & 0x3FFF) << 24) | (int(step) & 0xFFFFFF)


def _group_rank(group) -> int:
    if group is not None and torch.distributed.is_initialized():
        return torch.distributed.get_rank(group)
    return 0


def _check_dims(M: int, K: int, N: int, multiple: int = 128) -> None:
    """Every dimension is an output dimension of one GEMM and the contraction of another: multiples of 128 for
    ue5m3_gemm, of 256 under the output model (ue5m3_gemm_probe_matched)."""
    for name, v in (("tokens", M), ("in_features", K), ("out_features", N)):
        if v % multiple:
            raise ValueError(f"{name} = {v}: the three GEMMs of this linear need every dimension to be a multiple of {multiple}")


class _NoSecondDerivative(torch.autograd.Function):
    """A gradient as a value: the library has no derivative of its backward passes, so going through one is an error."""

    @staticmethod
    def forward(ctx, name, grad, *sources):
        ctx.name = name
        return grad.view_as(grad)

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError(f"{ctx.name} has no second derivative")


def _once(name, grads, *sources):
    """`grads` as a backward pass returns them.  Asked for with a graph (create_graph), they hang on the tensors they depend on, so
    that a second derivative is refused in place of being left out of the sum.  (torch's once_differentiable looks at the upstream
    gradient alone, which need not require one.)"""
    sources = [t for t in sources if t is not None and t.requires_grad] if torch.is_grad_enabled() else []
    return tuple(None if g is None else _NoSecondDerivative.apply(name, g, *sources) for g in grads) if sources else tuple(grads)


class _Ue5m3LinearFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, layer, step):
        M, K = x.shape
        N = w.shape[0]
        _check_dims(M, K, N, 128 if layer.grid_denominator is None else 256)
        ax = layer.scale_x.get(x, step)
        aw = layer.scale_w.get(w, step)
        y, _, qw = B.linear_forward(x, w, ax, aw, layer.target_T, x.dtype, grid_denominator=layer.grid_denominator)
        ctx.save_for_backward(x)
        ctx.qw, ctx.ax, ctx.layer, ctx.step = qw, ax, layer, step
        ctx.w = w                               # only to refuse a second derivative: the weight may change after the forward pass
        return y

    @staticmethod
    def backward(ctx, dy):
        (x,) = ctx.saved_tensors
        layer, step, upstream = ctx.layer, ctx.step, dy
        dy = dy.contiguous()
        ag = layer.scale_dy.get(dy, step)
        dx, dw = B.linear_backward(dy, x, ctx.qw, ag, ctx.ax, seed=sr_stream_seed(layer.seed, layer.rank, step), target_T=layer.target_T,
                                   target_T_wgrad_dy=layer.target_T_wgrad_dy, out_dtype=dy.dtype,
                                   grid_denominator=layer.grid_denominator, grad_rounding=layer.grad_rounding)
        return *_once("Ue5m3Linear", (dx, dw), upstream, x, ctx.w), None, None


class Ue5m3Linear(torch.nn.Module):
    """y = x W^T with UE5M3-FP4 operands in all three GEMMs.  `x` is [tokens, in_features] (bfloat16 or float32);
    call `advance()` once per optimizer step so that the held references refresh every `interval` steps.
    `grid_denominator` not None runs the three products under the Section 6.2 output model (0: without its grid
    step); `grad_rounding` is the rounding of the upstream gradient (stochastic by default).  `seed` names the layer's
    stochastic-rounding stream (default: the count of layers built before it); the rank inside `group` and the step are
    mixed in, so layers, ranks and steps draw independently."""

    def __init__(self, in_features: int, out_features: int, device="cuda", dtype=torch.bfloat16, interval: int = 50,
                 target_T: float = 448.0, target_T_wgrad_dy: Optional[float] = None, seed: Optional[int] = None, group=None,
                 grid_denominator: Optional[int] = None, grad_rounding: int = B.ROUND_SR):
        super().__init__()
        self.weight = torch.nn.Parameter(torch.empty(out_features, in_features, device=device, dtype=dtype).normal_(0, 0.02))
        self.target_T = float(target_T)
        self.target_T_wgrad_dy = float(target_T if target_T_wgrad_dy is None else target_T_wgrad_dy)
        global _layer_counter
        self.seed = _layer_counter if seed is None else int(seed)     # default: a stream of its own per layer
        _layer_counter += 1
        self.rank = _group_rank(group)          # mixed into the draws only; the tensor references stay rank-independent
        self.grid_denominator = grid_denominator
        self.grad_rounding = int(grad_rounding)
        self.step = 0
        self.scale_x, self.scale_w, self.scale_dy = (OperandScale(interval, group) for _ in range(3))

    def advance(self) -> None:
        self.step += 1

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        return _Ue5m3LinearFn.apply(x, self.weight, self, self.step)


# ---------------------------------------------------------------------------------------------
# Between the linears
def _as_rows(t: torch.Tensor) -> torch.Tensor:
    """[.., cols] as a matrix with contiguous rows (a copy only where the strides leave no other way, e.g. an expanded gradient)."""
    t = t.reshape(t.shape[:-1].numel(), t.shape[-1])
    ok = (t.stride(1) == 1 or t.shape[1] == 1) and (t.shape[0] <= 1 or t.stride(0) >= t.shape[1])
    return t if ok else t.contiguous()


def _as_heads(t: torch.Tensor) -> torch.Tensor:
    """[batch, tokens, heads, dim] in a form that the attention calls take (a copy only where the strides or the start do not fit)."""
    ok = (t.stride(3) == 1 or t.shape[3] == 1) and t.data_ptr() % 16 == 0 and \
        all(t.shape[i] <= 1 or (t.stride(i) > 0 and t.stride(i) % 8 == 0) for i in range(3))
    return t if ok else t.clone(memory_format=torch.contiguous_format)


class _LayerNormFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        rows = _as_rows(x)
        y, mean, rstd = B.layer_norm(rows, weight, bias, eps)
        ctx.save_for_backward(x, weight, mean, rstd)
        ctx.bias_dtype = None if bias is None else bias.dtype
        return y.view(x.shape)

    @staticmethod
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        want_w, want_b = ctx.needs_input_grad[1], ctx.needs_input_grad[2]
        dx, dw, db = B.layer_norm_backward(_as_rows(dy), _as_rows(x), weight, mean, rstd, want_weight=want_w, want_bias=want_b,
                                           bias_dtype=ctx.bias_dtype)
        return *_once("layer_norm", (dx.view(x.shape), dw, db), dy, x, weight), None


def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5) -> torch.Tensor:
    """Differentiable ue5m3_layer_norm over the last dimension of `x`."""
    return _LayerNormFn.apply(x, weight, bias, eps)


class LayerNorm(torch.nn.Module):
    """Layer norm over the last dimension with learned weight and (by default) bias; the parameters may have another type than the
    activations (float32 parameters with bfloat16 activations by default)."""

    def __init__(self, features: int, eps: float = 1e-5, bias: bool = True, device="cuda", dtype=torch.float32):
        super().__init__()
        self.weight = torch.nn.Parameter(torch.ones(features, device=device, dtype=dtype))
        self.bias = torch.nn.Parameter(torch.zeros(features, device=device, dtype=dtype)) if bias else None
        self.eps = float(eps)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        return layer_norm(x, self.weight, self.bias, self.eps)


class _DropoutAddFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, p, seed):
        ctx.p, ctx.seed, ctx.residual_shape = p, seed, None if residual is None else residual.shape
        y = B.dropout_add(_as_rows(x), p, seed, None if residual is None else _as_rows(residual))
        return y.view(x.shape)

    @staticmethod
    def backward(ctx, dy):
        dx = dropout_add(dy, ctx.p, ctx.seed) if ctx.needs_input_grad[0] else None         # the same linear map, differentiable again
        return dx, dy.reshape(ctx.residual_shape) if ctx.needs_input_grad[1] else None, None, None


def dropout_add(x: torch.Tensor, p: float, seed: int, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Differentiable ue5m3_dropout_add: residual + dropout(x); the mask is drawn again from (seed, index) in the backward pass."""
    return _DropoutAddFn.apply(x, residual, p, seed)


class DropoutAdd(torch.nn.Module):
    """residual + dropout(x) with a draw stream of its own per layer, rank and step.  Call `advance()` once per batch that a gradient is
    taken of: per optimizer step and, where gradients are accumulated, per micro-batch.  In between the same mask is drawn every time, so
    a recomputed forward pass meets the same one; a module that stands twice in a model therefore draws one mask for both places.
    In evaluation mode nothing is dropped."""

    def __init__(self, p: float, seed: Optional[int] = None, group=None):
        super().__init__()
        if not 0.0 <= p <= 1.0:
            raise ValueError(f"p = {p} is no probability")
        global _layer_counter
        self.p = float(p)
        self.seed = _layer_counter if seed is None else int(seed)
        _layer_counter += 1
        self.rank = _group_rank(group)
        self.step = 0

    def advance(self) -> None:
        self.step += 1

    def forward(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
        return dropout_add(x, self.p if self.training else 0.0, sr_stream_seed(self.seed, self.rank, self.step), residual)


class _AttentionFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, causal, window_left, k_lens, scale, sinks):
        o, lse = B.attention(_as_heads(q), _as_heads(k), _as_heads(v), causal, window_left, k_lens, scale, None, sinks)
        ctx.save_for_backward(q, k, v, o, lse, k_lens)
        ctx.args = causal, window_left, scale, sinks
        return o

    @staticmethod
    def backward(ctx, do):
        q, k, v, o, lse, k_lens = ctx.saved_tensors
        causal, window_left, scale, sinks = ctx.args
        grads = B.attention_backward(*(_as_heads(t) for t in (do, q, k, v)), o, lse, causal, window_left, k_lens, scale, None, sinks)
        return *_once("attention", grads, do, q, k, v), None, None, None, None, None


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, causal: bool = False, window_left: int = -1,
              k_lens: Optional[torch.Tensor] = None, scale: Optional[float] = None, sinks: int = 0) -> torch.Tensor:
    """Differentiable ue5m3_attention and ue5m3_attention_sinks: o [batch, tokens, heads, head_dim] (arguments as in the binding's
    `attention`)."""
    return _AttentionFn.apply(q, k, v, causal, window_left, k_lens, scale, sinks)


def _as_turnable(t: Optional[torch.Tensor]) -> Optional[torch.Tensor]:
    """[batch, tokens, heads, dim] in a form that the rotary calls take (a copy only where the strides leave no other way)."""
    if t is None:
        return None
    ok = (t.stride(3) == 1 or t.shape[3] == 1) and all(t.shape[i] <= 1 or t.stride(i) > 0 for i in range(3))
    return t if ok else t.clone(memory_format=torch.contiguous_format)


def _save(ctx, positions, frequencies, *tensors) -> None:
    """Keeps what the backward pass reads again where torch sees whether it was written to meanwhile (positions may be a number or None; tensors of
    inference mode have no version)."""
    two = positions, frequencies
    seen = [torch.is_tensor(t) and not t.is_inference() for t in two]
    ctx.unseen = [None if s else t for s, t in zip(seen, two)]
    ctx.save_for_backward(*(t if s else None for s, t in zip(seen, two)), *tensors)


def _saved(ctx) -> tuple:
    positions, frequencies, *tensors = ctx.saved_tensors
    return (ctx.unseen[0] if positions is None else positions, ctx.unseen[1] if frequencies is None else frequencies, *tensors)


class _RotaryFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, frequencies, positions, interleaved, amplitude, inverse):
        _save(ctx, positions, frequencies)
        ctx.args = interleaved, amplitude, not inverse
        return B.rotary(_as_turnable(q), _as_turnable(k), frequencies, positions, interleaved, amplitude, inverse)

    @staticmethod
    def backward(ctx, dq, dk):
        positions, frequencies = _saved(ctx)
        return *_RotaryFn.apply(dq, dk, frequencies, positions, *ctx.args), None, None, None, None, None         # the transposed linear map, differentiable again


def rotary(q: torch.Tensor, k: Optional[torch.Tensor], frequencies: torch.Tensor, positions=None, interleaved: bool = False,
           amplitude: float = 1.0) -> tuple:
    """Differentiable ue5m3_rotary (arguments as in the binding's `rotary`).  Positions are read again in the backward pass, which refuses
    a tensor of them that was written to meanwhile."""
    return _RotaryFn.apply(q, k, frequencies, positions, interleaved, amplitude, False)


class _QKNormRotaryFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, frequencies, positions, interleaved, amplitude, eps):
        _save(ctx, positions, frequencies, q, k, q_weight, k_weight)
        ctx.args = interleaved, amplitude, eps
        return B.qk_norm_rotary(_as_turnable(q), _as_turnable(k), q_weight, k_weight, frequencies, positions, *ctx.args)

    @staticmethod
    def backward(ctx, dq, dk):
        positions, frequencies, q, k, q_weight, k_weight = _saved(ctx)
        grads = B.qk_norm_rotary_backward(_as_turnable(dq), _as_turnable(dk), _as_turnable(q), _as_turnable(k), q_weight, k_weight, frequencies,
                                          positions, *ctx.args, want_weights=any(ctx.needs_input_grad[2:4]))
        return *_once("qk_norm_rotary", grads, dq, dk, q, k, q_weight, k_weight), None, None, None, None, None


def qk_norm_rotary(q: torch.Tensor, k: Optional[torch.Tensor], q_weight: Optional[torch.Tensor], k_weight: Optional[torch.Tensor],
                   frequencies: torch.Tensor, positions=None, interleaved: bool = False, amplitude: float = 1.0, eps: float = 1e-6) -> tuple:
    """Differentiable ue5m3_qk_norm_rotary (arguments as in the binding's `qk_norm_rotary`; positions as in `rotary`)."""
    return _QKNormRotaryFn.apply(q, k, q_weight, k_weight, frequencies, positions, interleaved, amplitude, eps)


class QKNormRotary(torch.nn.Module):
    """Rotary positions of q and k, with learned norms of every head's row in front of them (`norm`).  `rotary_dim` (default: the whole head)
    and the arguments of `rotary_frequencies` say which pairs turn how fast."""

    def __init__(self, head_dim: int, rotary_dim: Optional[int] = None, norm: bool = True, eps: float = 1e-6, interleaved: bool = False,
                 device="cuda", dtype=torch.float32, **frequencies):
        super().__init__()
        self.q_weight, self.k_weight = (torch.nn.Parameter(torch.ones(head_dim, device=device, dtype=dtype)) if norm else None for _ in range(2))
        self.norm, self.eps, self.interleaved = bool(norm), float(eps), bool(interleaved)
        # not a buffer: a module that is cast to another type must keep its frequencies in 64 bits
        self.frequencies, self.amplitude = B.rotary_frequencies(head_dim if rotary_dim is None else rotary_dim, device=device, **frequencies)

    def forward(self, q: torch.Tensor, k: torch.Tensor, positions=None) -> tuple:
        if self.frequencies.device != q.device:
            self.frequencies = self.frequencies.to(q.device)
        if not self.norm:
            return rotary(q, k, self.frequencies, positions, self.interleaved, self.amplitude)
        return qk_norm_rotary(q, k, self.q_weight, self.k_weight, self.frequencies, positions, self.interleaved, self.amplitude, self.eps)
