"""Plain 64-bit forms of rotary positions and of the norm of queries and keys in front of them, each with the bound of a binary32 evaluation
before its last rounding."""
import torch

D64 = torch.float64
# Of a turned value, relative to A (|a| + |b|): the angle's fraction of a turn is rounded to binary32 (2 pi 2^-26), sine and cosine are off by
# a unit in the last place (2^-23), the amplitude, two products and a sum by half a unit each: 3.4 * 2^-23 in all.
TURN = 2.0 ** -21


def _pairs(R, interleaved, device):
    i = torch.arange(R // 2, device=device)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)


def rotate(x, frequencies, positions, interleaved, amplitude, inverse=False):
    """x [B, L, H, D] in 64 bits turned, and the sum of magnitudes A (|a| + |b|) behind every turned value (0 where it stays)."""
    i, j = _pairs(2 * frequencies.numel(), interleaved, x.device)
    t = positions.to(D64)[..., None] * frequencies.to(D64)
    t = (-t if inverse else t)[:, :, None, :]
    c, s = torch.cos(t) * amplitude, torch.sin(t) * amplitude
    y, size = x.clone(), torch.zeros_like(x)
    a, b = x[..., i], x[..., j]
    y[..., i], y[..., j] = a * c - b * s, a * s + b * c
    size[..., i] = size[..., j] = (a.abs() + b.abs()) * abs(amplitude)
    return y, size


def rotary(x, frequencies, positions, interleaved=False, amplitude=1.0, inverse=False):
    y, size = rotate(x.to(D64), frequencies, positions, interleaved, amplitude, inverse)
    return y, TURN * size


# The norm: a sum of up to 256 squares, of which no value passes more than 16 products and 5 sums across lanes (21 roundings, halved by the root), the mean
# (1), the reciprocal root (2 units in the last place, 4 roundings), and two products: 2^-24 (10.5 + 1 + 4 + 2) < 2^-19.
NORM = 2.0 ** -19


def qk_norm_rotary(x, w, frequencies, positions, interleaved, amplitude, eps):
    x = x.to(D64)
    w = torch.ones(x.shape[-1], dtype=D64, device=x.device) if w is None else w.to(D64)
    n = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w
    y, size = rotate(n, frequencies, positions, interleaved, amplitude)
    return y, (TURN + NORM) * size + NORM * y.abs()


def qk_norm_rotary_backward(dy, x, w, frequencies, positions, interleaved, amplitude, eps, chain):
    """((dx, bound), (dw, bound)).  `chain`: most values that one sum of dw adds one after the other."""
    x, dy = x.to(D64), dy.to(D64)
    w = torch.ones(x.shape[-1], dtype=D64, device=x.device) if w is None else w.to(D64)
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    u, size = rotate(dy, frequencies, positions, interleaved, amplitude, inverse=True)
    eu = TURN * size
    xh, g = x * r, u * w
    m = lambda t: t.mean(-1, keepdim=True)
    dx = r * (g - xh * m(g * xh))
    # r enters the last term three times, each 2^-20 at most; the mean of products passes 23 roundings
    bound = r * (eu * w.abs() + 2.0 ** -18 * (g.abs() + xh.abs() * m((g * xh).abs())) + xh.abs() * m(eu * (w * xh).abs()))
    dw = (u * xh).sum((0, 1, 2))
    bound_dw = (eu * xh.abs()).sum((0, 1, 2)) + (2.0 ** -19 + chain * 2.0 ** -24) * (u * xh).abs().sum((0, 1, 2))
    return (dx, bound), (dw, bound_dw)
