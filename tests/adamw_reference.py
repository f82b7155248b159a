"""The AdamW step in numpy: moments and codes with every binary32 rounding of the definition, the weights in 64 bits."""
import numpy as np

F32, F64 = np.float32, np.float64
BLOCK = 256
E4M3, UE5M3 = (448.0, -6, 0x7E), (61440.0, -14, 0xF7)         # largest value, exponent of the smallest normal value, code of the largest


def draws(n, seed, stream, step):
    u, lo = np.uint64, np.uint64(0xFFFFFFFF)
    g = (n + 7) // 8
    c = [np.arange(g, dtype=u)] + [np.full(g, x & 0xFFFFFFFF, dtype=u) for x in (stream, 2, step)]
    k = [seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF]
    for r in range(7):
        p0, p1 = u(0xD2511F53) * c[0], u(0xCD9E8D57) * c[2]
        k0, k1 = u((k[0] + r * 0x9E3779B9) & 0xFFFFFFFF), u((k[1] + r * 0xBB67AE85) & 0xFFFFFFFF)
        c = [(p1 >> u(32)) ^ c[1] ^ k0, p1 & lo, (p0 >> u(32)) ^ c[3] ^ k1, p0 & lo]
    words = np.stack(c, 1)
    return np.stack([words & u(0xFFFF), words >> u(16)], 2).reshape(-1)[:n].astype(np.uint32)


def values(fmt):
    """Value of every code 0..255 (m: sign in bit 7)."""
    _, low, last = fmt
    c = np.arange(256)
    mag = c & 0x7F if last == 0x7E else c
    v = np.where(mag < 8, mag * 2.0 ** (low - 3), (1 + mag % 8 / 8) * 2.0 ** (mag // 8 - 1 + low))
    return np.where((c & 0x80 != 0) & (last == 0x7E), -v, v).astype(F32)


def decode(codes, scale, fmt):
    return values(fmt)[codes] * np.repeat(scale, BLOCK)[:codes.size]


def encode(x, r, fmt):
    """(codes, scales) of a binary32 vector."""
    top, low, last = fmt
    n = x.size
    pad = (-n) % BLOCK
    xb, rb = np.pad(x, (0, pad)).reshape(-1, BLOCK), np.pad(r, (0, pad)).reshape(-1, BLOCK)
    with np.errstate(all="ignore"):
        most = np.abs(xb).max(1, keepdims=True)
        bad = ~(most < np.inf)
        used = (most >= F32(2.0 ** -110)) & ~bad
        inv = F32(1) / np.where(used, most, F32(1))
        t = np.abs(np.where(used, xb, F32(0))) * (inv * F32(top)) * F32(2.0 ** (-126 - low))
        code = np.minimum((t.astype(F32).view(np.uint32) + (rb << np.uint32(4)) + np.uint32(8)) >> np.uint32(20), last)
        if last == 0x7E:
            code = code | np.where(np.signbit(xb), 0x80, 0).astype(np.uint32)
        else:
            code = np.where(xb > 0, np.maximum(code, 1), code)
        scale = np.where(bad, F32(np.nan), np.where(used, most * (F32(1) / F32(top)), F32(0)))
    return np.where(used, code, 0).astype(np.uint8).reshape(-1)[:n], scale.reshape(-1).astype(F32)


def moments(m, v, g, betas, grad_scale=None):
    """m', v' in binary32, every operation rounded."""
    b1, b2 = betas
    g = g.astype(F32)
    with np.errstate(all="ignore"):
        if grad_scale is not None:
            g = g * F32(grad_scale)
        return m * F32(b1) + g * F32(1 - b1), v * F32(b2) + g * F32(1 - b2) * g


def weights(w, m, v, step, lr, betas, eps, decay):
    """w' in 64 bits from the binary32 moments, and the bound of the kernel's: the update's factors are rounded to binary32 (step size and bias, 2^-24
    each), the root is off by 2^-22, the quotient by 2 units in the last place (2^-22), sum and products by 2^-24 each: below 2^-20 of the update; the weight's
    factor and product by 2^-23."""
    m, v, w = m.astype(F64), v.astype(F64), w.astype(F64)
    update = lr / (1 - betas[0] ** step) * m / (np.sqrt(v / (1 - betas[1] ** step)) + eps)
    return w * (1 - lr * decay) - update, 2.0 ** -20 * np.abs(update) + 2.0 ** -23 * np.abs(w) + 1e-38
