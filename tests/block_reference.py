"""Plain 64-bit forms of the operators between the linears (layer norm, dropout, attention), each with the sums of magnitudes that
the error bounds of its kernel are made of.  Everything is computed from the formulas on whatever device the inputs are on."""
import math

import numpy as np
import torch

D64 = torch.float64


# ---- layer norm ------------------------------------------------------------------------------
def layer_norm(x, w, b, eps):
    """y, mean, rstd and the bound of a binary32 evaluation of y before its rounding."""
    x = x.to(D64)
    n = x.shape[1]
    w = torch.ones(n, dtype=D64, device=x.device) if w is None else w.to(D64)
    b = torch.zeros(n, dtype=D64, device=x.device) if b is None else b.to(D64)
    mean = x.sum(1, keepdim=True) / n
    c = x - mean
    rstd = 1.0 / torch.sqrt((c * c).sum(1, keepdim=True) / n + eps)
    y = c * rstd * w + b
    # the mean is off by a few units of the row's largest magnitude, every later step by a unit of its own result
    size = x.abs().amax(1, keepdim=True)
    bound = 2.0 ** -20 * ((c.abs() + size) * rstd * w.abs() + b.abs())
    return y, mean[:, 0], rstd[:, 0], bound


def layer_norm_backward(dy, x, w, mean, rstd):
    """(dx, dw, db) for the given mean and rstd, and their bounds before the last rounding."""
    dy, x, mean, rstd = dy.to(D64), x.to(D64), mean.to(D64)[:, None], rstd.to(D64)[:, None]
    n = x.shape[1]
    w = torch.ones(n, dtype=D64, device=x.device) if w is None else w.to(D64)
    xh = (x - mean) * rstd
    exh = 2.0 ** -22 * (x.abs() + mean.abs()) * rstd
    g = dy * w
    m = lambda t: t.sum(1, keepdim=True) / n
    dx = rstd * (g - m(g) - xh * m(g * xh))
    mx = m((g * xh).abs())
    bound_dx = rstd * (2.0 ** -19 * (g.abs() + m(g.abs()) + xh.abs() * mx) + exh * mx + xh.abs() * m(g.abs() * exh))
    dw, db = (dy * xh).sum(0), dy.sum(0)
    bound_dw = (dy.abs() * (2.0 ** -18 * xh.abs() + exh)).sum(0)
    return (dx, bound_dx), (dw, bound_dw), (db, 2.0 ** -18 * dy.abs().sum(0))


# ---- dropout ---------------------------------------------------------------------------------
def draws(n, seed):
    """16 random bits of elements 0..n-1 from Philox4x32 with 7 rounds, in Python-sized integers (numpy uint64)."""
    u = np.uint64
    m = u(0xFFFFFFFF)
    g = np.arange((n + 7) // 8, dtype=u)
    c = [g & m, g >> u(32), np.full_like(g, 1), np.zeros_like(g)]
    k = [seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF]
    for r in range(7):
        p0, p1 = u(0xD2511F53) * c[0], u(0xCD9E8D57) * c[2]
        k0, k1 = u((k[0] + r * 0x9E3779B9) & 0xFFFFFFFF), u((k[1] + r * 0xBB67AE85) & 0xFFFFFFFF)
        c = [(p1 >> u(32)) ^ c[1] ^ k0, p1 & m, (p0 >> u(32)) ^ c[3] ^ k1, p0 & m]
    words = np.stack(c, 1)
    return np.stack([words & u(0xFFFF), words >> u(16)], 2).reshape(-1)[:n].astype(np.int64)


def dropout_add(x, p, seed, residual=None):
    """residual + dropout(x) and the mask."""
    t = int(math.floor(p * 65536 + 0.5))
    keep = torch.from_numpy((draws(x.numel(), seed) >= t).reshape(tuple(x.shape))).to(x.device)
    scale = 65536.0 / (65536 - t) if t < 65536 else 0.0
    y = torch.where(keep, x.to(D64) * scale, torch.zeros((), dtype=D64, device=x.device))
    return y if residual is None else y + residual.to(D64), keep


# ---- attention -------------------------------------------------------------------------------
TINY = 2.0 ** -118        # probabilities below the smallest normal binary32 number (times the 2^8 by which they may be scaled) are zero


def allowed(q_len, k_len, causal, left, n_keys, device):
    pos = torch.arange(q_len, device=device)[:, None] + k_len - q_len
    j = torch.arange(k_len, device=device)[None, :]
    ok = (j < n_keys).expand(q_len, k_len).clone()
    if causal:
        ok &= j <= pos
    if left >= 0:
        ok &= j >= pos - left
    return ok


def _clean(t, n):
    """Keys and values behind the sequence's end do not exist, whatever they hold."""
    t = t.to(D64).clone()
    t[n:] = 0
    return t


def attention(q, k, v, causal=False, left=-1, lens=None, scale=None):
    """o, lse and their bounds.  o: the probabilities are rounded to BF16 (2^-8 of each); the rest is binary32, up to o's own
    rounding.  lse: a sum of D products and one exponential sum in binary32."""
    B, Lq, H, D = q.shape
    Lk, Hk = k.shape[1], k.shape[2]
    scale = D ** -0.5 if scale is None else scale
    o = torch.zeros(q.shape, dtype=D64, device=q.device)
    bo = torch.zeros_like(o)
    lse = torch.full((B, H, Lq), -math.inf, dtype=D64, device=q.device)
    bl = torch.zeros_like(lse)
    for b in range(B):
        n = Lk if lens is None else min(max(int(lens[b]), 0), Lk)
        ok = allowed(Lq, Lk, causal, left, n, q.device)
        some = ok.any(1)
        for h in range(H):
            qq, kk, vv = q[b, :, h].to(D64), _clean(k[b, :, h // (H // Hk)], n), _clean(v[b, :, h // (H // Hk)], n)
            s = (qq @ kk.T * scale).masked_fill(~ok, -math.inf)
            z = torch.logsumexp(s[some], 1)
            lse[b, h, some] = z
            size = ((qq.abs() @ kk.abs().T) * scale).masked_fill(~ok, 0.0).amax(1)[some] if Lk else z
            bl[b, h, some] = D * 2.0 ** -24 * size + 2.0 ** -20 * (1 + z.abs())
            P = torch.exp(s[some] - z[:, None])
            o[b, some, h] = P @ vv
            bo[b, some, h] = (2.0 ** -8 + 2.0 ** -12) * (P @ vv.abs()) + TINY * (ok[some].to(D64) @ vv.abs())
    return o, lse, bo, bl


def attention_backward(do, q, k, v, o, lse, causal=False, left=-1, lens=None, scale=None):
    """((dq, bound), (dk, bound), (dv, bound)) for the given o and lse.  P and dS are rounded to BF16 (2^-8 of each); dS carries the binary32 errors of two sums of D products."""
    B, Lq, H, D = q.shape
    Lk, Hk = k.shape[1], k.shape[2]
    g = H // Hk
    scale = D ** -0.5 if scale is None else scale
    out = [torch.zeros(t.shape, dtype=D64, device=q.device) for t in (q, k, v)]
    bound = [torch.zeros_like(t) for t in out]
    r = 2.0 ** -8 + 2.0 ** -11
    for b in range(B):
        n = Lk if lens is None else min(max(int(lens[b]), 0), Lk)
        ok = allowed(Lq, Lk, causal, left, n, q.device)
        some = ok.any(1)
        for h in range(H):
            qq, kk, vv = q[b, :, h].to(D64), _clean(k[b, :, h // g], n), _clean(v[b, :, h // g], n)
            dd, oo = do[b, :, h].to(D64), o[b, :, h].to(D64)
            z = torch.where(some, lse[b, h].to(D64), torch.zeros((), dtype=D64, device=q.device))
            P = torch.exp((qq @ kk.T * scale - z[:, None]).masked_fill(~ok, -math.inf))
            dS = P * (dd @ vv.T - (dd * oo).sum(1, keepdim=True))
            A = 2.0 ** -15 * P * (dd.abs() @ vv.abs().T + (dd * oo).abs().sum(1, keepdim=True))
            E = r * dS.abs() + A + TINY * ok * (dd.abs() @ vv.abs().T + (dd * oo).abs().sum(1, keepdim=True))
            out[0][b, :, h] += scale * dS @ kk
            bound[0][b, :, h] += scale * E @ kk.abs()
            out[1][b, :, h // g] += scale * dS.T @ qq
            bound[1][b, :, h // g] += scale * E.T @ qq.abs()
            out[2][b, :, h // g] += P.T @ dd
            bound[2][b, :, h // g] += (r * P + TINY * ok).T @ dd.abs()
    return tuple(zip(out, bound))


# ---- comparison ------------------------------------------------------------------------------
def assert_within(got, want, bound, what=""):
    """|got - want| <= bound + half a unit in the last place of got's own type (at most 2^-p of the value for p significant bits:
    8 in BF16, 24 in binary32), -inf equal to -inf, nothing else non-finite."""
    want, bound = want.to(got.device), bound.to(got.device)
    g = got.to(D64)
    half = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}[got.dtype]
    same_inf = torch.isinf(want) & (g == want)
    err = torch.where(same_inf, torch.zeros_like(g), (g - want).abs())
    tol = torch.where(same_inf, torch.ones_like(g), bound + half * 1.01 * want.abs() + 1e-37)
    bad = ~(err <= tol)
    if bool(bad.any()):
        i = tuple(int(t) for t in torch.nonzero(bad)[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} values out of bounds, first at {i}: got {g[i]:.6g}, want {want[i]:.6g}, "
                             f"bound {tol[i]:.3g}; worst ratio {float((err / tol)[torch.isfinite(err)].max()) if torch.isfinite(err).any() else float('nan'):.3g}")
