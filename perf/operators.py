"""Timed cases of the operators that stand between the FP4 linears of a transformer block: attention with its backward
pass, layer norm with its backward pass, and dropout added to the residual stream.

`run` computes a case in its plain form (elementary torch operations in 32 bits, rounded once at the end) or, with
`own = True`, through the package's entry points.  `exact` is the definition in 64 bits.

The model sizes are those of the package's layer stack: hidden 4096, a QKV projection 4096 -> 6144 (32 query heads and
2 x 8 key/value heads of 128), MLP width 16384, 8192 or 16384 tokens."""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # a short prompt scored on its own: launch latency is all there is
        dict(name="attention 61 tokens", op="attention", batch=1, lq=61, lk=61, heads=8, kv_heads=2, dim=64, causal=True, left=-1, ragged=False),
        # a right-padded batch that attends to a longer, unmasked context (one sequence of the batch is empty)
        dict(name="attention ragged", op="attention", batch=3, lq=517, lk=1031, heads=16, kv_heads=16, dim=80, causal=False, left=-1, ragged=True),
        # one micro-batch of the 8B-shaped stack: 8192 tokens in two sequences
        dict(name="attention 2x4096", op="attention", batch=2, lq=4096, lk=4096, heads=32, kv_heads=8, dim=128, causal=True, left=-1, ragged=False),
        # the backward pass of a small batch of short sequences
        dict(name="attention backward 2x200", op="attention_backward", batch=2, lq=200, lk=200, heads=8, kv_heads=8, dim=64, causal=True, left=-1, ragged=False),
        # a layer with a sliding window, one sequence of odd length, grouped heads
        dict(name="attention backward window", op="attention_backward", batch=1, lq=2501, lk=2501, heads=16, kv_heads=4, dim=128, causal=True, left=511, ragged=False),
        # the backward pass of the same micro-batch of the 8B-shaped stack
        dict(name="attention backward 2x4096", op="attention_backward", batch=2, lq=4096, lk=4096, heads=32, kv_heads=8, dim=128, causal=True, left=-1, ragged=False),
        # the last hidden states of a few sequences before the output head
        dict(name="layer norm 16x4096", op="layer_norm", rows=16, cols=4096, dtype="bf16", wdtype="f32", bias=True),
        # the norm before every linear of the stack
        dict(name="layer norm 8192x4096", op="layer_norm", rows=8192, cols=4096, dtype="bf16", wdtype="bf16", bias=True),
        # a float32 model of odd width
        dict(name="layer norm backward odd", op="layer_norm_backward", rows=1000, cols=1537, dtype="f32", wdtype="f32", bias=True),
        # the gradient of the norm at the stack's 16384 tokens
        dict(name="layer norm backward 16384", op="layer_norm_backward", rows=16384, cols=4096, dtype="bf16", wdtype="f32", bias=True),
        # an odd number of elements, float32, no residual: the backward pass of a small model's dropout
        dict(name="dropout odd", op="dropout_add", rows=777, cols=129, dtype="f32", p=0.2, residual=False),
        # the residual stream after attention or the MLP at the stack's 16384 tokens
        dict(name="dropout add 16384x4096", op="dropout_add", rows=16384, cols=4096, dtype="bf16", p=0.1, residual=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attention", "attention", "attention_backward", "attention_backward", "layer_norm", "layer_norm_backward", "dropout_add"])
    if op.startswith("attention"):
        most = 2 * 32 * 4096 * 4096 * 128 // 2                     # the largest listed case (causal: half of the pairs)
        kv = rng.choice([1, 2, 4, 8])
        heads = kv * rng.choice([1, 2, 3, 4])
        dim = rng.choice([64, 128, 128, rng.randrange(2, 17) * 8])
        batch = rng.randint(1, 5)
        lk = _log_uniform(rng, 1, 8192)
        while batch * heads * lk * lk * dim > most:
            lk = max(1, lk * 2 // 3)
        lq = lk if rng.random() < 0.7 else _log_uniform(rng, 1, max(2, lk))
        causal = rng.random() < 0.7
        left = _log_uniform(rng, 1, max(2, lk)) if causal and rng.random() < 0.25 else -1
        return dict(op=op, batch=batch, lq=lq, lk=lk, heads=heads, kv_heads=kv, dim=dim, causal=causal, left=left, ragged=rng.random() < 0.3)
    rows = _log_uniform(rng, 1, 16384)
    cols = rng.choice([4096, _log_uniform(rng, 16, 4096), 8 * _log_uniform(rng, 2, 512), _log_uniform(rng, 4096, 16384)])
    while rows * cols > 16384 * 4096:
        rows = max(1, rows * 2 // 3)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if dtype == "f32":
        rows = max(1, rows // 2)
    if op == "dropout_add":
        return dict(op=op, rows=rows, cols=cols, dtype=dtype, p=rng.choice([0.05, 0.1, 0.2, 0.5]), residual=rng.random() < 0.7)
    return dict(op=op, rows=rows, cols=cols, dtype=dtype, wdtype=rng.choice(["f32", dtype]), bias=rng.random() < 0.7)


# ------------------------------------------------------------------------------------------------ inputs
def _attention_inputs(c, g):
    B, Lq, Lk, H, Hk, D = (c[k] for k in ("batch", "lq", "lk", "heads", "kv_heads", "dim"))
    n = lambda *s: torch.randn(*s, generator=g, device=DEV)
    # query and key rows of different sharpness per head (softmax from nearly flat to nearly one-hot)
    sharp = torch.exp(torch.rand(H, 1, generator=g, device=DEV) * 1.8 - 0.7)
    if Lq == Lk:
        # what a fused QKV projection writes: one row per token, heads side by side; q, k and v are views of it
        qkv = n(B, Lq, (H + 2 * Hk) * D)
        qkv[:, :, :H * D].view(B, Lq, H, D).mul_(sharp)
        qkv = qkv.to(torch.bfloat16)
        q = qkv[:, :, :H * D].view(B, Lq, H, D)
        k = qkv[:, :, H * D:(H + Hk) * D].view(B, Lk, Hk, D)
        v = qkv[:, :, (H + Hk) * D:].view(B, Lk, Hk, D)
    else:
        q = (n(B, Lq, H, D) * sharp).to(torch.bfloat16)
        k, v = n(B, Lk, Hk, D).to(torch.bfloat16), n(B, Lk, Hk, D).to(torch.bfloat16)
    lens = None
    if c["ragged"]:
        lens = torch.randint(0, Lk + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
        lens[0] = Lk
        if B > 2:
            lens[1] = 0
    return q, k, v, lens


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = dict(case)
    n = lambda *shape: torch.randn(*shape, generator=g, device=DEV)
    if case["op"].startswith("attention"):
        s["q"], s["k"], s["v"], s["lens"] = _attention_inputs(case, g)
        if case["op"] == "attention_backward":
            s["do"] = (n(*s["q"].shape) * 1e-3).to(torch.bfloat16)
            s["o"], s["lse"] = _plain_attention(s)            # what the forward pass kept
        return s
    dt = DTYPES[case["dtype"]]
    rows, cols = case["rows"], case["cols"]
    if case["op"] == "dropout_add":
        s["x"] = n(rows, cols).to(dt)
        s["res"] = (3.0 * n(rows, cols)).to(dt) if case["residual"] else None
        s["seed"] = int(torch.randint(0, 2 ** 62, (1,), generator=g, device=DEV))
        return s
    # a residual stream: channels of different size around a mean
    x = n(rows, cols) * torch.exp(torch.rand(cols, generator=g, device=DEV) * 4.6 - 2.3) + 0.5
    s["x"] = x.to(dt)
    s["w"] = (1.0 + 0.1 * n(cols)).to(DTYPES[case["wdtype"]])
    s["b"] = (0.1 * n(cols)).to(DTYPES[case["wdtype"]]) if case["bias"] else None
    if case["op"] == "layer_norm_backward":
        s["dy"] = (n(rows, cols) * 1e-3).to(dt)
        _, s["mean"], s["rstd"] = _plain_layer_norm(s)        # what the forward pass kept
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _allowed(s):
    """[B or 1, 1, Lq, Lk]: query i stands at key position i + Lk - Lq and sees `left` keys back (-1: all) and, when
    causal, none ahead; keys from lens[b] on do not exist."""
    Lq, Lk = s["q"].shape[1], s["k"].shape[1]
    pos = torch.arange(Lq, device=DEV)[:, None] + (Lk - Lq)
    j = torch.arange(Lk, device=DEV)[None, :]
    ok = torch.ones(Lq, Lk, dtype=torch.bool, device=DEV)
    if s["causal"]:
        ok = ok & (j <= pos)
    if s["left"] >= 0:
        ok = ok & (j >= pos - s["left"])
    ok = ok[None, None]
    if s["lens"] is not None:
        ok = ok & (j[None, None] < s["lens"][:, None, None, None])
    return ok


def _heads_first(t, repeat=1):
    """[B, L, H, D] -> [B, H * repeat, L, D] in 32 bits, each head `repeat` times."""
    return t.float().permute(0, 2, 1, 3).repeat_interleave(repeat, dim=1)


def _plain_attention(s):
    group = s["heads"] // s["kv_heads"]
    q, k, v = _heads_first(s["q"]), _heads_first(s["k"], group), _heads_first(s["v"], group)
    score = (q @ k.transpose(-1, -2)).mul_(1.0 / math.sqrt(s["dim"]))
    score.masked_fill_(~_allowed(s), -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)     # a row that sees nothing
    e = score.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    o = (e @ v) / torch.where(total == 0, torch.ones_like(total), total)
    lse = (top + total.log()).squeeze(-1)
    return o.permute(0, 2, 1, 3).to(s["q"].dtype).contiguous(), lse


def _plain_attention_backward(s):
    group, scale = s["heads"] // s["kv_heads"], 1.0 / math.sqrt(s["dim"])
    q, k, v = _heads_first(s["q"]), _heads_first(s["k"], group), _heads_first(s["v"], group)
    do, o = _heads_first(s["do"]), _heads_first(s["o"])
    score = (q @ k.transpose(-1, -2)).mul_(scale).sub_(s["lse"][..., None])
    p = score.masked_fill_(~_allowed(s), -math.inf).exp_()
    shared = lambda t: t.unflatten(1, (s["kv_heads"], group)).sum(2)    # heads that share a key/value head
    back = lambda t: t.permute(0, 2, 1, 3).to(s["q"].dtype).contiguous()
    dv = shared(p.transpose(-1, -2) @ do)
    ds = (do @ v.transpose(-1, -2)).sub_((do * o).sum(-1, keepdim=True)).mul_(p)
    dq = (ds @ k).mul_(scale)
    dk = shared(ds.transpose(-1, -2) @ q).mul_(scale)
    return back(dq), back(dk), back(dv)


EPS = 1e-5


def _plain_layer_norm(s):
    x = s["x"].float()
    mean = x.mean(-1)
    c = x - mean[:, None]
    rstd = (c * c).mean(-1).add(EPS).rsqrt()
    y = c * rstd[:, None] * s["w"].float()
    if s["b"] is not None:
        y = y + s["b"].float()
    return y.to(s["x"].dtype), mean, rstd


def _plain_layer_norm_backward(s):
    x, dy = s["x"].float(), s["dy"].float()
    xh = (x - s["mean"][:, None]) * s["rstd"][:, None]
    g = dy * s["w"].float()
    dx = (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True)) * s["rstd"][:, None]
    dw = (dy * xh).sum(0).to(s["w"].dtype)
    return dx.to(s["x"].dtype), dw, dy.sum(0).to(s["w"].dtype) if s["b"] is not None else None


def _plain_draws(n, seed):
    """The 16 random bits of elements 0..n-1: Philox4x32 with 7 rounds, key = seed, counter = (i >> 3, 0, 1, 0); element
    lane j = i & 7 takes half j & 1 of output word j >> 1.  Products wrap modulo 2^64, which keeps all the bits wanted."""
    m = 0xFFFFFFFF
    c0 = torch.arange((n + 7) // 8, device=DEV)
    c1, c2, c3 = torch.zeros_like(c0), torch.ones_like(c0), torch.zeros_like(c0)
    k0, k1 = seed & m, seed >> 32
    for _ in range(7):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & m) ^ c1 ^ k0, p1 & m, ((p0 >> 32) & m) ^ c3 ^ k1, p0 & m
        k0, k1 = (k0 + 0x9E3779B9) & m, (k1 + 0xBB67AE85) & m
    w = torch.stack([c0, c1, c2, c3], 1)
    return torch.stack([w & 0xFFFF, w >> 16], 2).reshape(-1)[:n]


def _plain_dropout_add(s):
    x = s["x"].float()
    t = int(math.floor(s["p"] * 65536 + 0.5))                          # of 65536 draws, t drop the element
    keep = (_plain_draws(x.numel(), s["seed"]) >= t).view_as(x)
    y = torch.where(keep, x * (65536.0 / (65536 - t)), torch.zeros_like(x))
    if s["res"] is not None:
        y = y + s["res"].float()
    return y.to(s["x"].dtype)


PLAIN = {"attention": _plain_attention, "attention_backward": _plain_attention_backward, "layer_norm": _plain_layer_norm,
         "layer_norm_backward": _plain_layer_norm_backward, "dropout_add": _plain_dropout_add}


# ------------------------------------------------------------------------------------------------ the package's calls
def run(s):
    if not own:
        return PLAIN[s["op"]](s)
    import paper_2609_02846_b200 as lib
    if s["op"] == "attention":
        return lib.attention(s["q"], s["k"], s["v"], causal=s["causal"], window_left=s["left"], k_lens=s["lens"])
    if s["op"] == "attention_backward":
        return lib.attention_backward(s["do"], s["q"], s["k"], s["v"], s["o"], s["lse"], causal=s["causal"], window_left=s["left"],
                                      k_lens=s["lens"])
    if s["op"] == "layer_norm":
        return lib.layer_norm(s["x"], s["w"], s["b"], EPS)
    if s["op"] == "layer_norm_backward":
        return lib.layer_norm_backward(s["dy"], s["x"], s["w"], s["mean"], s["rstd"], want_bias=s["b"] is not None)
    return lib.dropout_add(s["x"], s["p"], s["seed"], s["res"])


# ------------------------------------------------------------------------------------------------ what a pass needs
def _pairs(c):
    """(query, key) pairs of one head and sequence that the mask leaves (lengths taken as whole)."""
    i = np.arange(c["lq"], dtype=np.int64) + c["lk"] - c["lq"]
    hi = np.minimum(i + 1, c["lk"]) if c["causal"] else np.full_like(i, c["lk"])
    lo = np.maximum(i - c["left"], 0) if c["left"] >= 0 else np.zeros_like(i)
    return int(np.maximum(hi - lo, 0).sum())


def work(c):
    if c["op"].startswith("attention"):
        q, kv = c["batch"] * c["lq"] * c["heads"] * c["dim"] * 2, c["batch"] * c["lk"] * c["kv_heads"] * c["dim"] * 2
        pairs = _pairs(c) * c["batch"] * c["heads"]
        if c["ragged"] and c["batch"] > 1:
            pairs = pairs * 2 // 3                                     # lengths are uniform, the first is whole
        if c["op"] == "attention":
            return {"bytes": 2 * q + 2 * kv + c["batch"] * c["lq"] * c["heads"] * 4, "flops": 4 * c["dim"] * pairs}
        return {"bytes": 4 * q + 4 * kv + c["batch"] * c["lq"] * c["heads"] * 4, "flops": 10 * c["dim"] * pairs}
    size = 2 if c["dtype"] == "bf16" else 4
    n = c["rows"] * c["cols"]
    if c["op"] == "layer_norm":
        return {"bytes": 2 * n * size + 8 * c["rows"] + 8 * c["cols"], "flops": 8 * n}
    if c["op"] == "layer_norm_backward":
        return {"bytes": 3 * n * size + 8 * c["rows"] + 12 * c["cols"], "flops": 14 * n}
    return {"bytes": (3 if c["residual"] else 2) * n * size, "flops": 10 * n}


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    d = torch.float64
    if case["op"].startswith("attention"):
        B, Lq, H, D = s["q"].shape
        Lk, Hk = s["k"].shape[1:3]
        first = case["op"] == "attention"
        outs = [torch.zeros(t.shape, dtype=d, device=DEV) for t in ([s["q"]] if first else [s["q"], s["k"], s["v"]])]
        lse = torch.full((B, H, Lq), -math.inf, dtype=d, device=DEV)
        for b in range(B):
            n = Lk if s["lens"] is None else int(s["lens"][b])
            at = torch.arange(Lq, device=DEV)[:, None] + Lk - Lq - torch.arange(n, device=DEV)[None, :]      # how far back key j lies
            hide = torch.zeros_like(at, dtype=torch.bool)
            if case["causal"]:
                hide |= at < 0
            if case["left"] >= 0:
                hide |= at > case["left"]
            seen = ~hide.all(1)
            for h in range(H):
                kh = h * Hk // H
                q, k, v = s["q"][b, :, h].to(d), s["k"][b, :n, kh].to(d), s["v"][b, :n, kh].to(d)
                t = torch.einsum("id,jd->ij", q, k) / D ** 0.5
                if first:
                    t[hide] = -math.inf
                    total = torch.logsumexp(t, 1)
                    lse[b, h] = total
                    outs[0][b, seen, h] = torch.exp(t[seen] - total[seen, None]) @ v
                    continue
                do, o = s["do"][b, :, h].to(d), s["o"][b, :, h].to(d)
                p = torch.exp(t - torch.where(seen, s["lse"][b, h].to(d), 0)[:, None])
                p[hide] = 0
                ds = p * (torch.einsum("id,jd->ij", do, v) - torch.einsum("id,id->i", do, o)[:, None]) / D ** 0.5
                outs[0][b, :, h] = ds @ k
                outs[1][b, :n, kh] += torch.einsum("ij,id->jd", ds, q)
                outs[2][b, :n, kh] += torch.einsum("ij,id->jd", p, do)
        return (outs[0], lse) if first else tuple(outs)
    x = s["x"].to(d)
    if case["op"] == "layer_norm":
        mean, var = x.mean(1), x.var(1, unbiased=False)
        y = torch.addcmul(torch.zeros((), dtype=d, device=DEV) if s["b"] is None else s["b"].to(d), (x - mean[:, None]) / (var + EPS).sqrt()[:, None], s["w"].to(d))
        return y, mean, 1 / (var + EPS).sqrt()
    if case["op"] == "layer_norm_backward":
        dy, mean, rstd = s["dy"].to(d), s["mean"].to(d), s["rstd"].to(d)
        xh = (x - mean[:, None]) * rstd[:, None]
        dyw = dy * s["w"].to(d)
        dx = rstd[:, None] * (dyw - (dyw.sum(1)[:, None] + xh * (dyw * xh).sum(1)[:, None]) / case["cols"])
        return dx, torch.einsum("rc,rc->c", dy, xh), dy.sum(0) if s["b"] is not None else None
    # dropout: the generator once more, in unsigned numpy words
    n, u = x.numel(), np.uint64
    lo = u(0xFFFFFFFF)
    a = [np.arange((n + 7) // 8, dtype=u), np.zeros((n + 7) // 8, dtype=u), np.ones((n + 7) // 8, dtype=u), np.zeros((n + 7) // 8, dtype=u)]
    for r in range(7):
        key = [u((s["seed"] + r * 0x9E3779B9) & 0xFFFFFFFF), u(((s["seed"] >> 32) + r * 0xBB67AE85) & 0xFFFFFFFF)]
        left, right = u(0xD2511F53) * a[0], u(0xCD9E8D57) * a[2]
        a = [(right >> u(32)) ^ a[1] ^ key[0], right & lo, (left >> u(32)) ^ a[3] ^ key[1], left & lo]
    bits = np.stack(a, 1).astype(np.uint32).view(np.uint16).reshape(-1)[:n]
    t = int(math.floor(case["p"] * 65536 + 0.5))
    keep = torch.from_numpy((bits >= t).reshape(x.shape)).to(DEV)
    y = torch.where(keep, x * 65536 / (65536 - t), torch.zeros_like(x))
    return y + s["res"].to(d) if s["res"] is not None else y
