"""Timed cases of what a transformer block of FP4 linears needs besides its linears, norms, dropout and plain attention: rotary
positions, norms of queries and keys with the rotation in the same pass, attention with a sliding window and first tokens
that stay visible (sinks), and the AdamW step with states in 32 or in 8 bits.

`run` computes a case in its plain form (elementary torch operations in 32 bits, angles in 64, rounded once at the end) or, with
`own = True`, through the package's entry points.  `exact` is the definition in 64 bits.

The model sizes are those of the package's layer stack: hidden 4096, a QKV projection 4096 -> 6144 (32 query heads and
2 x 8 key/value heads of 128), MLP width 16384, 8192 or 16384 tokens."""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6
BLOCK = 256                      # elements of a tensor that share a scale of an 8-bit state
BETAS, ADAM_EPS, LR, DECAY = (0.9, 0.95), 1e-8, 3e-4, 0.1
STACK = "6144x4096,4096x4096,16384x4096,4096x16384,4096,4096,4096,4096"      # the weights of one block of the stack


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one new token of 16 sequences, each far into its own context: launch latency is all there is
        dict(name="rotary 16 single tokens", op="rotary", batch=16, tokens=1, heads=32, kv_heads=8, dim=128, rot=128, interleaved=False,
             dtype="bf16", positions="each", scaling="parts", inverse=False),
        # the queries and keys of the stack's 16384 tokens, as the fused projection wrote them
        dict(name="rotary 4x4096", op="rotary", batch=4, tokens=4096, heads=32, kv_heads=8, dim=128, rot=128, interleaved=False,
             dtype="bf16", positions="none", scaling="none", inverse=False),
        # the norms of queries and keys of the stack's 8192 tokens
        dict(name="qk norm rotary 2x4096", op="qk_norm_rotary", batch=2, tokens=4096, heads=32, kv_heads=8, dim=128, rot=128, interleaved=False,
             dtype="bf16", wdtype="f32", positions="none", scaling="none"),
        # a small float32 model: neighbouring pairs, a part of an odd-sized head, sequences packed behind one another
        dict(name="qk norm rotary backward 3x517", op="qk_norm_rotary_backward", batch=3, tokens=517, heads=16, kv_heads=4, dim=80, rot=40,
             interleaved=True, dtype="f32", wdtype="f32", positions="packed", scaling="linear"),
        # the gradient of the norms at the stack's 16384 tokens
        dict(name="qk norm rotary backward 4x4096", op="qk_norm_rotary_backward", batch=4, tokens=4096, heads=32, kv_heads=8, dim=128, rot=128,
             interleaved=False, dtype="bf16", wdtype="f32", positions="none", scaling="none"),
        # a prompt of odd length in a small model, window and sinks well inside it
        dict(name="sinks 777 tokens", op="attention", batch=1, lq=777, lk=777, heads=8, kv_heads=2, dim=64, left=200, sinks=4, ragged=False),
        # one micro-batch of the stack with a sliding window
        dict(name="sinks 2x4096", op="attention", batch=2, lq=4096, lk=4096, heads=32, kv_heads=8, dim=128, left=1023, sinks=4, ragged=False),
        # a right-padded batch of short sequences in training
        dict(name="sinks backward 3x500", op="attention_backward", batch=3, lq=500, lk=500, heads=8, kv_heads=8, dim=64, left=127, sinks=2, ragged=True),
        # the backward pass of the micro-batch
        dict(name="sinks backward 2x4096", op="attention_backward", batch=2, lq=4096, lk=4096, heads=32, kv_heads=8, dim=128, left=1023, sinks=4, ragged=False),
        # the step of a small float32 model: eight tensors, most of them vectors
        dict(name="adamw small", op="adamw", shapes="768x256,256x256,1000x256,256x1000,256,256,256,256", param="f32", grad="f32", master=False, bits=32, scaled=False),
        # the step of one block of the stack: bfloat16 weights with a float32 copy, states in 32 bits
        dict(name="adamw block", op="adamw", shapes=STACK, param="bf16", grad="bf16", master=True, bits=32, scaled=True),
        # the same block with states in 8 bits
        dict(name="adamw block 8 bits", op="adamw", shapes=STACK, param="bf16", grad="bf16", master=True, bits=8, scaled=False),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotary", "qk_norm_rotary", "qk_norm_rotary_backward", "attention", "attention_backward", "adamw", "adamw"])
    if op.startswith("attention"):
        most = 2 * 32 * 4096 * 4096                                # scores of the plain form: the largest listed case
        kv = rng.choice([1, 2, 4, 8])
        heads = kv * rng.choice([1, 2, 3, 4])
        dim = rng.choice([64, 128, 128, rng.randrange(2, 17) * 8])
        batch = rng.randint(1, 5)
        lk = _log_uniform(rng, 1, 6000)
        while batch * heads * lk * lk > most:
            lk = max(1, lk * 2 // 3)
        lq = lk if op == "attention_backward" or rng.random() < 0.7 else _log_uniform(rng, 1, max(2, lk))
        return dict(op=op, batch=batch, lq=lq, lk=lk, heads=heads, kv_heads=kv, dim=dim, left=_log_uniform(rng, 1, max(2, lk)),
                    sinks=rng.choice([1, 2, 4, 4, 8, 16, rng.randint(1, 128)]), ragged=rng.random() < 0.3)
    if op == "adamw":
        param = rng.choice(["bf16", "bf16", "f32"])
        count = rng.choice([1, 2, 5, 9, rng.randint(1, 10)])
        room, shapes = 1.6e8, []
        for _ in range(count):
            n = _log_uniform(rng, 1, max(2, int(room * 0.8)))
            room = max(1, room - n)
            cols = rng.choice([1, _log_uniform(rng, 1, 5000), 128])
            shapes.append("%d" % n if cols == 1 or n < cols else "%dx%d" % (n // cols, cols))
        return dict(op=op, shapes=",".join(shapes), param=param, grad=rng.choice([param, "f32"]), master=param == "bf16" and rng.random() < 0.6,
                    bits=rng.choice([8, 32]), scaled=rng.random() < 0.3)
    kv = rng.choice([1, 2, 4, 8])
    heads = kv * rng.choice([1, 2, 3, 4])
    dim = rng.choice([64, 128, 128, rng.randrange(2, 33) * 8])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    batch = rng.randint(1, 8)
    tokens = _log_uniform(rng, 1, 16384)
    while batch * tokens * (heads + kv) * dim * (2 if dtype == "f32" else 1) > 4 * 4096 * 40 * 128:
        tokens = max(1, tokens * 2 // 3)
    c = dict(op=op, batch=batch, tokens=tokens, heads=heads, kv_heads=kv, dim=dim, rot=rng.choice([dim, dim, dim // 4 * 2, 2 * rng.randint(1, dim // 2)]),
             interleaved=rng.random() < 0.4, dtype=dtype, positions=rng.choice(["none", "each", "packed"]), scaling=rng.choice(["none", "linear", "parts"]))
    return {**c, "inverse": rng.random() < 0.5} if op == "rotary" else {**c, "wdtype": rng.choice(["f32", dtype])}


# ------------------------------------------------------------------------------------------------ inputs
def _frequencies(rot, scaling):
    """(radians per position of every pair, in 64 bits; factor on the rotated values).  `linear`: positions shrunk by 8.  `parts`: pairs that
    turn less than once in 4096 positions are shrunk by 8, those that turn 32 times or more stay, a ramp in between."""
    f = 10000.0 ** (-np.arange(rot // 2) * 2.0 / rot)
    if scaling == "linear":
        return f / 8, 1.0
    if scaling == "parts":
        turns = 4096 * f / (2 * math.pi)
        keep = np.clip((turns - 1) / (32 - 1), 0, 1)
        return f * keep + f / 8 * (1 - keep), 0.1 * math.log(8) + 1
    return f, 1.0


def _qkv(c, g, lq, lk):
    """q, k, v: where queries and keys are as many, views of what a fused QKV projection writes (one row per token, heads side by side)."""
    B, H, Hk, D = (c[k] for k in ("batch", "heads", "kv_heads", "dim"))
    dt = DTYPES[c.get("dtype", "bf16")]
    n = lambda *s: torch.randn(*s, generator=g, device=DEV)
    # query rows of different sharpness per head (softmax from nearly flat to nearly one-hot)
    sharp = torch.exp(torch.rand(H, 1, generator=g, device=DEV) * 1.8 - 0.7)
    if lq != lk:
        return (n(B, lq, H, D) * sharp).to(dt), n(B, lk, Hk, D).to(dt), n(B, lk, Hk, D).to(dt)
    qkv = n(B, lq, (H + 2 * Hk) * D)
    qkv[:, :, :H * D].view(B, lq, H, D).mul_(sharp)
    qkv = qkv.to(dt)
    return qkv[:, :, :H * D].view(B, lq, H, D), qkv[:, :, H * D:(H + Hk) * D].view(B, lk, Hk, D), qkv[:, :, (H + Hk) * D:].view(B, lk, Hk, D)


def _shapes(case):
    return [tuple(int(n) for n in s.split("x")) for s in case["shapes"].split(",")]


def _prepare_adamw(s, n, g):
    """Weights in the middle of a run: gradients, and moments that earlier gradients of that size left."""
    s["step"] = 1000
    s["seed"] = int(torch.randint(0, 2 ** 62, (1,), generator=g, device=DEV))
    s["grad_scale"] = torch.full((1,), 0.37, device=DEV) if s["scaled"] else None          # what clipping by the norm multiplies by
    for key in ("p", "g", "m", "v", "m_scale", "v_scale", "master"):
        s[key] = []
    for shape in _shapes(s):
        size = 1e-3 * torch.exp(torch.randn(shape[:1] + (1,) * (len(shape) - 1), generator=g, device=DEV))      # rows of different size
        grad = n(*shape) * size
        p = 0.02 * n(*shape)
        m = 0.3 * n(*shape) * size
        v = size * size * (0.2 + torch.rand(shape, generator=g, device=DEV))
        s["g"].append(grad.to(DTYPES[s["grad"]]))
        s["p"].append(p.to(DTYPES[s["param"]]))
        s["master"].append(p if s["master_kept"] else None)
        if s["bits"] == 32:
            s["m"].append(m)
            s["v"].append(v)
            s["m_scale"].append(None)
            s["v_scale"].append(None)
            continue
        half = torch.full((m.numel(),), 1 << 15, dtype=torch.int32, device=DEV)
        for key, x, fmt in (("m", m, E4M3), ("v", v, UE5M3)):
            code, scale = _encode(x.view(-1), half, *fmt)
            s[key].append(code[:m.numel()].clone().view(shape))
            s[key + "_scale"].append(scale)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = dict(case)
    n = lambda *shape: torch.randn(*shape, generator=g, device=DEV)
    if case["op"] == "adamw":
        s["master_kept"] = case["master"]
        _prepare_adamw(s, n, g)
        return s
    if case["op"].startswith("attention"):
        s["q"], s["k"], s["v"] = _qkv(case, g, case["lq"], case["lk"])
        s["lens"] = None
        if case["ragged"]:
            s["lens"] = torch.randint(0, case["lk"] + 1, (case["batch"],), generator=g, device=DEV, dtype=torch.int32)
            s["lens"][0] = case["lk"]
            if case["batch"] > 2:
                s["lens"][1] = 0
        if case["op"] == "attention_backward":
            s["do"] = (n(*s["q"].shape) * 1e-3).to(torch.bfloat16)
            s["o"], s["lse"] = _plain_attention(s)            # what the forward pass kept
        return s
    B, L, D = case["batch"], case["tokens"], case["dim"]
    s["q"], s["k"], _ = _qkv(case, g, L, L)
    f, s["amplitude"] = _frequencies(case["rot"], case["scaling"])
    s["f"] = torch.from_numpy(f).to(DEV)
    s["pos"] = None
    if case["positions"] != "none":
        # every sequence somewhere in a long context, or rows that several sequences share, each counted from zero
        start = torch.randint(0, 1 << 20, (B, 1), generator=g, device=DEV)
        at = torch.arange(L, device=DEV)
        s["pos"] = start + at if case["positions"] == "each" else at - at // 200 * 200 + 0 * start
    if case["op"] != "rotary":
        s["wq"], s["wk"] = ((1.0 + 0.1 * n(D)).to(DTYPES[case["wdtype"]]) for _ in range(2))
    if case["op"] == "qk_norm_rotary_backward":
        s["dq"], s["dk"] = ((n(*s[k].shape) * 1e-3).to(s[k].dtype) for k in ("q", "k"))
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _cos_sin(s, sign=1.0):
    """[B or 1, L, 1, R / 2] in 32 bits from angles in 64."""
    pos = torch.arange(s["tokens"], device=DEV)[None] if s["pos"] is None else s["pos"]
    angle = (pos.double()[..., None] * s["f"])[:, :, None, :]
    return (torch.cos(angle) * s["amplitude"]).float(), (sign * torch.sin(angle) * s["amplitude"]).float()


def _rotate(x, cs, s):
    """x [B, L, H, D] in 32 bits, its first R columns turned."""
    cos, sin = cs
    R = s["rot"]
    part = x[..., :R]
    a, b = (part[..., 0::2], part[..., 1::2]) if s["interleaved"] else (part[..., :R // 2], part[..., R // 2:])
    c, d = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([c, d], -1).flatten(-2) if s["interleaved"] else torch.cat([c, d], -1)
    return torch.cat([turned, x[..., R:]], -1)


def _plain_rotary(s):
    cs = _cos_sin(s, -1.0 if s["inverse"] else 1.0)
    return tuple(_rotate(s[k].float(), cs, s).to(s[k].dtype) for k in ("q", "k"))


def _plain_qk_norm_rotary(s):
    cs = _cos_sin(s)
    one = lambda x, w: _rotate(x * (x * x).mean(-1, keepdim=True).add(EPS).rsqrt() * w, cs, s)
    return tuple(one(s[k].float(), s[w].float()).to(s[k].dtype) for k, w in (("q", "wq"), ("k", "wk")))


def _plain_qk_norm_rotary_backward(s):
    cs = _cos_sin(s, -1.0)

    def one(x, dy, w):
        r = (x * x).mean(-1, keepdim=True).add(EPS).rsqrt()
        xh = x * r
        back = _rotate(dy, cs, s)
        g = back * w
        return (g - xh * (g * xh).mean(-1, keepdim=True)) * r, (back * xh).sum((0, 1, 2))

    dq, dwq = one(s["q"].float(), s["dq"].float(), s["wq"].float())
    dk, dwk = one(s["k"].float(), s["dk"].float(), s["wk"].float())
    return dq.to(s["q"].dtype), dk.to(s["k"].dtype), dwq.to(s["wq"].dtype), dwk.to(s["wk"].dtype)


def _allowed(s):
    """[B or 1, 1, Lq, Lk]: query i stands at key position i + Lk - Lq and sees no key ahead of it; of the others those that
    are at most `left` back, and the first `sinks` keys; keys from lens[b] on do not exist."""
    Lq, Lk = s["q"].shape[1], s["k"].shape[1]
    pos = torch.arange(Lq, device=DEV)[:, None] + (Lk - Lq)
    j = torch.arange(Lk, device=DEV)[None, :]
    ok = ((j <= pos) & ((j >= pos - s["left"]) | (j < s["sinks"])))[None, None]
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


# 8-bit formats of the moments, by their largest value, smallest exponent of a normal value and largest code; three fraction bits each:
# a sign and E4M3 for the first, unsigned E5M3 (the format of the FP4 block scales) for the second.
E4M3, UE5M3 = (448.0, -6, 0x7E), (61440.0, -14, 0xF7)


def _blocks(x):
    """[n] -> [blocks, 256], the last block filled up with zeros."""
    return torch.nn.functional.pad(x, (0, -x.numel() % BLOCK)).view(-1, BLOCK)


def _encode(x, draws, top, low, last):
    """(codes, scale of every block): magnitudes relative to the block's largest, rounded up with the probability of their place between two
    codes (16 random bits each).  A product with 2^(-126 - low) puts the format's subnormal values on those of binary32, whose bits 20.. are the code then."""
    x = _blocks(x)
    most = x.abs().amax(1, keepdim=True)
    used = most >= 2.0 ** -110
    most = torch.where(used, most, torch.ones_like(most))
    bits = (x.abs() * (top / most) * 2.0 ** (-126 - low)).view(torch.int32)
    code = ((bits + (_blocks(draws) << 4) + 8) >> 20).clamp(max=last)
    code = code | ((x < 0).int() << 7) if last == 0x7E else torch.where(x > 0, code.clamp(min=1), code)
    code = torch.where(used, code, torch.zeros_like(code))
    return code.to(torch.uint8).view(-1), torch.where(used, most / top, torch.zeros_like(most)).view(-1)


def _decode(code, scale, low, signed):
    c = _blocks(code.view(-1).int())
    x = ((c & 0x7F if signed else c) << 20).view(torch.float32) * 2.0 ** (126 + low)
    if signed:
        x = torch.where(c > 0x7F, -x, x)
    return (x * scale[:, None]).view(-1)[:code.numel()]


def _plain_draws(n, seed, stream, step):
    """16 random bits of elements 0..n-1: Philox4x32 with 7 rounds, key = seed, counter = (i >> 3, stream, 2, step); element
    lane j = i & 7 takes half j & 1 of output word j >> 1.  Products wrap modulo 2^64, which keeps all the bits wanted."""
    m = 0xFFFFFFFF
    c0 = torch.arange((n + 7) // 8, device=DEV)
    c1, c2, c3 = torch.full_like(c0, stream), torch.full_like(c0, 2), torch.full_like(c0, step)
    k0, k1 = seed & m, seed >> 32
    for _ in range(7):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & m) ^ c1 ^ k0, p1 & m, ((p0 >> 32) & m) ^ c3 ^ k1, p0 & m
        k0, k1 = (k0 + 0x9E3779B9) & m, (k1 + 0xBB67AE85) & m
    w = torch.stack([c0, c1, c2, c3], 1)
    return torch.stack([w & 0xFFFF, w >> 16], 2).reshape(-1)[:n].int()


def _plain_adamw(s):
    b1, b2 = BETAS
    for i, (p, g) in enumerate(zip(s["p"], s["g"])):
        n = p.numel()
        grad = g.view(-1).float()
        if s["grad_scale"] is not None:
            grad = grad * s["grad_scale"]
        eight = s["bits"] == 8
        m, v = s["m"][i], s["v"][i]
        m0 = _decode(m, s["m_scale"][i], E4M3[1], True) if eight else m.view(-1)
        v0 = _decode(v, s["v_scale"][i], UE5M3[1], False) if eight else v.view(-1)
        m1 = m0 * b1 + grad * (1 - b1)
        v1 = v0 * b2 + grad * (1 - b2) * grad
        if eight:
            r = _plain_draws(n, s["seed"], i, s["step"])
            turned = ((r & 0xFF) << 8) | (r >> 8)              # the same bits, bytes exchanged, for the first moment
            for key, x, draws, fmt in (("m", m1, turned, E4M3), ("v", v1, r, UE5M3)):
                code, scale = _encode(x, draws, *fmt)
                s[key][i].view(-1).copy_(code[:n])
                s[key + "_scale"][i].copy_(scale)
        else:
            m.view(-1).copy_(m1)
            v.view(-1).copy_(v1)
        w = (p if s["master"][i] is None else s["master"][i]).view(-1).float()
        root = (v1 / (1 - b2 ** s["step"])).sqrt()
        w = w * (1 - LR * DECAY) - (LR / (1 - b1 ** s["step"])) * (m1 / (root + ADAM_EPS))
        if s["master"][i] is not None:
            s["master"][i].view(-1).copy_(w)
        p.view(-1).copy_(w)
    return _adamw_outputs(s)


def _adamw_outputs(s):
    """Weights, float32 copies and moments; moments of 8 bits as the values that their codes stand for in units of the blocks' scales
    (a UE5M3 code is the upper byte of a positive float16, one bit down)."""
    if s["bits"] == 32:
        return s["p"], s["master"], s["m"], s["v"]
    seven = torch.full((1,), 7, dtype=torch.int16, device=DEV)
    return s["p"], s["master"], s["m_scale"], s["v_scale"], [m.view(torch.float8_e4m3fn) for m in s["m"]], \
        [torch.bitwise_left_shift(v, seven).view(torch.float16) for v in s["v"]]


PLAIN = {"rotary": _plain_rotary, "qk_norm_rotary": _plain_qk_norm_rotary, "qk_norm_rotary_backward": _plain_qk_norm_rotary_backward,
         "attention": _plain_attention, "attention_backward": _plain_attention_backward, "adamw": _plain_adamw}


# ------------------------------------------------------------------------------------------------ the package's calls
def run(s):
    if not own:
        return PLAIN[s["op"]](s)
    import paper_2609_02846_b200 as lib
    if s["op"] == "rotary":
        return lib.rotary(s["q"], s["k"], s["f"], s["pos"], interleaved=s["interleaved"], amplitude=s["amplitude"], inverse=s["inverse"])
    if s["op"] == "qk_norm_rotary":
        return lib.qk_norm_rotary(s["q"], s["k"], s["wq"], s["wk"], s["f"], s["pos"], interleaved=s["interleaved"], amplitude=s["amplitude"], eps=EPS)
    if s["op"] == "qk_norm_rotary_backward":
        return lib.qk_norm_rotary_backward(s["dq"], s["dk"], s["q"], s["k"], s["wq"], s["wk"], s["f"], s["pos"], interleaved=s["interleaved"],
                                           amplitude=s["amplitude"], eps=EPS)
    if s["op"] == "attention":
        return lib.attention(s["q"], s["k"], s["v"], causal=True, window_left=s["left"], k_lens=s["lens"], sinks=s["sinks"])
    if s["op"] == "attention_backward":
        return lib.attention_backward(s["do"], s["q"], s["k"], s["v"], s["o"], s["lse"], causal=True, window_left=s["left"], k_lens=s["lens"],
                                      sinks=s["sinks"])
    lib.adamw(s["p"], s["g"], s["m"], s["v"], s["step"], lr=LR, betas=BETAS, eps=ADAM_EPS, weight_decay=DECAY, master=s["master"] if s["master_kept"] else None,
              m_scale=s["m_scale"] if s["bits"] == 8 else None, v_scale=s["v_scale"] if s["bits"] == 8 else None, grad_scale=s["grad_scale"], seed=s["seed"])
    return _adamw_outputs(s)


# ------------------------------------------------------------------------------------------------ what a pass needs
def _pairs(c):
    """(query, key) pairs of one head and sequence that the mask leaves (lengths taken as whole)."""
    pos = np.arange(c["lq"], dtype=np.int64) + c["lk"] - c["lq"]
    lo = np.maximum(pos - c["left"], 0)
    return int((np.maximum(pos + 1 - lo, 0) + np.clip(np.minimum(lo, pos + 1), 0, c["sinks"])).sum())


def work(c):
    if c["op"].startswith("attention"):
        q, kv = c["batch"] * c["lq"] * c["heads"] * c["dim"] * 2, c["batch"] * c["lk"] * c["kv_heads"] * c["dim"] * 2
        pairs = _pairs(c) * c["batch"] * c["heads"]
        if c["ragged"] and c["batch"] > 1:
            pairs = pairs * 2 // 3                                     # lengths are uniform, the first is whole
        if c["op"] == "attention":
            return {"bytes": 2 * q + 2 * kv + c["batch"] * c["lq"] * c["heads"] * 4, "flops": 4 * c["dim"] * pairs}
        return {"bytes": 4 * q + 4 * kv + c["batch"] * c["lq"] * c["heads"] * 4, "flops": 10 * c["dim"] * pairs}
    if c["op"] == "adamw":
        n = sum(math.prod(t) for t in _shapes(c))
        p, g = (2 if c[k] == "bf16" else 4 for k in ("param", "grad"))
        weight = p + 8 if c["master"] else 2 * p
        return {"bytes": n * (weight + g + (16 if c["bits"] == 32 else 4 + 16 / BLOCK)), "flops": 15 * n}
    size = 2 if c["dtype"] == "bf16" else 4
    n = c["batch"] * c["tokens"] * (c["heads"] + c["kv_heads"]) * c["dim"]
    pos = 0 if c["positions"] == "none" else 8 * c["batch"] * c["tokens"]
    return {"bytes": (3 if c["op"].endswith("backward") else 2) * n * size + pos, "flops": {"rotary": 3, "qk_norm_rotary": 7}.get(c["op"], 14) * n}


# ------------------------------------------------------------------------------------------------ 64 bits
def _exact_turn(x, s, back):
    """Every pair of columns as a complex number times e^(i angle)."""
    R, d = s["rot"], torch.float64
    at = torch.arange(s["tokens"], device=DEV, dtype=d)[None] if s["pos"] is None else s["pos"].to(d)
    turn = torch.polar(torch.full((), s["amplitude"], dtype=d, device=DEV), (-at if back else at)[:, :, None, None] * s["f"])
    y = x.clone()
    i = torch.arange(R // 2, device=DEV)
    ia, ib = (2 * i, 2 * i + 1) if s["interleaved"] else (i, i + R // 2)
    z = torch.complex(x[..., ia], x[..., ib]) * turn
    y[..., ia], y[..., ib] = z.real, z.imag
    return y


def _exact_code(x, r, top, low, last):
    """The code of every magnitude relative to its block's largest: its place on the ladder of codes plus the draw, rounded down."""
    most = x.abs().amax(1, keepdim=True)
    used = most >= 2.0 ** -110
    z = x.abs() / torch.where(used, most, torch.ones_like(most)) * top
    e = torch.floor(torch.log2(torch.clamp(z, min=2.0 ** low)))
    e = e - (torch.exp2(e) > torch.clamp(z, min=2.0 ** low)).double()
    place = 8 * (e - low) + z / torch.exp2(e - 3)
    code = torch.clamp(torch.floor(place + (r * 16 + 8) / 2.0 ** 20), max=last)
    if last == 0xF7:
        code = torch.where(x > 0, torch.clamp(code, min=1), code)
    up = torch.clamp(torch.floor(code / 8), min=1)                     # exponent field; 8 codes to a binade
    value = torch.exp2(up - 1 + low) * torch.where(code < 8, code / 8, 1 + code / 8 - up)
    return torch.where(used, value * torch.sign(x), torch.zeros_like(x)), torch.where(used, most / top, torch.zeros_like(most)).view(-1)


def _exact_draws(n, seed, stream, step):
    u = np.uint64
    lo, groups = u(0xFFFFFFFF), (n + 7) // 8
    a = [np.arange(groups, dtype=u)] + [np.full(groups, k, dtype=u) for k in (stream, 2, step)]
    for r in range(7):
        key = [u((seed + r * 0x9E3779B9) & 0xFFFFFFFF), u(((seed >> 32) + r * 0xBB67AE85) & 0xFFFFFFFF)]
        left, right = u(0xD2511F53) * a[0], u(0xCD9E8D57) * a[2]
        a = [(right >> u(32)) ^ a[1] ^ key[0], right & lo, (left >> u(32)) ^ a[3] ^ key[1], left & lo]
    return torch.from_numpy(np.stack(a, 1).astype(np.uint32).view(np.uint16).reshape(-1)[:n].astype(np.int32)).to(DEV).double()


def _exact_adamw(s):
    d = torch.float64
    t, (b1, b2) = s["step"], BETAS
    ps, masters, ms, vs, scales = [], [], [], [], ([], [])
    for i in range(len(s["p"])):
        n, shape = s["p"][i].numel(), s["p"][i].shape
        g = s["g"][i].to(d).reshape(-1) * (1.0 if s["grad_scale"] is None else float(s["grad_scale"]))
        old = []
        for key, table in (("m", torch.arange(256, device=DEV, dtype=torch.uint8).view(torch.float8_e4m3fn).to(d)), ("v", None)):
            x = s[key][i].reshape(-1)
            if s["bits"] == 8:
                c = torch.arange(256, device=DEV, dtype=d)
                if table is None:
                    table = torch.where(c < 8, c * 2.0 ** -17, (1 + c % 8 / 8) * torch.exp2(torch.floor(c / 8) - 15))
                x = table[x.long()] * torch.repeat_interleave(s[key + "_scale"][i].to(d), BLOCK)[:n]
            old.append(x.to(d))
        m, v = b1 * old[0] + (1 - b1) * g, b2 * old[1] + (1 - b2) * g * g
        w = (s["p"][i] if s["master"][i] is None else s["master"][i]).to(d).reshape(-1)
        w = w - LR * DECAY * w - LR * (m / (1 - b1 ** t)) / (torch.sqrt(v / (1 - b2 ** t)) + ADAM_EPS)
        ps.append(w.view(shape))
        masters.append(None if s["master"][i] is None else w.view(shape))
        if s["bits"] == 32:
            ms.append(m.view(shape))
            vs.append(v.view(shape))
            continue
        r = _exact_draws(n, s["seed"], i, t)
        for x, draws, fmt, out, k in ((m, r % 256 * 256 + torch.floor(r / 256), E4M3, ms, 0), (v, r, UE5M3, vs, 1)):
            value, scale = _exact_code(_blocks(x), _blocks(draws), *fmt)
            out.append(value.view(-1)[:n].view(shape))
            scales[k].append(scale)
    return (ps, masters, ms, vs) if s["bits"] == 32 else (ps, masters, *scales, ms, vs)


def exact(case, seed):
    s = prepare(case, seed)
    d = torch.float64
    if case["op"] == "adamw":
        return _exact_adamw(s)
    if case["op"] == "rotary":
        return tuple(_exact_turn(s[k].to(d), s, case["inverse"]) for k in ("q", "k"))
    if case["op"].startswith("qk_norm"):
        outs, sums = [], []
        for k, w, up in (("q", "wq", "dq"), ("k", "wk", "dk")):
            x, weight = s[k].to(d), s[w].to(d)
            size = torch.sqrt(torch.einsum("blhd,blhd->blh", x, x) / case["dim"] + EPS)[..., None]
            if case["op"] == "qk_norm_rotary":
                outs.append(_exact_turn(x / size * weight, s, False))
                continue
            back = _exact_turn(s[up].to(d), s, True)
            sums.append(torch.einsum("blhd,blhd->d", back, x / size))
            along = torch.einsum("blhd,blhd->blh", back * weight, x)[..., None]
            outs.append(back * weight / size - x * along / (case["dim"] * size ** 3))
        return tuple(outs + sums)
    B, Lq, H, D = s["q"].shape
    Lk, Hk = s["k"].shape[1:3]
    first = case["op"] == "attention"
    outs = [torch.zeros(t.shape, dtype=d, device=DEV) for t in ([s["q"]] if first else [s["q"], s["k"], s["v"]])]
    lse = torch.full((B, H, Lq), -math.inf, dtype=d, device=DEV)
    for b in range(B):
        n = Lk if s["lens"] is None else int(s["lens"][b])
        back = torch.arange(Lq, device=DEV)[:, None] + Lk - Lq - torch.arange(n, device=DEV)[None, :]      # how far back key j lies
        hide = back > case["left"]
        hide[:, :case["sinks"]] = False
        hide |= back < 0
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
