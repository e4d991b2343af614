"""What a program asks of the library around a compressed cache, from a prompt's projections to the
tokens generated after it: the cases that these operators are measured on.

`listed()` names the cases, `draw(rng)` gives more of the same ranges.  A case is a plain dict; `op` says
which operator it is:

    rotate    norms of queries and keys for each head and the position rotation, from the projections'
              rows to queries and to rows of the cache (values are copied): Context.rotate
    attend    attention over a cache, causal, with an optional window and first tokens that stay visible;
              m new tokens a sequence, whole prompts (m = n) or single tokens: Context.attend
    pack      the gather of a selection into 4 bits, and the rows that these stand for again:
              Context.compact_mx, Context.expand_mx
    kept      attention of m new tokens over the rows that a selection kept, in the cache's type or in
              4 bits, and over the tokens generated since: Context.attend_kept, Context.attend_kept_mx

and the sizes are

    count     sequences; kv: KV heads; group: query heads per KV head
    m, n      new tokens of a sequence, and its tokens in all (of the longest; ragged: the others are
              shorter, a few have fewer than m tokens)
    window, sinks, norm (weights for the norms given), pairs (neighbours rotate together, else halves)
    keep      rows kept per head (ragged: drawn unevenly over the heads); tail: tokens since (kept)
    dtype     "bf16" or "fp32"; mx: the kept rows are held in 4 bits

Head dimension 128 throughout, as in the configurations of paper_2509_15038_amd/workloads.py.
"""

import math

import numpy as np
import torch

D, EPS = 128, 1e-5
own = False


def _case(op, count=1, kv=8, group=4, m=1, n=1, window=0, sinks=0, dtype="bf16", norm=False, pairs=False, ragged=False, keep=0, tail=0,
          mx=False, name=None):
    c = {"op": op, "count": count, "kv": kv, "group": group, "m": m, "n": n, "window": window, "sinks": sinks, "dtype": dtype,
         "norm": norm, "pairs": pairs, "ragged": ragged, "keep": keep, "tail": tail, "mx": mx}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the projections of one generated token of 4 sequences: latency only
        _case("rotate", count=4, m=1, n=256, ragged=True, norm=True, name="rotate-token"),
        # one layer of a 32k prompt, 8B-shaped, queries and keys normalised
        _case("rotate", count=1, m=32768, n=32768, norm=True, name="rotate-prompt-32k"),
        # one layer of an 8k prompt, causal: what pre-fills the cache that is then compressed
        _case("attend", m=8192, n=8192, name="prompt-8k"),
        # one layer of a 32k prompt with a window of 4096 and four first tokens that stay
        _case("attend", m=32768, n=32768, window=4096, sinks=4, name="prompt-32k-window"),
        # a few odd prompts side by side in fp32, with a window, ragged
        _case("attend", count=3, kv=2, m=1021, n=1021, window=257, sinks=4, dtype="fp32", ragged=True, name="prompts-1021-fp32"),
        # a generated token of 32 sequences of up to 16k tokens through the window
        _case("attend", count=32, m=1, n=16384, window=4096, sinks=4, ragged=True, name="token-window-batch"),
        # a generated token over one whole 128k cache, before any compression
        _case("attend", m=1, n=131072, name="token-128k"),
        # one layer's selection (10 % of 32k tokens, uneven budgets) into 4 bits, as a hook does it layer by layer
        _case("pack", n=32768, keep=3276, ragged=True, name="pack-layer-32k"),
        # the same for the whole model at once: 32 layers of 8 heads
        _case("pack", count=32, n=32768, keep=3276, name="pack-model-32k"),
        # a generated token of one sequence after that, over 4 bits and 200 tokens since
        _case("kept", m=1, keep=3276, tail=200, mx=True, ragged=True, name="kept-token"),
        # a batch of 32 long sequences (10 % of 128k tokens), 4 bits
        _case("kept", count=32, m=1, keep=13107, tail=513, mx=True, ragged=True, name="kept-batch-mx"),
        # four drafted tokens of 8 sequences over rows kept as they were
        _case("kept", count=8, m=4, keep=6553, tail=77, ragged=True, name="kept-drafts-bf16"),
    ]


def _size(rng, low, high):
    """Spread over the logarithm, odd half the time (and no multiple of 1024 but powers of two)."""
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    v = v | 1 if rng.random() < 0.5 else v
    return max(low, min(high, v if v % 1024 or not v & (v - 1) else v + 1))


def draw(rng):
    """One more case: within the listed ones' ranges and costs."""
    op = rng.choice(["rotate", "attend", "attend", "attend", "pack", "kept", "kept"])
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    kv, group = rng.choice([(8, 4), (8, 4), (8, 1), (2, 4), (1, 8), (2, 7), (8, 5), (1, 1)])
    if (group + 2) * kv == 24 or group * kv == 24:                     # (rows as wide as no configuration has them)
        kv, group = 8, 4
    if op == "rotate":
        m = 1 if rng.random() < 0.4 else _size(rng, 2, 32768)
        count = _size(rng, 1, max(1, min(64, 32768 // m)))
        return _case(op, count, kv, group, m, max(m, 256) + rng.choice([0, 1, 130]), dtype=dtype, norm=rng.random() < 0.6,
                     pairs=rng.random() < 0.3, ragged=count > 1 and rng.random() < 0.7)
    if op == "attend":
        window = 0 if rng.random() < 0.4 else _size(rng, 16, 8192)
        sinks = rng.choice([0, 4, 4, 4, 64]) if window else 0
        if rng.random() < 0.5:                                         # a few tokens a sequence
            m, n = rng.choice([1, 1, 1, 2, 5]), _size(rng, 8, 131072)
            most = 2 ** 21 // (kv * (2 if dtype == "fp32" else 1))     # rows in all
            return _case(op, _size(rng, 1, max(1, min(64, most // n))), kv, group, m, n, window, sinks, dtype, ragged=rng.random() < 0.5)
        n = _size(rng, 64, 4096 if dtype == "fp32" else 16384)
        m = n if rng.random() < 0.7 else _size(rng, 8, n)
        most = (2 ** 28 if dtype == "fp32" else 2 ** 31) // (kv * group * m * (min(n, window + 512) if window else n))
        return _case(op, _size(rng, 1, max(1, min(8, most))), kv, group, m, n, window, sinks, dtype, ragged=rng.random() < 0.5)
    if op == "pack":
        n = _size(rng, 64, 131072)
        keep = max(1, int(n * rng.choice([0.05, 0.1, 0.25, 0.5])))
        count = _size(rng, 1, max(1, min(32, 2 ** 22 // (n * kv))))
        return _case(op, count, kv, 4, 1, n, dtype=dtype, keep=keep, ragged=rng.random() < 0.5)
    keep = _size(rng, 1, 16384)
    count = _size(rng, 1, max(1, min(64, 2 ** 21 // (keep * kv))))
    return _case(op, count, kv, group, rng.choice([1, 1, 1, 2, 3, 6]), dtype=dtype, keep=keep, tail=rng.choice([0, 1, 130, 513]) or 8,
                 mx=rng.random() < 0.6, ragged=rng.random() < 0.6)


# ---- inputs -------------------------------------------------------------------------------------


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _rows(g, shape, dtype, channels):
    """Rows of a cache [.., heads, rows, 128]: keys have outlier channels, values heavy-tailed row norms."""
    x = torch.randn(shape, generator=g, device="cuda")
    if channels:
        x *= torch.exp(0.7 * torch.randn((*shape[:-2], 1, D), generator=g, device="cuda"))
    else:
        z = torch.randn((*shape[:-1], 4), generator=g, device="cuda")
        x *= (z[..., :1] / (z[..., 1:].square().sum(-1, keepdim=True) / 3.0).sqrt()).abs()
    return x.to(dtype)


def _lengths(case, seed, top):
    """Tokens of every sequence: the longest has `top`; ragged: the others from a quarter of it on, one of four shorter than m."""
    c, r = case, np.random.default_rng([seed, 7])
    v = np.full(c["count"], top, dtype=np.int64)
    if c["ragged"]:
        v[1:] = r.integers(max(0, top // 4), top + 1, c["count"] - 1)
        few = r.integers(0, c["m"] + 1, c["count"])
        v[3::4] = np.minimum(few, top)[3::4]
    return v.astype(np.int32)


def _budgets(case, seed, heads):
    """Rows kept per head: equal, or a layer's (a sequence's) total shared out unevenly over its heads."""
    c = case
    b = np.full(heads, c["keep"], dtype=np.int64)
    if c["ragged"]:
        share = np.random.default_rng([seed, 8]).dirichlet(np.ones(c["kv"]), c["count"])
        b = np.floor(share * c["keep"] * c["kv"]).astype(np.int64).reshape(-1)
        if c["op"] == "pack":
            b = np.minimum(b, c["n"])
    return b.astype(np.int32)


def _context(case, layers, tokens):
    from paper_2509_15038_amd import binding
    return binding.Context(layers, case["kv"], case["group"], D, 32, case["dtype"], tokens, 1)


def prepare(case, seed):
    c, dt = case, _type(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(1000 + seed)
    count, kv, group, m, n = c["count"], c["kv"], c["group"], c["m"], c["n"]
    s = {"case": c}
    if c["op"] == "rotate":
        s["qkv"] = torch.randn((count, m, (group + 2) * kv * D), generator=g, device="cuda").to(dt)
        if c["norm"]:
            s["qw"] = (1 + 0.2 * torch.randn((D,), generator=g, device="cuda")).to(dt)
            s["kw"] = (1 + 0.2 * torch.randn((D,), generator=g, device="cuda")).to(dt)
        # positions run on from those of the prompt, cache rows from those of the tokens since
        start = np.random.default_rng([seed, 9]).integers(0, n - m + 1, count) if c["ragged"] else np.zeros(count, dtype=np.int64)
        s["starts"] = torch.from_numpy(start.astype(np.int32)).cuda()
        first = np.random.default_rng([seed, 10]).integers(0, 1 + 98304 * (m == 1), count)
        s["positions"] = torch.from_numpy((first[:, None] + np.arange(m)[None]).astype(np.int32)).cuda()
        angle = torch.arange(131072, dtype=torch.float64, device="cuda")[:, None] * 500000.0 ** (-torch.arange(0, D, 2, device="cuda") / D)
        s["table"] = torch.stack([angle.cos(), angle.sin()], 1).float().contiguous()
        s["Q"] = torch.empty((count, m, kv * group, D), dtype=dt, device="cuda")
        s["K"] = torch.zeros((count, kv, n, D), dtype=dt, device="cuda")
        s["V"] = torch.zeros_like(s["K"])
    elif c["op"] == "attend":
        s["K"], s["V"] = (_rows(g, (count, kv, n, D), dt, ch) for ch in (True, False))
        s["Q"] = torch.randn((count, m, kv * group, D), generator=g, device="cuda").to(dt)
        s["lengths"] = torch.from_numpy(_lengths(c, seed, n)).cuda()
    elif c["op"] == "pack":
        s["K"], s["V"] = (_rows(g, (count, kv, n, D), dt, ch) for ch in (True, False))
        b = _budgets(c, seed, count * kv)
        s["offsets"] = np.concatenate([[0], np.cumsum(b, dtype=np.int64)])
        s["rows_at"], rows = torch.from_numpy(s["offsets"]).cuda(), int(s["offsets"][-1])
        # kept tokens of every head, ascending: those whose score is among the head's `budget` largest
        order = torch.rand((count * kv, n), generator=g, device="cuda").argsort(1).argsort(1)
        s["indices"] = (order < torch.from_numpy(b).cuda()[:, None]).nonzero()[:, 1].to(torch.int32)
        s["K_codes"], s["V_codes"] = (torch.empty((rows, D // 2), dtype=torch.uint8, device="cuda") for _ in range(2))
        s["K_scales"], s["V_scales"] = (torch.empty((rows, D // 32), dtype=torch.uint8, device="cuda") for _ in range(2))
        s["K_out"], s["V_out"] = (torch.empty((rows, D), dtype=dt, device="cuda") for _ in range(2))
    else:
        b = _budgets(c, seed, count * kv)
        off = np.concatenate([[0], np.cumsum(b, dtype=np.int64)])
        s["total"], s["most"] = int(off[-1]), int(b.max())
        s["offsets"] = torch.from_numpy(off).cuda()
        rows = max(1, s["total"])
        s["K"], s["V"] = (_rows(g, (rows, D), dt, ch) for ch in (True, False))
        if c["mx"]:
            for t in "KV":
                s[t + "_codes"], s[t + "_scales"] = _in_four_bits(s.pop(t).float())
        s["K_tail"], s["V_tail"] = (_rows(g, (count, kv, c["tail"], D), dt, ch) for ch in (True, False))
        s["lengths"] = torch.from_numpy(_lengths(c, seed, c["tail"])).cuda()
        s["Q"] = torch.randn((count, m, kv * group, D), generator=g, device="cuda").to(dt)
    if c["op"] in ("attend", "kept"):
        s["out"] = torch.empty((count, m, kv * group, D), dtype=dt, device="cuda")
        s["lse"] = torch.empty((count, kv * group, m), dtype=torch.float32, device="cuda")
    if own:
        s["ctx"] = _context(c, count if c["op"] == "pack" else 1, max(n, c["tail"], 1))
    return s


# ---- one pass -----------------------------------------------------------------------------------


def run(s):
    c = s["case"]
    if not own:
        return {"rotate": _plain_rotate, "attend": _plain_attend, "pack": _plain_pack, "kept": _plain_kept}[c["op"]](s)
    ctx = s["ctx"]
    if c["op"] == "rotate":
        ctx.rotate(s["qkv"], c["count"], c["m"], s["table"], s["Q"], s["K"], s["V"], c["n"], starts=s["starts"], positions=s["positions"],
                   q_weight=s.get("qw"), k_weight=s.get("kw"), eps=EPS, pairs=c["pairs"])
        return {"Q": s["Q"], "K": s["K"], "V": s["V"]}
    if c["op"] == "attend":
        ctx.attend(s["Q"], s["K"], s["V"], c["count"], c["m"], c["n"], c["n"], s["out"], lengths=s["lengths"], window=c["window"],
                   n_sink=c["sinks"], lse=s["lse"])
        return {"out": s["out"], "lse": s["lse"]}
    if c["op"] == "pack":
        rows = s["K_out"].shape[0]
        ctx.compact_mx(s["K"], s["V"], c["n"], s["indices"], s["rows_at"], rows, s["K_codes"], s["K_scales"], s["V_codes"], s["V_scales"])
        for t in "KV":
            ctx.expand_mx(s[t + "_codes"], s[t + "_scales"], rows, s[t + "_out"])
        return {"K": s["K_out"], "V": s["V_out"]}
    since = dict(K_tail=s["K_tail"], V_tail=s["V_tail"], tail_n=c["tail"], tail_stride=c["tail"], tail_lengths=s["lengths"], lse=s["lse"])
    if c["mx"]:
        ctx.attend_kept_mx(s["Q"], s["K_codes"], s["K_scales"], s["V_codes"], s["V_scales"], s["offsets"], c["count"], c["m"], s["total"],
                           s["out"], **since)
    else:
        ctx.attend_kept(s["Q"], s["K"], s["V"], s["offsets"], c["count"], c["m"], s["total"], s["out"], **since)
    return {"out": s["out"], "lse": s["lse"]}


# ---- the plain forms ----------------------------------------------------------------------------


def _plain_rotate(s):
    c, dt = s["case"], _type(s["case"])
    count, kv, group, m = c["count"], c["kv"], c["group"], c["m"]
    x = s["qkv"].view(count, m, (group + 2) * kv, D)
    q, k, v = x[:, :, : group * kv].float(), x[:, :, group * kv: (group + 1) * kv].float(), x[:, :, (group + 1) * kv:]
    if c["norm"]:
        q = q * torch.rsqrt(q.square().mean(-1, keepdim=True) + EPS) * s["qw"].float()
        k = k * torch.rsqrt(k.square().mean(-1, keepdim=True) + EPS) * s["kw"].float()
    t = s["table"][s["positions"].long()]
    cos, sin = t[:, :, None, 0], t[:, :, None, 1]

    def turned(y):
        if c["pairs"]:
            a, b = y[..., 0::2], y[..., 1::2]
            return torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        a, b = y[..., : D // 2], y[..., D // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    s["Q"].copy_(turned(q))
    rows = (s["starts"].long()[:, None] + torch.arange(m, device="cuda"))[:, None, :, None].expand(count, kv, m, D)
    s["K"].scatter_(2, rows, turned(k).to(dt).transpose(1, 2).contiguous())
    s["V"].scatter_(2, rows, v.transpose(1, 2).contiguous())
    return {"Q": s["Q"], "K": s["K"], "V": s["V"]}


def _softmax_product(parts, dt, count, m, kv, group):
    """Joint softmax over several (scores [.., rows, keys] with -inf where hidden, values [.., keys, 128]); out and log-sum-exp."""
    top = torch.stack([x.amax(-1, keepdim=True) for x, _ in parts]).amax(0)
    top = torch.where(top == -math.inf, 0.0, top)
    p = [(x.sub_(top).exp_(), v) for x, v in parts]
    total = sum(x.sum(-1, keepdim=True) for x, _ in p)
    out = sum(torch.matmul(x, v) for x, v in p) / torch.where(total == 0, 1.0, total)
    lse = top + total.log()                                            # [count, kv, .., group * tokens, 1]
    return out, lse


def _plain_attend(s):
    c, dt = s["case"], _type(s["case"])
    count, kv, group, m, n = c["count"], c["kv"], c["group"], c["m"], c["n"]
    sinks = c["sinks"]
    window = c["window"] if 0 < c["window"] < n else n
    block = m if window == n else max(64, min(m, 512, 1 << (window - 1).bit_length()))
    blocks = -(-m // block)
    len_ = s["lengths"].long()
    Q = torch.zeros((count, blocks * block, kv, group, D), device="cuda")
    Q[:, :m] = s["Q"].view(count, m, kv, group, D)
    Q = Q.view(count, blocks, block, kv, group, D).permute(0, 3, 1, 4, 2, 5).reshape(count, kv, blocks, group * block, D) * D ** -0.5
    at = len_[:, None, None] - m + torch.arange(blocks * block, device="cuda").view(1, blocks, block)       # positions of the queries
    K, V = s["K"].float(), s["V"].float()
    if window == n:
        j = torch.arange(n, device="cuda").expand(count, 1, n)
        Kw, Vw = K[:, :, None], V[:, :, None]
    else:
        j = at[:, :, :1] - window + 1 + torch.arange(window + block - 1, device="cuda")
        pick = (torch.arange(count * kv, device="cuda").view(count, kv, 1) * n + j.clamp(0, n - 1).view(count, 1, -1)).view(-1)
        Kw, Vw = (x.view(-1, D)[pick].view(count, kv, blocks, -1, D) for x in (K, V))
    seen = (j[:, :, None] <= at[..., None]) & (at[..., None] - j[:, :, None] < window) & (j[:, :, None] >= 0)
    hidden = ~seen[:, None, :, None]
    S = torch.matmul(Q, Kw.transpose(-1, -2)).view(count, kv, blocks, group, block, -1)
    parts = [(S.masked_fill_(hidden, -math.inf).view(count, kv, blocks, group * block, -1), Vw)]
    if sinks and window < n:
        j = torch.arange(min(sinks, n), device="cuda")
        seen = (j <= at[..., None]) & (at[..., None] - j >= window)                                         # those not in the window
        Ks, Vs = K[:, :, None, : len(j)], V[:, :, None, : len(j)]
        S = torch.matmul(Q, Ks.transpose(-1, -2)).view(count, kv, blocks, group, block, -1)
        parts.append((S.masked_fill_(~seen[:, None, :, None], -math.inf).view(count, kv, blocks, group * block, -1), Vs))
    out, lse = _softmax_product(parts, dt, count, m, kv, group)
    out = out.view(count, kv, blocks, group, block, D).permute(0, 2, 4, 1, 3, 5).reshape(count, -1, kv * group, D)[:, :m]
    lse = lse.view(count, kv, blocks, group, block).transpose(2, 3).reshape(count, kv * group, -1)[..., :m]
    return {"out": out.to(dt), "lse": lse.contiguous()}


def _two_to(e):
    """2^(e - 127) in 32 bits, from the bits (a power function may be a rounding off), 0 <= e <= 254."""
    return torch.where(e == 0, 1 << 22, e << 23).to(torch.int32).view(torch.float32)


def _in_four_bits(x):
    """Rows [.., 128] in 32 bits as blocks of 32 values in 4 bits with a power of two: codes [.., 64] (the even channel in the low half), exponents + 127 [.., 4]."""
    b = x.view(*x.shape[:-1], D // 32, 32)
    e = ((b.abs().amax(-1).view(torch.int32) >> 23) - 2).clamp(min=0)                                       # + 127
    y = b * _two_to(254 - e)[..., None]
    a = y.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5)) | (y < 0).to(torch.uint8) << 3
    code = code.view(*x.shape[:-1], D // 2, 2)
    return code[..., 0] | code[..., 1] << 4, e.to(torch.uint8)


def _from_four_bits(codes, scales):
    code = torch.stack([codes & 15, codes >> 4], -1).view(*codes.shape[:-1], D // 32, 32).long()
    value = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device="cuda")[code]
    return (value * _two_to(scales.int())[..., None]).view(*codes.shape[:-1], D)


def _plain_pack(s):
    c, dt = s["case"], _type(s["case"])
    off = torch.from_numpy(s["offsets"]).cuda()
    head = torch.repeat_interleave(torch.arange(off.numel() - 1, device="cuda"), off.diff(), output_size=int(s["offsets"][-1]))
    pick = head * c["n"] + s["indices"].long()
    K, V = (_from_four_bits(*_in_four_bits(s[t].view(-1, D)[pick].float())).to(dt) for t in "KV")
    return {"K": K, "V": V}


def _plain_kept(s):
    c, dt = s["case"], _type(s["case"])
    count, kv, group, m = c["count"], c["kv"], c["group"], c["m"]
    K, V = ((_from_four_bits(s[t + "_codes"], s[t + "_scales"]) if c["mx"] else s[t].float()) for t in "KV")
    Q = s["Q"].view(count, m, kv, group, D).permute(0, 2, 3, 1, 4).reshape(count, kv, group * m, D).float() * D ** -0.5
    begin, rows = s["offsets"][:-1].view(count, kv, 1), s["offsets"].diff().view(count, kv, 1)
    j = torch.arange(max(1, s["most"]), device="cuda")
    pick = (begin + j).clamp(max=K.shape[0] - 1).view(-1)
    Kk, Vk = (x[pick].view(count, kv, -1, D) for x in (K, V))
    S = torch.matmul(Q, Kk.transpose(-1, -2)).masked_fill_((j >= rows)[:, :, None], -math.inf)
    at = s["lengths"].long()[:, None] - m + torch.arange(m, device="cuda")
    hidden = torch.arange(c["tail"], device="cuda") > at[..., None]
    Kt, Vt = s["K_tail"].float(), s["V_tail"].float()
    T = torch.matmul(Q, Kt.transpose(-1, -2)).view(count, kv, group, m, -1).masked_fill_(hidden[:, None, None], -math.inf).view(count, kv, group * m, -1)
    out, lse = _softmax_product([(S, Vk), (T, Vt)], dt, count, m, kv, group)
    out = out.view(count, kv, group, m, D).permute(0, 3, 1, 2, 4).reshape(count, m, kv * group, D)
    return {"out": out.to(dt), "lse": lse.view(count, kv * group, m).contiguous()}


# ---- what a pass cannot do without ----------------------------------------------------------------


def _visible(case, lengths):
    """(pairs of a token and a key that it sees, keys that any token sees), over all sequences, one KV head."""
    c, pairs, keys = case, 0, 0
    for L in lengths.tolist():
        at = np.arange(max(0, L - c["m"]), L, dtype=np.int64)
        if not at.size:
            continue
        w = c["window"] or L
        near = np.minimum(at + 1, w)
        first = np.minimum(np.maximum(at + 1 - w, 0), c["sinks"])
        pairs += int((near + first).sum())
        keys += int(min(L, L - at[0] + w - 1)) + int(first[0])
    return pairs, min(keys, int(lengths.sum()))


def work(case):
    c = case
    b = 2 if c["dtype"] == "bf16" else 4
    count, kv, group, m, row = c["count"], c["kv"], c["group"], c["m"], D * b
    if c["op"] == "rotate":
        return {"bytes": count * m * (2 * (group + 2) * kv * row + 2 * D // 2 * 4 + 4), "flops": count * m * (group + 1) * kv * D * (3 + 4 * c["norm"])}
    if c["op"] == "attend":
        pairs, keys = _visible(c, _lengths(c, 0, c["n"]))
        return {"bytes": 2 * keys * kv * row + count * m * kv * group * (2 * row + 4), "flops": 4 * D * pairs * kv * group}
    if c["op"] == "pack":
        kept = int(_budgets(c, 0, count * kv).sum())
        return {"bytes": kept * (2 * row + 4 + 4 * (D // 2 + D // 32) + 2 * row), "flops": 2 * kept * 2 * D}
    kept, tail = int(_budgets(c, 0, count * kv).sum()), int(_lengths(c, 0, c["tail"]).sum()) * kv
    kept_row = D // 2 + D // 32 if c["mx"] else row
    return {"bytes": 2 * kept * kept_row + 2 * tail * row + count * m * kv * group * (2 * row + 4), "flops": 4 * D * m * group * (kept + tail)}


# ---- the same in 64 bits ------------------------------------------------------------------------


def _attention64(q, K, V, seen):
    """One head: q [rows, 128], K, V [keys, 128], seen [rows, keys] or None -> out, log-sum-exp, in 64 bits."""
    x = (q @ K.T) / math.sqrt(D)
    if seen is not None:
        x[~seen] = -math.inf
    lse = torch.logsumexp(x, 1)
    return torch.nan_to_num(torch.exp(x - lse[:, None]) if x.shape[1] else x, nan=0.0) @ V, lse


def exact(case, seed):
    """The operators from their definitions, head by head and stretch by stretch."""
    c = case
    plain = prepare_inputs(c, seed)
    count, kv, group, m, n = c["count"], c["kv"], c["group"], c["m"], c["n"]
    if c["op"] == "pack":
        levels = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device="cuda")
        odd = 1e-12 * (torch.arange(8, device="cuda") % 2)             # of two levels equally near, the one of the even code
        found = {}
        for t in "KV":
            found[t], begin = torch.empty((int(plain["offsets"][-1]), D), dtype=torch.float64, device="cuda"), plain["offsets"].tolist()
            for h in range(count * kv):
                pick = plain["indices"][begin[h]: begin[h + 1]].long()
                x = plain[t].view(count * kv, n, D)[h].index_select(0, pick).double().view(-1, 32)
                unit = 2.0 ** (torch.floor(torch.log2(x.abs().amax(1, keepdim=True))) - 2)
                near = ((x / unit).abs()[..., None] - levels).abs().add_(odd).argmin(-1)
                found[t][begin[h]: begin[h + 1]] = (levels[near] * x.sign() * unit).view(-1, D)
        return found
    if c["op"] == "rotate":
        Q, K, V = (plain[t].double() for t in "QKV")
        Q.zero_()
        half = D // 2
        first = [2 * i for i in range(half)] if c["pairs"] else list(range(half))
        second = [2 * i + 1 for i in range(half)] if c["pairs"] else list(range(half, D))
        for b in range(count):
            start = int(plain["starts"][b])
            z = torch.view_as_complex(plain["table"][plain["positions"][b].long()].double().transpose(1, 2).contiguous())   # e^(i angle) [m, 64]
            x = plain["qkv"][b].double().view(m, -1, D)
            for h in range((group + 1) * kv):
                y, query = x[:, h], h < group * kv
                if c["norm"]:
                    y = y / (torch.linalg.vector_norm(y, dim=1, keepdim=True) ** 2 / D + EPS).sqrt() * plain["qw" if query else "kw"].double()
                w = torch.complex(y[:, first], y[:, second]) * z
                to = Q[b, :, h] if query else K[b, h - group * kv, start: start + m]
                to[:, first], to[:, second] = w.real, w.imag
            V[b, :, start: start + m] = x[:, (group + 1) * kv:].transpose(0, 1)
        return {"Q": Q, "K": K, "V": V}
    out = torch.zeros((count, m, kv * group, D), dtype=torch.float64, device="cuda")
    lse = torch.full((count, kv * group, m), -math.inf, dtype=torch.float64, device="cuda")
    if c["op"] == "attend":
        rows, K, V = _lengths(c, seed, n).tolist(), plain["K"], plain["V"]
        pairs = _visible(c, np.array(rows))[0] * kv * group
        if pairs > 2 ** 34:
            return None
        for b in range(count):
            for t0 in range(0, m, 2048):
                t1 = min(m, t0 + 2048)
                low, high = rows[b] - m + t0, rows[b] - m + t1         # positions of these tokens
                if high <= 0:
                    continue
                w = c["window"] or n
                j = torch.tensor(sorted(set(range(max(0, low - w + 1), high)) | set(range(min(c["sinks"], high)))), device="cuda")
                at = torch.arange(low, high, device="cuda")[:, None]
                seen = (j <= at) & ((at - j < w) | (j < c["sinks"]))
                for h in range(kv):
                    k, v = K[b, h].index_select(0, j).double(), V[b, h].index_select(0, j).double()
                    for q in range(h * group, (h + 1) * group):
                        out[b, t0:t1, q], lse[b, q, t0:t1] = _attention64(plain["Q"][b, t0:t1, q].double(), k, v, seen)
        return {"out": out, "lse": lse}
    off, tails = plain["offsets"].tolist(), _lengths(c, seed, c["tail"]).tolist()
    levels = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device="cuda")

    def kept(t, a, b):
        if not c["mx"]:
            return plain[t][a:b].double()
        x, e = plain[t + "_codes"][a:b].long(), plain[t + "_scales"][a:b].double() - 127
        y = torch.empty((b - a, D), dtype=torch.float64, device="cuda")
        for part, code in ((0, x % 16), (1, x // 16)):
            y[:, part::2] = levels[code % 8] * torch.where(code >= 8, -1.0, 1.0)
        return y * torch.repeat_interleave(2.0 ** e, 32, dim=1)

    for b in range(count):
        L = tails[b]
        for h in range(kv):
            a, z = off[b * kv + h], off[b * kv + h + 1]
            k = torch.cat([kept("K", a, z), plain["K_tail"][b, h, :L].double()])
            v = torch.cat([kept("V", a, z), plain["V_tail"][b, h, :L].double()])
            at = torch.arange(L - m, L, device="cuda")[:, None]
            seen = torch.cat([torch.ones((m, z - a), dtype=torch.bool, device="cuda"), torch.arange(L, device="cuda") <= at], 1)
            for q in range(h * group, (h + 1) * group):
                out[b, :, q], lse[b, q] = _attention64(plain["Q"][b, :, q].double(), k, v, seen)
    return {"out": out, "lse": lse}


def prepare_inputs(case, seed):
    """The inputs alone, whatever `own` says."""
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was
