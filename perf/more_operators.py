"""What a program asks of the library once a cache has to stay at its size and to serve several answers: the
cases that these operators are measured on, beside those of operators.py.

`listed()` names the cases, `draw(rng)` gives more of the same ranges.  A case is a plain dict; `op` says
which operator it is:

    axes      norms and the position rotation where a token stands at several positions (time, height,
              width), each angle turned by that of its axis; the new rows of the cache: Context.rotate_axes
    weights   the attention weight that every cached key got from m tokens of a sequence, over all query heads
              of its KV head, added to what it had: whole prompts (m = n), the last tokens of a prompt,
              generated tokens: Context.attend_weights
    evict     the rows of least accumulated weight leave a cache, first and recent tokens stay; in place, as
              between generated tokens, or into another cache, as after a prompt: Context.evict
    shared    attention of m new tokens of each of `share` sequences over the kept rows that they have in common,
              in the cache's type or in 4 bits, and over their own tokens since: Context.attend_shared,
              Context.attend_shared_mx

and the sizes are

    count     sequences (shared: prefixes, each with `share` sequences); kv: KV heads; group: query heads per KV head
    m, n      new tokens of a sequence, and its tokens in all (of the longest; ragged: the others are shorter)
    axes, mixed (neighbouring angles are of different axes; else an axis has a stretch of them), norm, pairs
    window, sinks; decay of the weights before (weights); recent tokens that stay (evict)
    keep      rows kept per head (shared, ragged: drawn unevenly over the heads); place: evict in place
    tail      tokens since (shared)
    dtype     "bf16" or "fp32"; mx: the kept rows are held in 4 bits

Head dimension 128 throughout, as in the configurations of paper_2509_15038_amd/workloads.py.
"""

import math

import numpy as np
import torch

D, EPS = 128, 1e-5
own = False


def _case(op, count=1, kv=8, group=4, m=1, n=1, dtype="bf16", axes=0, mixed=False, norm=False, pairs=False, window=0, sinks=0, decay=1.0, recent=0, keep=0,
          place=False, share=1, tail=0, mx=False, ragged=False, name=None):
    c = {"op": op, "count": count, "kv": kv, "group": group, "m": m, "n": n, "dtype": dtype, "axes": axes, "mixed": mixed, "norm": norm, "pairs": pairs,
         "window": window, "sinks": sinks, "decay": decay, "recent": recent, "keep": keep, "place": place, "share": share, "tail": tail, "mx": mx,
         "ragged": ragged}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the projections of one generated token of 4 sequences after prompts with pictures: latency only
        _case("axes", count=4, m=1, n=256, axes=3, norm=True, ragged=True, name="axes-token"),
        # one layer of a video prompt, 32 frames of 32 x 32 patches: time, height and width, queries and keys normalised
        _case("axes", m=32768, n=32768, axes=3, norm=True, name="axes-video-32k"),
        # the weights of a whole 8k prompt, one layer: what the first eviction goes by
        _case("weights", m=8192, n=8192, decay=0.0, name="weights-prompt-8k"),
        # the weights that the last 32 tokens of a 32k prompt give it (an observation window)
        _case("weights", m=32, n=32768, decay=0.0, name="weights-last-32-of-32k"),
        # a generated token of 32 sequences over caches of 4096 rows, older weights fading
        _case("weights", count=32, m=1, n=4096, decay=0.99, ragged=True, name="weights-token-batch"),
        # a few odd prompts side by side in fp32, with a window and four first tokens, ragged
        _case("weights", count=3, kv=2, m=1021, n=1021, window=257, sinks=4, dtype="fp32", decay=0.0, ragged=True, name="weights-1021-fp32"),
        # 10 % of a 32k prompt into a cache of its own, one layer
        _case("evict", n=32768, keep=3276, sinks=4, recent=64, name="evict-prompt-32k"),
        # one row a head for the token that was just generated, 32 sequences, in place
        _case("evict", count=32, n=3277, keep=3276, sinks=4, recent=64, place=True, name="evict-token-batch"),
        # a whole model's caches at once (16 layers as sequences), ragged, to a quarter
        _case("evict", count=16, n=16384, keep=4096, sinks=4, recent=256, ragged=True, name="evict-model-16k"),
        # a token of 16 answers to one compressed prompt (10 % of 32k), 200 tokens since
        _case("shared", share=16, keep=3276, tail=200, ragged=True, name="shared-answers-16"),
        # 4 prompts of 128k tokens, 10 % kept in 4 bits, 16 answers each
        _case("shared", count=4, share=16, keep=13107, tail=513, mx=True, ragged=True, name="shared-batch-mx"),
        # 64 sequences that begin with the same 128k tokens, all of them kept
        _case("shared", share=64, keep=131072, tail=77, name="shared-128k-64"),
    ]


def _size(rng, low, high):
    """Spread over the logarithm, odd half the time (and no multiple of 1024 but powers of two)."""
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    v = v | 1 if rng.random() < 0.5 else v
    return max(low, min(high, v if v % 1024 or not v & (v - 1) else v + 1))


def draw(rng):
    """One more case: within the listed ones' ranges and costs."""
    op = rng.choice(["axes", "weights", "weights", "weights", "evict", "evict", "shared", "shared", "shared"])
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    kv, group = rng.choice([(8, 4), (8, 4), (8, 2), (2, 4), (1, 8), (2, 7), (8, 5), (1, 1)])
    if op == "axes":
        m = 1 if rng.random() < 0.3 else _size(rng, 2, 32768 if dtype == "bf16" else 16384)
        count = _size(rng, 1, max(1, min(64, 32768 // m)))
        return _case(op, count, kv, group, m, max(m, 256) + rng.choice([0, 1, 130]), dtype, axes=rng.choice([1, 2, 3, 3, 4]), mixed=rng.random() < 0.4,
                     norm=rng.random() < 0.6, pairs=rng.random() < 0.3, ragged=count > 1 and rng.random() < 0.7)
    if op == "weights":
        window = 0 if rng.random() < 0.6 else _size(rng, 16, 4096)
        sinks = rng.choice([0, 4, 4, 64]) if window else 0
        decay = rng.choice([0.0, 1.0, 0.99])
        if rng.random() < 0.4:                                         # generated tokens, a few a sequence
            m, n = rng.choice([1, 1, 1, 2, 5]), _size(rng, 8, 131072)
            most = 2 ** 21 // (kv * (2 if dtype == "fp32" else 1))     # rows in all
            return _case(op, _size(rng, 1, max(1, min(64, most // n))), kv, group, m, n, dtype, window=window, sinks=sinks, decay=decay,
                         ragged=rng.random() < 0.5)
        n = _size(rng, 64, 2048 if dtype == "fp32" else 8192)
        m = n if rng.random() < 0.5 else _size(rng, 8, n)
        if rng.random() < 0.3:                                         # the last tokens of a long prompt
            m, n = _size(rng, 8, 64), _size(rng, 1024, 32768)
        most = (2 ** 28 if dtype == "fp32" else 2 ** 31) // (kv * group * m * n)
        return _case(op, _size(rng, 1, max(1, min(8, most))), kv, group, m, n, dtype, window=window, sinks=sinks, decay=decay, ragged=rng.random() < 0.5)
    if op == "evict":
        place = rng.random() < 0.5
        keep = _size(rng, 16, 16384)
        n = keep + (_size(rng, 1, 64) if place else _size(rng, 1, 8 * keep))
        sinks = rng.choice([0, 1, 4])
        count = _size(rng, 1, max(1, min(64, 2 ** 21 // (n * kv))))
        return _case(op, count, kv, group, 1, n, dtype, sinks=sinks, recent=rng.choice([0, 1, (keep - sinks) // 2, keep - sinks]), keep=keep, place=place,
                     ragged=rng.random() < 0.5)
    keep = _size(rng, 1, 65536)
    count = _size(rng, 1, max(1, min(16, 2 ** 19 // (keep * kv))))
    m, tail = rng.choice([1, 1, 1, 2, 5]), rng.choice([0, 1, 130, 513]) or 8
    most = (2 ** 26 if dtype == "fp32" else 2 ** 28) // (count * kv * group * m * (keep + tail))
    return _case(op, count, kv, group, m, dtype=dtype, share=_size(rng, 1, max(1, min(64, most, 2 ** 21 // (count * kv * tail)))), keep=keep, tail=tail,
                 mx=rng.random() < 0.4, ragged=rng.random() < 0.6)


# ---- inputs -------------------------------------------------------------------------------------


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _rows(g, shape, dtype, channels):
    """Rows of a cache [.., heads, rows, 128]: keys have outlier channels, values heavy-tailed row norms."""
    x = torch.randn(shape, generator=g, device="cuda")
    if channels:
        x *= torch.exp(0.5 * torch.randn((*shape[:-2], 1, D), generator=g, device="cuda"))
    else:
        z = torch.randn((*shape[:-1], 4), generator=g, device="cuda")
        x *= (z[..., :1] / (z[..., 1:].square().sum(-1, keepdim=True) / 3.0).sqrt()).abs()
    return x.to(dtype)


def _lengths(case, seed, count, top, least):
    """Tokens of every sequence: the longest has `top`; ragged: the others from a quarter of it on, one of four fewer than `least`."""
    v = np.full(count, top, dtype=np.int64)
    if case["ragged"]:
        r = np.random.default_rng([seed, 7])
        v[1:] = r.integers(max(0, top // 4), top + 1, count - 1)
        few = r.integers(0, least + 1, count)
        v[3::4] = np.minimum(few, top)[3::4]
    return v.astype(np.int32)


def _sequences(case, seed):
    """The lengths that a case's arrays of lengths hold."""
    c = case
    if c["op"] == "weights":
        return _lengths(c, seed, c["count"], c["n"], c["m"])
    if c["op"] == "evict":
        return _lengths(c, seed, c["count"], c["n"], c["keep"])
    return _lengths(c, seed, c["count"] * c["share"], c["tail"], c["m"])


def _budgets(case, seed):
    """Rows kept per head of every prefix: equal, or a prefix's total shared out unevenly over its heads."""
    c = case
    if not c["ragged"]:
        return np.full(c["count"] * c["kv"], c["keep"], dtype=np.int64)
    share = np.random.default_rng([seed, 8]).dirichlet(np.ones(c["kv"]), c["count"])
    return np.floor(share * c["keep"] * c["kv"]).astype(np.int64).reshape(-1)


def _axis_of(case):
    """The axis of each of the 64 angles: in turn, or a stretch of them each, the first axis with the highest frequencies and the fewest."""
    axes = case["axes"]
    if case["mixed"]:
        return (np.arange(D // 2) % axes).astype(np.uint8)
    ends = {1: [64], 2: [32, 64], 3: [16, 40, 64], 4: [16, 32, 48, 64]}[axes]
    return np.searchsorted(ends, np.arange(D // 2), side="right").astype(np.uint8)


def prepare(case, seed):
    c, dt = case, _type(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(2000 + seed)
    count, kv, group, m, n = c["count"], c["kv"], c["group"], c["m"], c["n"]
    s = {"case": c}
    if c["op"] == "axes":
        s["qkv"] = torch.randn((count, m, (group + 2) * kv * D), generator=g, device="cuda").to(dt)
        if c["norm"]:
            s["qw"] = (1 + 0.2 * torch.randn((D,), generator=g, device="cuda")).to(dt)
            s["kw"] = (1 + 0.2 * torch.randn((D,), generator=g, device="cuda")).to(dt)
        r = np.random.default_rng([seed, 9])
        start = r.integers(0, n - m + 1, count) if c["ragged"] else np.zeros(count, dtype=np.int64)
        s["starts"] = torch.from_numpy(start.astype(np.int32)).cuda()
        # a prompt is frames of up to 32 x 32 patches: frame, row and column, all from a sequence's first position on; a generated token stands at one position
        # on all axes; a fourth axis counts the tokens
        first, i = r.integers(0, 1 + 98304 * (m == 1), count)[:, None], np.arange(m)[None]
        at = np.stack([i // 1024 + first, i // 32 % 32 + first, i % 32 + first, i + first])[: c["axes"]]
        s["positions"] = torch.from_numpy(at.astype(np.int32).reshape(c["axes"], count * m)).cuda()
        s["axis_of"] = _axis_of(c)
        angle = torch.arange(131072, dtype=torch.float64, device="cuda")[:, None] * 500000.0 ** (-torch.arange(0, D, 2, device="cuda") / D)
        s["table"] = torch.stack([angle.cos(), angle.sin()], 1).float().contiguous()
        s["Q"] = torch.empty((count, m, kv * group, D), dtype=dt, device="cuda")
        s["K"] = torch.zeros((count, kv, n, D), dtype=dt, device="cuda")
        s["V"] = torch.zeros_like(s["K"])
    elif c["op"] == "weights":
        s["K"] = _rows(g, (count, kv, n, D), dt, True)
        s["Q"] = torch.randn((count, m, kv * group, D), generator=g, device="cuda").to(dt)
        s["lengths"] = torch.from_numpy(_sequences(c, seed)).cuda()
        s["mass"] = torch.exp(2 * torch.randn((count, kv, n), generator=g, device="cuda"))
        s["lse"] = torch.stack([torch.stack([torch.logsumexp(_scores(s, b, h), -1) for h in range(kv)]) for b in range(count)])   # [count, kv, group, m]
        s["lse"] = s["lse"].view(count, kv * group, m).float()
    elif c["op"] == "evict":
        s["K"], s["V"] = (_rows(g, (count, kv, n, D), dt, ch) for ch in (True, False))
        # weights over several magnitudes, one of eight tokens nobody has looked at
        s["mass"] = torch.exp(2 * torch.randn((count, kv, n), generator=g, device="cuda")) * (torch.rand((count, kv, n), generator=g, device="cuda") > 0.125)
        s["lengths"] = torch.from_numpy(_sequences(c, seed)).cuda()
        s["positions"] = torch.arange(n, dtype=torch.int32, device="cuda").expand(count, kv, n).contiguous()
        if c["place"]:
            # rows have moved before: those below `keep` in an order of their own, with gaps between their positions
            order = torch.rand((count, kv, c["keep"]), generator=g, device="cuda").argsort(-1)
            s["positions"][:, :, : c["keep"]] = order.int() * 3
            s["positions"][:, :, c["keep"]:] += 2 * c["keep"]
        room = n if c["place"] else c["keep"] + 64
        s["room"] = room
        s["K_out"], s["V_out"] = (s["K"], s["V"]) if c["place"] else (torch.zeros((count, kv, room, D), dtype=dt, device="cuda") for _ in "KV")
        s["mass_out"], s["positions_out"] = torch.zeros((count, kv, room), device="cuda"), torch.zeros((count, kv, room), dtype=torch.int32, device="cuda")
        s["rows"] = torch.empty((count, kv, c["keep"]), dtype=torch.int32, device="cuda")
    else:
        b = _budgets(c, seed)
        off = np.concatenate([[0], np.cumsum(b, dtype=np.int64)])
        s["total"], s["most"] = int(off[-1]), int(b.max())
        s["offsets"] = torch.from_numpy(off).cuda()
        rows = max(1, s["total"])
        s["K"], s["V"] = (_rows(g, (rows, D), dt, ch) for ch in (True, False))
        if c["mx"]:
            for t in "KV":
                s[t + "_codes"], s[t + "_scales"] = _in_four_bits(s.pop(t).float())
        every = count * c["share"]
        s["K_tail"], s["V_tail"] = (_rows(g, (every, kv, c["tail"], D), dt, ch) for ch in (True, False))
        s["lengths"] = torch.from_numpy(_sequences(c, seed)).cuda()
        s["Q"] = torch.randn((every, m, kv * group, D), generator=g, device="cuda").to(dt)
        s["out"] = torch.empty((every, m, kv * group, D), dtype=dt, device="cuda")
        s["lse"] = torch.empty((every, kv * group, m), dtype=torch.float32, device="cuda")
    if own:
        from paper_2509_15038_amd import binding
        s["ctx"] = binding.Context(1, kv, group, D, 32, c["dtype"], max(n, c["tail"], 1), 1)
    return s


def _scores(s, b, h):
    """One KV head's scores, -infinity where a key is not seen: [group, m, n] in 32 bits."""
    c = s["case"]
    m, n, group = c["m"], c["n"], c["group"]
    q = s["Q"][b].view(m, c["kv"], group, D)[:, h].transpose(0, 1).reshape(group * m, D).float() * D ** -0.5
    x = (q @ s["K"][b, h].float().T).view(group, m, n)
    return x.masked_fill_(~_seen(c, s["lengths"][b]), -math.inf)


def _seen(c, lengths):
    """Whether token t of a sequence sees key j: lengths [..] -> [.., m, n]."""
    at = (lengths.long()[..., None] - c["m"] + torch.arange(c["m"], device="cuda"))[..., None]
    j = torch.arange(c["n"], device="cuda")
    seen = j <= at
    if c["window"]:
        seen = seen & ((at - j < c["window"]) | (j < c["sinks"]))
    return seen


# ---- one pass -----------------------------------------------------------------------------------


def run(s):
    c = s["case"]
    if not own:
        return {"axes": _plain_axes, "weights": _plain_weights, "evict": _plain_evict, "shared": _plain_shared}[c["op"]](s)
    ctx = s["ctx"]
    if c["op"] == "axes":
        ctx.rotate_axes(s["qkv"], c["count"], c["m"], s["table"], s["positions"], s["axis_of"], s["Q"], s["K"], s["V"], c["n"], starts=s["starts"],
                        q_weight=s.get("qw"), k_weight=s.get("kw"), eps=EPS, pairs=c["pairs"])
        return {"Q": s["Q"], "K": s["K"], "V": s["V"]}
    if c["op"] == "weights":
        ctx.attend_weights(s["Q"], s["K"], s["lse"], c["count"], c["m"], c["n"], c["n"], s["mass"], lengths=s["lengths"], window=c["window"],
                           n_sink=c["sinks"], decay=c["decay"])
        return {"mass": s["mass"]}
    if c["op"] == "evict":
        ctx.evict(s["K"], s["V"], s["mass"], c["count"], c["n"], c["n"], c["keep"], s["rows"], positions=s["positions"], lengths=s["lengths"],
                  n_sink=c["sinks"], recent=c["recent"], K_out=s["K_out"], V_out=s["V_out"], mass_out=s["mass_out"], positions_out=s["positions_out"],
                  out_stride=s["room"])
        return {"K": s["K_out"], "V": s["V_out"], "mass": s["mass_out"], "positions": s["positions_out"], "rows": s["rows"]}
    since = dict(K_tail=s["K_tail"], V_tail=s["V_tail"], tail_n=c["tail"], tail_stride=c["tail"], tail_lengths=s["lengths"], lse=s["lse"])
    if c["mx"]:
        ctx.attend_shared_mx(s["Q"], s["K_codes"], s["K_scales"], s["V_codes"], s["V_scales"], s["offsets"], c["count"], c["share"], c["m"], s["total"],
                             s["out"], **since)
    else:
        ctx.attend_shared(s["Q"], s["K"], s["V"], s["offsets"], c["count"], c["share"], c["m"], s["total"], s["out"], **since)
    return {"out": s["out"], "lse": s["lse"]}


# ---- the plain forms ----------------------------------------------------------------------------


def _plain_axes(s):
    c, dt = s["case"], _type(s["case"])
    count, kv, group, m = c["count"], c["kv"], c["group"], c["m"]
    x = s["qkv"].view(count, m, (group + 2) * kv, D)
    q, k, v = x[:, :, : group * kv].float(), x[:, :, group * kv: (group + 1) * kv].float(), x[:, :, (group + 1) * kv:]
    if c["norm"]:
        q = q * torch.rsqrt(q.square().mean(-1, keepdim=True) + EPS) * s["qw"].float()
        k = k * torch.rsqrt(k.square().mean(-1, keepdim=True) + EPS) * s["kw"].float()
    axis = torch.from_numpy(s["axis_of"]).cuda().long()
    at = s["positions"].long()[axis].T                                 # [tokens, 64]
    angle = torch.arange(D // 2, device="cuda")
    cos, sin = (s["table"][at, part, angle].view(count, m, 1, D // 2) for part in (0, 1))

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


def _plain_weights(s):
    c = s["case"]
    count, kv, group, m, n = c["count"], c["kv"], c["group"], c["m"], c["n"]
    q = s["Q"].view(count, m, kv, group, D).permute(0, 2, 3, 1, 4).reshape(count, kv, group * m, D).float() * D ** -0.5
    x = torch.matmul(q, s["K"].float().transpose(-1, -2).contiguous()).view(count, kv, group, m, n)
    lse = s["lse"].view(count, kv, group, m, 1)
    x = x.sub_(torch.where(lse == -math.inf, 0.0, lse)).masked_fill_(~_seen(c, s["lengths"])[:, None, None], -math.inf).exp_()
    got = x.view(count, kv, group * m, n).sum(2)
    rows = torch.arange(n, device="cuda") < s["lengths"].long()[:, None, None]
    s["mass"].copy_(torch.where(rows, (c["decay"] * s["mass"] if c["decay"] else 0.0) + got, s["mass"]))
    return {"mass": s["mass"]}


def _plain_evict(s):
    c = s["case"]
    n, keep = c["n"], c["keep"]
    rows = torch.arange(n, device="cuda")
    length = s["lengths"].long()[:, None, None]
    inside, at = rows < length, s["positions"].long()
    newest = torch.where(inside, at, -1).amax(-1, keepdim=True)
    first = (at < c["sinks"]) | (at > newest - c["recent"])
    # by protection, then weight (its bits, of numbers that are not negative), then the lower row; rows that are none come last
    key = torch.where(inside, (first.long() << 32) + s["mass"].view(torch.int32), -1)
    order = torch.sort(key, dim=-1, descending=True, stable=True)[1]
    rank = torch.empty_like(order).scatter_(-1, order, rows.expand_as(order).contiguous())
    stays = length.clamp(max=keep)
    chosen = (rank < stays) & inside
    # the k-th place below that is not of a chosen row takes the k-th chosen row from beyond
    hole, beyond = (rows < stays) & ~chosen, (rows >= stays) & chosen
    moved = torch.sort(torch.where(beyond, rows, n), dim=-1)[0]
    source = torch.where(hole, moved.gather(-1, (hole.long().cumsum(-1) - 1).clamp(min=0)), rows)[..., :keep]
    kept = rows[:keep] < stays
    source = torch.where(kept, source, 0)
    pick = source[..., None].expand(*source.shape, D)
    for t in "KV":
        s[t + "_out"][:, :, :keep] = torch.where(kept[..., None], s[t].gather(2, pick), s[t + "_out"][:, :, :keep])
    for t in ("mass", "positions"):
        s[t + "_out"][:, :, :keep] = torch.where(kept, s[t].gather(2, source), s[t + "_out"][:, :, :keep])
    s["rows"].copy_(torch.where(kept, source, -1))
    return {"K": s["K_out"], "V": s["V_out"], "mass": s["mass_out"], "positions": s["positions_out"], "rows": s["rows"]}


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


def _plain_shared(s):
    c, dt = s["case"], _type(s["case"])
    count, kv, group, m, share, tail = c["count"], c["kv"], c["group"], c["m"], c["share"], c["tail"]
    K, V = ((_from_four_bits(s[t + "_codes"], s[t + "_scales"]) if c["mx"] else s[t].float()) for t in "KV")
    Q = s["Q"].view(count, share, m, kv, group, D).permute(0, 3, 1, 4, 2, 5).float() * D ** -0.5           # [count, kv, share, group, m, 128]
    begin, rows = s["offsets"][:-1].view(count, kv, 1), s["offsets"].diff().view(count, kv, 1)
    j = torch.arange(max(1, s["most"]), device="cuda")
    pick = (begin + j).clamp(max=K.shape[0] - 1).view(-1)
    Kk, Vk = (x[pick].view(count, kv, -1, D) for x in (K, V))
    S = torch.matmul(Q.reshape(count, kv, -1, D), Kk.transpose(-1, -2).contiguous()).masked_fill_((j >= rows)[:, :, None], -math.inf)
    at = s["lengths"].long()[:, None] - m + torch.arange(m, device="cuda")
    hidden = torch.arange(tail, device="cuda") > at[..., None]                                             # [count * share, m, tail]
    Kt, Vt = (x.float().view(count, share, kv, tail, D).transpose(1, 2) for x in (s["K_tail"], s["V_tail"]))
    T = torch.matmul(Q.reshape(count, kv, share, group * m, D), Kt.transpose(-1, -2).contiguous()).view(count, kv, share, group, m, tail)
    T = T.masked_fill_(hidden.view(count, 1, share, 1, m, tail), -math.inf).view(count, kv, -1, tail)
    top = torch.maximum(S.amax(-1, keepdim=True), T.amax(-1, keepdim=True))
    top = torch.where(top == -math.inf, 0.0, top)
    S, T = S.sub_(top).exp_(), T.sub_(top).exp_()
    total = S.sum(-1, keepdim=True) + T.sum(-1, keepdim=True)
    out = torch.matmul(S, Vk) + torch.matmul(T.view(count, kv, share, group * m, tail), Vt.contiguous()).view(count, kv, -1, D)
    out = (out / torch.where(total == 0, 1.0, total)).view(count, kv, share, group, m, D).permute(0, 2, 4, 1, 3, 5)
    lse = (top + total.log()).view(count, kv, share, group, m).transpose(1, 2)
    return {"out": out.reshape(count * share, m, kv * group, D).to(dt), "lse": lse.reshape(count * share, kv * group, m).contiguous()}


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
    if c["op"] == "axes":
        return {"bytes": count * m * (2 * (group + 2) * kv * row + 2 * D // 2 * 4 + 4 * c["axes"]), "flops": count * m * (group + 1) * kv * D * (3 + 4 * c["norm"])}
    lengths = _sequences(c, 0)
    if c["op"] == "weights":
        pairs, keys = _visible(c, lengths)
        return {"bytes": keys * kv * row + count * m * kv * group * (row + 4) + int(lengths.sum()) * kv * (8 if c["decay"] else 4), "flops": 2 * D * pairs * kv * group}
    if c["op"] == "evict":
        kept = np.minimum(lengths, c["keep"])
        moved = (lengths - kept).clip(max=kept) if c["place"] else kept           # (in place: at most as many as leave)
        return {"bytes": kv * (8 * int(lengths.sum()) + 4 * count * c["keep"] + int(kept.sum()) * 8 + int(moved.sum()) * 4 * row), "flops": int(lengths.sum()) * kv}
    kept, tail = int(_budgets(c, 0).sum()), int(lengths.sum()) * kv
    kept_row = D // 2 + D // 32 if c["mx"] else row
    return {"bytes": 2 * kept * kept_row + 2 * tail * row + count * c["share"] * m * kv * group * (2 * row + 4),
            "flops": 4 * D * m * group * (c["share"] * kept + tail)}


# ---- the same in 64 bits ------------------------------------------------------------------------


def _inputs(case, seed):
    """The inputs alone, whatever `own` says."""
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was


def exact(case, seed):
    """The operators from their definitions, head by head and token by token."""
    return {"axes": _exact_axes, "weights": _exact_weights, "evict": _exact_evict, "shared": _exact_shared}[case["op"]](case, seed, _inputs(case, seed))


def _exact_axes(c, seed, given):
    count, kv, group, m = c["count"], c["kv"], c["group"], c["m"]
    Q, K, V = (given[t].double() for t in "QKV")
    Q.zero_()
    half = D // 2
    first = list(range(0, D, 2)) if c["pairs"] else list(range(half))
    second = list(range(1, D, 2)) if c["pairs"] else list(range(half, D))
    table = torch.view_as_complex(given["table"].double().transpose(1, 2).contiguous())                    # e^(i angle) [rows, 64]
    for b in range(count):
        start = int(given["starts"][b])
        z = torch.empty((m, half), dtype=torch.complex128, device="cuda")
        for i, axis in enumerate(given["axis_of"].tolist()):
            z[:, i] = table[:, i].index_select(0, given["positions"][axis, b * m: (b + 1) * m].long())
        x = given["qkv"][b].double().view(m, -1, D)
        for h in range((group + 1) * kv):
            y, query = x[:, h], h < group * kv
            if c["norm"]:
                y = y / (torch.linalg.vector_norm(y, dim=1, keepdim=True) ** 2 / D + EPS).sqrt() * given["qw" if query else "kw"].double()
            w = torch.complex(y[:, first], y[:, second]) * z
            to = Q[b, :, h] if query else K[b, h - group * kv, start: start + m]
            to[:, first], to[:, second] = w.real, w.imag
        V[b, :, start: start + m] = x[:, (group + 1) * kv:].transpose(0, 1)
    return {"Q": Q, "K": K, "V": V}


def _exact_weights(c, seed, given):
    kv, group, m, n = c["kv"], c["group"], c["m"], c["n"]
    if _visible(c, _sequences(c, seed))[0] * kv * group > 2 ** 33:
        return None
    mass = given["mass"].double()
    for b, L in enumerate(_sequences(c, seed).tolist()):
        mass[b, :, :L] *= c["decay"]
        for t0 in range(0, m, 1024):
            t1 = min(m, t0 + 1024)
            low, high = L - m + t0, L - m + t1                         # positions of these tokens
            if high <= 0:
                continue
            j = torch.tensor(sorted(set(range(max(0, low - (c["window"] or n) + 1), high)) | set(range(min(c["sinks"], high)))), device="cuda")
            at = torch.arange(low, high, device="cuda")[:, None]
            unseen = (j > at) | ((at - j >= (c["window"] or n)) & (j >= c["sinks"]))
            for h in range(kv):
                k = given["K"][b, h].index_select(0, j).double()
                for q in range(h * group, (h + 1) * group):
                    x = (given["Q"][b, t0:t1, q].double() @ k.T) / math.sqrt(D) - given["lse"][b, q, t0:t1, None].double()
                    mass[b, h].index_add_(0, j, x.masked_fill_(unseen, -math.inf).exp_().sum(0))
    return {"mass": mass}


def _exact_evict(c, seed, given):
    K, V, mass, at = (given[t].cpu() for t in ("K", "V", "mass", "positions"))
    out = {"K": given["K_out"].cpu().double(), "V": given["V_out"].cpu().double(), "mass": given["mass_out"].cpu().double(),
           "positions": given["positions_out"].cpu().long(), "rows": torch.full(given["rows"].shape, -1, dtype=torch.int64)}
    for b, L in enumerate(_sequences(c, seed).tolist()):
        stays = min(L, c["keep"])
        for h in range(c["kv"]):
            p = at[b, h, :L].numpy().astype(np.int64)
            left = (p >= c["sinks"]) & (p <= p.max(initial=-1) - c["recent"])
            chosen = np.lexsort((np.arange(L), -mass[b, h, :L].numpy().astype(np.float64), left))[:stays]
            here = np.zeros(stays, dtype=np.int64) - 1
            here[chosen[chosen < stays]] = chosen[chosen < stays]
            here[here < 0] = np.sort(chosen[chosen >= stays])
            source = torch.from_numpy(here)
            out["rows"][b, h, :stays] = source
            for name, x in (("K", K), ("V", V), ("mass", mass), ("positions", at)):
                out[name][b, h, :stays] = x[b, h][source].to(out[name].dtype)
    return out


def _exact_shared(c, seed, given):
    count, kv, group, m, share = c["count"], c["kv"], c["group"], c["m"], c["share"]
    off, tails = given["offsets"].tolist(), _sequences(c, seed).tolist()
    if share * m * group * off[-1] > 2 ** 33:
        return None
    levels = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device="cuda")
    out = torch.zeros(given["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(given["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")

    def kept(t, a, z):
        if not c["mx"]:
            return given[t][a:z].double()
        x, e = given[t + "_codes"][a:z].long(), given[t + "_scales"][a:z].double() - 127
        y = torch.empty((z - a, D), dtype=torch.float64, device="cuda")
        for part, code in ((0, x % 16), (1, x // 16)):
            y[:, part::2] = levels[code % 8] * torch.where(code >= 8, -1.0, 1.0)
        return y * torch.repeat_interleave(2.0 ** e, 32, dim=1)

    for b in range(count):
        for h in range(kv):
            a, z = off[b * kv + h], off[b * kv + h + 1]
            common = kept("K", a, z), kept("V", a, z)
            for i in range(b * share, (b + 1) * share):
                L = tails[i]
                k = torch.cat([common[0], given["K_tail"][i, h, :L].double()])
                v = torch.cat([common[1], given["V_tail"][i, h, :L].double()])
                for t in range(m):
                    see = z - a + max(0, L - m + t + 1)
                    if see == 0:
                        continue
                    q = given["Q"][i, t, h * group: (h + 1) * group].double()
                    x = (q @ k[:see].T) / math.sqrt(D)
                    lse[i, h * group: (h + 1) * group, t] = torch.logsumexp(x, 1)
                    out[i, t, h * group: (h + 1) * group] = torch.softmax(x, 1) @ v[:see]
    return {"out": out, "lse": lse}
