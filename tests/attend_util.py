"""Plain 64-bit forms of the operators around a compressed cache, written from their definitions, and the bounds that the kernels'
results are held to.  Not collected by pytest."""

from __future__ import annotations

import math

import numpy as np
import torch

from paper_2509_15038_amd import binding as B
from tests.gpu_util import Guarded

D = 128
LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def dtype_of(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def context(kv, group, dtype, max_tokens=4096):
    return B.Context(1, kv, group, D, 32, dtype, max_tokens, 1)


def randn(seed, shape, dtype, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def attention(q, K, V, seen, scale):
    """One head in 64 bits: q [m, 128], K, V [n, 128], seen [m, n] -> out, lse, sum of weights times |v|, largest sum of |q k| * scale.
    Rows that a token does not see do not enter, whatever they hold."""
    q, K, V = q.double(), K.double(), V.double()
    m = q.shape[0]
    out, mass = torch.zeros((m, D), dtype=torch.float64, device=q.device), torch.zeros((m, D), dtype=torch.float64, device=q.device)
    lse, most = torch.full((m,), -math.inf, dtype=torch.float64, device=q.device), 0.0
    if not m or not bool(seen.any()):
        return out, lse, mass, most
    some = seen.any(0)
    K, V, seen = K[some], V[some], seen[:, some]
    if bool(torch.isfinite(K).all()) and bool(torch.isfinite(V).all()):
        x = ((q @ K.T) * scale).masked_fill(~seen, -math.inf)
        lse = torch.logsumexp(x, 1)
        w = torch.exp(x - torch.where(lse == -math.inf, 0.0, lse)[:, None])
        return w @ V, lse, w @ V.abs(), float((q.abs() @ K.abs().T).max()) * scale
    patterns, which = torch.unique(seen, dim=0, return_inverse=True)
    for u in range(patterns.shape[0]):
        j = patterns[u].nonzero()[:, 0]
        if j.numel() == 0:
            continue
        rows = (which == u).nonzero()[:, 0]
        x = (q[rows] @ K[j].T) * scale
        lse[rows] = torch.logsumexp(x, 1)
        w = torch.exp(x - lse[rows][:, None])
        out[rows], mass[rows] = w @ V[j], w @ V[j].abs()
        most = max(most, float((q[rows].abs() @ K[j].abs().T).max()) * scale)
    return out, lse, mass, most


def check_attention(got, got_lse, want, dtype, keys, where=""):
    """Elementwise.  A bf16 weight (8 bits of significand) is off by 2^-8 of itself and the bf16 result by 2^-8: 2^-7 sum w|v| in all.  In 32 bits a score
    is off by 128 * 2^-24 * sum |q k| at most and the weights by twice that (numerator and sum), the sums of `keys` terms by keys * 2^-24, and
    2^-20 covers the exponentials and the joining of partial results."""
    out, lse, mass, most = want
    score = 128 * 2.0 ** -24 * most
    rel = 2 * score + (keys + 128) * 2.0 ** -24 + 2.0 ** -20 + (2.0 ** -7 * 1.01 if dtype == "bf16" else 2.0 ** -24)
    err = (got.double() - out).abs()
    bad = ~(err <= rel * mass + 1e-30)
    assert not bool(bad.any()), f"{where}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / (mass + 1e-30)).nan_to_num(9e9).max()):.3e} of {rel:.3e}"
    if got_lse is not None:
        empty = lse == -math.inf
        assert bool((got_lse.double()[empty] == -math.inf).all()), where
        e = (got_lse.double()[~empty] - lse[~empty]).abs()
        most_off = score + keys * 2.0 ** -24 + 2.0 ** -20 * (1 + lse[~empty].abs())
        assert bool((e <= most_off).all()), f"{where}: lse off by {float(e.max()):.3e}"


def causal(m, n, length, window, sinks, device="cuda"):
    """seen [m, n] of a sequence's last m tokens."""
    p = (length - m + torch.arange(m, device=device))[:, None]
    j = torch.arange(n, device=device)[None]
    return (j <= p) & (j < length) & ((p - j < window) | (j < sinks) if window else torch.ones_like(j, dtype=torch.bool))


def four_bits(x):
    """Rows [r, 128] -> the values that they are held as (64 bits), codes, scales, by the definition: the nearest level of a block's power of two, ties to the
    even code, NaN for blocks that are not finite."""
    x = x.double().cpu().view(-1, 4, 32)
    top = x.abs().amax(-1)
    finite = torch.isfinite(x).all(-1)
    e = torch.where((top > 0) & finite, torch.frexp(top)[1].double() - 1 - 2, torch.tensor(-127.0, dtype=torch.float64)).clamp(min=-127)
    y = (torch.where(finite[..., None], x, 0.0) * torch.exp2(-e)[..., None])
    levels = torch.tensor(LEVELS, dtype=torch.float64)
    far = (y.abs()[..., None] - levels).abs()
    near = far.amin(-1, keepdim=True)
    tied = far == near
    even = tied & (torch.arange(8) % 2 == 0)
    code = torch.where(even.any(-1), even.int().argmax(-1), tied.int().argmax(-1))
    value = torch.where(finite[..., None], levels[code] * torch.sign(y) * torch.exp2(e)[..., None], math.nan)
    code = torch.where(finite[..., None], code + 8 * (torch.signbit(x) & finite[..., None]).int(), 0).view(-1, 64, 2)
    scale = torch.where(finite, e + 127, 255.0)
    return value.view(-1, D), (code[..., 0] + 16 * code[..., 1]).to(torch.uint8), scale.to(torch.uint8)


def run_attend(case, Q, K, V, lengths, stride):
    """ctx.attend with guarded outputs -> out [count, m, heads, 128], lse [count, heads, m]."""
    c = case
    out = Guarded((c["count"] * c["m"] * c["kv"] * c["group"], D), Q.dtype, float("nan"))
    lse = Guarded((c["count"] * c["kv"] * c["group"], c["m"]), torch.float32, float("nan"))
    with context(c["kv"], c["group"], c["dtype"], max(c["n"], c["m"])) as ctx:
        ctx.attend(Q, K, V, c["count"], c["m"], c["n"], stride, out.t, lengths=lengths, window=c["window"], n_sink=c["sinks"], lse=lse.t)
        torch.cuda.synchronize()
    out.check("out")
    lse.check("lse")
    return out.t.view(c["count"], c["m"], -1, D), lse.t.view(c["count"], -1, c["m"])


def check_attend(case, seed=0, spoil=None, stride=None, lengths="ragged"):
    """A case on random inputs against the 64-bit form, every head.  Rows beyond a sequence's length hold NaN; spoil(K, V, lengths) may do more."""
    c = dict(dict(count=1, kv=2, group=4, m=1, n=1, window=0, sinks=0, dtype="bf16"), **case)
    dt, n, m = dtype_of(c["dtype"]), c["n"], c["m"]
    stride = n if stride is None else stride
    K, V = (randn(seed + i, (c["count"], c["kv"], stride, D), dt) for i in (1, 2))
    K *= torch.exp(0.5 * randn(seed + 4, (c["count"], c["kv"], 1, D), torch.float32)).to(dt)
    Q = randn(seed + 3, (c["count"], m, c["kv"] * c["group"], D), dt)
    rng = np.random.default_rng(seed)
    if isinstance(lengths, str):
        lens = np.full(c["count"], n) if lengths == "full" else np.concatenate([[n], rng.integers(0, n + 1, c["count"] - 1)])
    else:
        lens = np.asarray(lengths)
    for b in range(c["count"]):
        K[b, :, int(lens[b]):], V[b, :, int(lens[b]):] = math.nan, math.inf
    if spoil:
        spoil(K, V, lens)
    given = None if isinstance(lengths, str) and lengths == "full" else torch.from_numpy(lens.astype(np.int32)).cuda()
    out, lse = run_attend(c, Q, K, V, given, stride)
    for b in range(c["count"]):
        seen = causal(m, n, int(lens[b]), c["window"], c["sinks"])
        for h in range(c["kv"] * c["group"]):
            k, v = K[b, h // c["group"], :n], V[b, h // c["group"], :n]
            want = attention(Q[b, :, h], k, v, seen, D ** -0.5)
            check_attention(out[b, :, h], lse[b, h], want, c["dtype"], n, f"{c} seq {b} of {int(lens[b])}, head {h}")
    return out, lse
