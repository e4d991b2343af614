"""Attention where tokens see keys whose scores are not finite: keys of score -infinity weigh nothing, wherever they lie and whichever kernel takes them, and
NaN is NaN in the log-sum too."""

import math

import pytest
import torch

from tests import attend_util as U

pytestmark = pytest.mark.gpu
D = 128

# (count, kv, m, n, window, sinks), four query heads a KV head: a workgroup a head; workgroups of their own for each head; equal shares of all heads; a few tokens with
# masks; the prompts' kernels, in bf16 and in fp32 (four waves and eight), without and with parts of the keys; windows behind first rows
SHAPES = [(3, 2, 1, 300, 0, 0), (1, 2, 1, 5000, 0, 0), (65, 2, 1, 2200, 0, 0), (2, 2, 5, 300, 0, 0), (1, 4, 700, 700, 0, 0), (1, 2, 300, 5000, 0, 0), (6, 8, 100, 300, 0, 0),
          (24, 8, 520, 520, 0, 0), (2, 4, 700, 700, 90, 70), (2, 2, 3, 3000, 500, 70)]


def inputs(dtype, count, kv, m, n, first, kind):
    """Queries whose channel 5 is positive, keys of which the first `first` of every head score -infinity by it: an infinite key, or a finite one whose product is
    beyond the type's range."""
    dt = U.dtype_of(dtype)
    Q, K, V = U.randn(1, (count, m, kv * 4, D), dt), U.randn(2, (count, kv, n, D), dt), U.randn(3, (count, kv, n, D), dt)
    Q[..., 5] = Q[..., 5].abs() + 10
    K[..., 5] *= 0.1
    K[:, :, :first, 5] = -math.inf if kind == "infinite" else -3e38
    return Q, K, V


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["infinite", "beyond the range"])
@pytest.mark.parametrize("first", [1, 16, 67, 200])
@pytest.mark.parametrize("count,kv,m,n,window,sinks", SHAPES)
def test_first_keys_that_weigh_nothing(dtype, kind, first, count, kv, m, n, window, sinks):
    Q, K, V = inputs(dtype, count, kv, m, n, first, kind)
    out, lse = U.run_attend(dict(count=count, kv=kv, group=4, m=m, n=n, window=window, sinks=sinks, dtype=dtype), Q, K, V, None, n)
    seen = U.causal(m, n, n, window, sinks)
    seen[:, :first] = False                                             # (a token that sees no others: zeros and -infinity, as one that sees nothing)
    for b, h in {(0, 0), (0, kv * 4 - 1), (count - 1, 1)}:
        want = U.attention(Q[b, :, h], K[b, h // 4], V[b, h // 4], seen, D ** -0.5)
        U.check_attention(out[b, :, h], lse[b, h], want, dtype, n, f"seq {b} head {h}")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("first,every", [(0, 16), (32, 64), (64, 128), (5, 16)])
@pytest.mark.parametrize("m,n", [(1, 600), (1, 5000), (700, 700)])
def test_keys_that_weigh_nothing_between_others(dtype, first, every, m, n):
    Q, K, V = inputs(dtype, 1, 4, m, n, 0, "infinite")
    none = (torch.arange(n, device="cuda") - first) % every < every // 2
    K[:, :, none, 5] = -math.inf
    out, lse = U.run_attend(dict(count=1, kv=4, group=4, m=m, n=n, window=0, sinks=0, dtype=dtype), Q, K, V, None, n)
    seen = U.causal(m, n, n, 0, 0) & ~none
    for h in (0, 15):
        want = U.attention(Q[0, :, h], K[0, h // 4], V[0, h // 4], seen, D ** -0.5)
        U.check_attention(out[0, :, h], lse[0, h], want, dtype, n, f"head {h}")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m", [1, 400])
@pytest.mark.parametrize("first", [64, 130, 400])
def test_first_kept_rows_that_weigh_nothing(dtype, m, first):
    kv, kept, tail = 8, 400, 400
    Q, K, V = inputs(dtype, 1, kv, m, kept, first, "infinite")
    _, Kt, Vt = inputs(dtype, 1, kv, m, tail, 0, "infinite")
    out, lse = torch.empty_like(Q), torch.empty((kv * 4, m), device="cuda")
    offsets = torch.arange(kv + 1, device="cuda") * kept
    with U.context(kv, 4, dtype, tail) as ctx:
        ctx.attend_kept(Q, K, V, offsets, 1, m, kv * kept, out, K_tail=Kt, V_tail=Vt, tail_n=tail, tail_stride=tail, lse=lse)
        torch.cuda.synchronize()
    seen = torch.cat([torch.ones((m, kept), dtype=torch.bool, device="cuda"), U.causal(m, tail, tail, 0, 0)], 1)
    seen[:, :first] = False
    for h in (0, 31):
        k, v = torch.cat([K[0, h // 4], Kt[0, h // 4]]), torch.cat([V[0, h // 4], Vt[0, h // 4]])
        want = U.attention(Q[0, :, h], k, v, seen, D ** -0.5)
        U.check_attention(out[0, :, h], lse[h], want, dtype, kept + tail, f"head {h}")


def test_first_rows_of_4_bits_that_weigh_nothing():
    # the largest values that 4 bits stand for: their products with the queries are beyond the range
    kv, kept, first = 2, 3000, 700
    Q, K, V = inputs("bf16", 1, kv, 1, kept, first, "beyond the range")
    codes = [torch.empty((kv * kept, w), dtype=torch.uint8, device="cuda") for w in (64, 4, 64, 4)]
    indices, offsets = torch.arange(kept, dtype=torch.int32, device="cuda").repeat(kv), torch.arange(kv + 1, device="cuda") * kept
    out, lse = torch.empty_like(Q), torch.empty((kv * 4, 1), device="cuda")
    held = [torch.empty((kv * kept, D), dtype=torch.bfloat16, device="cuda") for _ in "KV"]
    with U.B.Context(1, kv, 4, D, 32, "bf16", kept, 1) as ctx:
        ctx.compact_mx(K, V, kept, indices, offsets, kv * kept, *codes)
        ctx.attend_kept_mx(Q, *codes, offsets, 1, 1, kv * kept, out, lse=lse)
        for x, c in zip(held, (codes[:2], codes[2:])):
            ctx.expand_mx(*c, kv * kept, x)
        torch.cuda.synchronize()
    seen = torch.arange(kept, device="cuda")[None] >= first
    for h in range(8):
        k, v = (x.view(kv, kept, D)[h // 4] for x in held)
        U.check_attention(out[0, :, h], lse[h], U.attention(Q[0, :, h], k, v, seen, D ** -0.5), "bf16", kept, f"head {h}")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("count,kv,m,n,window,sinks", SHAPES)
def test_a_query_of_nan(dtype, count, kv, m, n, window, sinks):
    # its token has NaN, in the log-sum too, and no other
    Q, K, V = inputs(dtype, count, kv, m, n, 0, "infinite")
    t = m // 2
    Q[:, t, 1, 77] = math.nan
    out, lse = U.run_attend(dict(count=count, kv=kv, group=4, m=m, n=n, window=window, sinks=sinks, dtype=dtype), Q, K, V, None, n)
    assert bool(torch.isnan(out[:, t, 1]).all()) and bool(torch.isnan(lse[:, 1, t]).all())
    assert int(torch.isnan(out).sum()) == count * D and int(torch.isnan(lse).sum()) == count
    assert not bool(torch.isinf(lse).any())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("count,kv,m,n,window,sinks", SHAPES)
def test_nothing_but_keys_of_nan(dtype, count, kv, m, n, window, sinks):
    # a token that sees something has NaN, one before the sequence's first zeros and -infinity; other heads are right
    Q, K, V = inputs(dtype, count, kv, m, n, 0, "infinite")
    K[:, 0] = math.nan
    length = n if m == 1 else m - 1
    lengths = torch.full((count,), length, dtype=torch.int32, device="cuda")
    out, lse = U.run_attend(dict(count=count, kv=kv, group=4, m=m, n=n, window=window, sinks=sinks, dtype=dtype), Q, K, V, lengths, n)
    none = m - min(m, length)
    assert bool(torch.isnan(out[:, none:, :4]).all()) and bool(torch.isnan(lse[:, :4, none:]).all())
    assert bool((out[:, :none] == 0).all()) and bool((lse[:, :, :none] == -math.inf).all())
    seen = U.causal(m, n, length, window, sinks)
    want = U.attention(Q[-1, :, 5], K[-1, 1], V[-1, 1], seen, D ** -0.5)
    U.check_attention(out[-1, :, 5], lse[-1, 5], want, dtype, n)


@pytest.mark.parametrize("dtype,mx", [("bf16", False), ("fp32", False), ("bf16", True), ("fp32", True)])
@pytest.mark.parametrize("m", [1, 400])
def test_a_query_of_nan_over_kept_rows(dtype, mx, m):
    kv, kept = 8, 500
    Q, K, V = inputs(dtype, 1, kv, m, kept, 0, "infinite")
    Q[0, 0, 2, 9] = math.nan
    out, lse = torch.empty_like(Q), torch.empty((kv * 4, m), device="cuda")
    offsets = torch.arange(kv + 1, device="cuda") * kept
    with U.B.Context(1, kv, 4, D, 32, dtype, kept, 1) as ctx:
        if mx:
            codes = [torch.empty((kv * kept, w), dtype=torch.uint8, device="cuda") for w in (64, 4, 64, 4)]
            ctx.compact_mx(K, V, kept, torch.arange(kept, dtype=torch.int32, device="cuda").repeat(kv), offsets, kv * kept, *codes)
            ctx.attend_kept_mx(Q, *codes, offsets, 1, m, kv * kept, out, lse=lse)
        else:
            ctx.attend_kept(Q, K, V, offsets, 1, m, kv * kept, out, lse=lse)
        torch.cuda.synchronize()
    assert bool(torch.isnan(out[0, 0, 2]).all()) and bool(torch.isnan(lse[2, 0])) and int(torch.isnan(out).sum()) == D and int(torch.isnan(lse).sum()) == 1
    assert not bool(torch.isinf(lse).any())
