"""Attention over a cache (curdkv_attend) against its definition in 64 bits: prompts and single tokens, windows and sinks, ragged lengths, rows
that see nothing, what lies in hidden rows, strides, streams, graphs, refusals."""

import math

import numpy as np
import pytest
import torch

from paper_2509_15038_amd import binding as B
from tests import attend_util as U

pytestmark = pytest.mark.gpu
D = 128


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 255, 257, 1000, 4099])
def test_single_tokens(dtype, n):
    U.check_attend(dict(count=3, m=1, n=n, dtype=dtype), seed=n)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 64, 65, 100, 255, 256, 257, 513, 1021])
def test_prompts(dtype, n):
    U.check_attend(dict(count=2, m=n, n=n, dtype=dtype), seed=n, lengths="full")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kv,group", [(1, 1), (1, 3), (2, 5), (1, 7), (3, 8), (1, 16), (1, 20), (2, 40)])
@pytest.mark.parametrize("m", [1, 2, 37])
def test_head_layouts(dtype, kv, group, m):
    U.check_attend(dict(count=2, kv=kv, group=group, m=m, n=301, dtype=dtype), seed=kv * group + m)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m", [1, 3, 130, 400])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 4), (16, 4), (63, 0), (64, 4), (65, 64), (100, 350), (399, 4), (400, 4), (401, 0), (5000, 4)])
def test_windows(dtype, m, window, sinks):
    U.check_attend(dict(count=3, m=m, n=400, window=window, sinks=sinks, dtype=dtype), seed=window + m)


@pytest.mark.parametrize("m,n,window,sinks", [(130, 130, 0, 0), (300, 300, 77, 5), (129, 400, 50, 64), (200, 333, 0, 0)])
def test_many_heads_in_fp32(m, n, window, sinks):
    # enough rows for the kernel of prompts
    U.check_attend(dict(count=3, kv=100, group=1, m=m, n=n, window=window, sinks=sinks, dtype="fp32"), seed=m, lengths=[n, n - 1, m // 2])


@pytest.mark.parametrize("spoiled", [False, True])
def test_many_heads_in_fp32_and_values_that_are_not_finite(spoiled):
    def spoil(K, V, lens):
        if spoiled:
            V[:, ::2, -1, 3], V[:, ::3, -1, 100], V[:, 1, 140] = math.nan, math.inf, -math.inf

    m, n = 150, 260
    K, V, Q = (U.randn(i, (2, 100, n, D) if i < 3 else (2, m, 200, D), torch.float32) for i in (1, 2, 3))
    spoil(K, V, None)
    out, lse = U.run_attend(dict(count=2, kv=100, group=2, m=m, n=n, window=0, sinks=0, dtype="fp32"), Q, K, V, None, n)
    for b in range(2):
        seen = U.causal(m, n, n, 0, 0)
        for h in range(0, 200, 3):
            k, v = K[b, h // 2], V[b, h // 2]
            fine = ~(seen & ~torch.isfinite(v).all(1)).any(1)
            U.check_attention(out[b, fine, h], lse[b, h, fine], U.attention(Q[b, fine, h], k, v, seen[fine], D ** -0.5), "fp32", n, f"head {h}")
            bad = ~torch.isfinite(v)
            got = out[b, -1, h]
            assert bool((torch.isfinite(got) == ~bad.any(0)).all())


@pytest.mark.parametrize("count,m,n,window,sinks", [(1, 12, 16000, 0, 0), (1, 40, 9001, 0, 0), (2, 33, 5000, 3000, 4), (1, 100, 4000, 0, 0), (3, 20, 2500, 0, 0), (1, 300, 3000, 2000, 100)])
def test_a_few_tokens_over_long_caches(count, m, n, window, sinks):
    # the tiles of keys of one row tile shared out over several workgroups
    U.check_attend(dict(count=count, kv=2, group=4, m=m, n=n, window=window, sinks=sinks), seed=m, lengths=[n, m + 3, 5][:count])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m", [1, 5, 64, 200])
def test_sequences_shorter_than_their_new_tokens(dtype, m):
    # the first m - length tokens stand before the sequence and see nothing: zeros and -infinity
    lengths = [0, 1, m - 1, m, max(0, m - 3)]
    out, lse = U.check_attend(dict(count=5, m=m, n=200, dtype=dtype, window=50, sinks=2), seed=m, lengths=lengths)
    for b, L in enumerate(lengths):
        none = max(0, m - L)
        assert bool((out[b, :none] == 0).all()) and bool((lse[b, :, :none] == -math.inf).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m", [1, 4, 7, 96, 300])
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 3)])
def test_infinities_and_nan_in_hidden_rows(dtype, m, window, sinks):
    # the last rows hold NaN and infinities: tokens before them must not notice; nor may those out of whose window bad rows have moved
    def spoil(K, V, lens):
        for b, L in enumerate(lens.tolist()):
            if m > 1 and L >= 2:
                K[b, :, L - 1], V[b, :, L - 1] = math.nan, math.nan
            if m > 2 and L >= m:
                V[b, 0, L - 2, 5], V[b, 0, L - 2, 77] = math.inf, -math.inf
            if window and L > window + m + sinks:
                K[b, :, sinks: L - window - m + 1], V[b, :, sinks: L - window - m + 1] = math.inf, math.nan

    c = dict(count=2, kv=2, group=4, m=m, n=300, window=window, sinks=sinks, dtype=dtype)
    dt = U.dtype_of(dtype)
    K, V = (U.randn(i, (2, 2, 300, D), dt) for i in (1, 2))
    Q = U.randn(3, (2, m, 8, D), dt)
    lens = np.array([300, 300])
    spoil(K, V, lens)
    out, lse = U.run_attend(c, Q, K, V, None, 300)
    for b in range(2):
        seen = U.causal(m, 300, 300, window, sinks)
        for h in range(8):
            k, v = K[b, h // 4], V[b, h // 4]
            fine = ~(seen & ~(torch.isfinite(k.float()).all(1) & torch.isfinite(v.float()).all(1))).any(1)
            if m > 2:
                assert int(fine.sum()) == m - 2 if h < 4 else m - 1
            want = U.attention(Q[b, fine, h], k, v, seen[fine], D ** -0.5)
            U.check_attention(out[b, fine, h], lse[b, h, fine], want, dtype, 300, f"m {m} head {h}")
            if m > 1:
                assert bool(torch.isnan(out[b, -1, h]).all())       # the token that sees them does


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m", [1, 70])
def test_strides_and_large_offsets(dtype, m):
    U.check_attend(dict(count=2, kv=2, m=m, n=150, dtype=dtype), stride=1000)
    # heads more than 2^31 elements apart: only the rows that are looked at are written
    kv, n, dt = 3, 99, U.dtype_of(dtype)
    stride = (2 ** 31 // D if dtype == "bf16" else 2 ** 30 // D) + 5
    K, V = (torch.empty((kv, stride, D), dtype=dt, device="cuda") for _ in range(2))
    K[:, :n], V[:, :n] = U.randn(1, (kv, n, D), dt), U.randn(2, (kv, n, D), dt)
    Q = U.randn(3, (1, m, kv * 2, D), dt)
    out, lse = U.run_attend(dict(count=1, kv=kv, group=2, m=m, n=n, window=0, sinks=0, dtype=dtype), Q, K, V, None, stride)
    for h in range(kv * 2):
        want = U.attention(Q[0, :, h], K[h // 2, :n], V[h // 2, :n], U.causal(m, n, n, 0, 0), D ** -0.5)
        U.check_attention(out[0, :, h], lse[0, h], want, dtype, n)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m", [1, 100])
@pytest.mark.parametrize("gain", [1e-3, 30.0])
def test_flat_and_peaked_scores(dtype, m, gain):
    # all scores nearly equal, and one weight that is nearly all: the running maximum moves late and far
    n, dt = 2000, U.dtype_of(dtype)
    K, V = U.randn(1, (1, 1, n, D), dt), U.randn(2, (1, 1, n, D), dt)
    K *= torch.linspace(0.1, 1, n, device="cuda").to(dt)[None, None, :, None]
    Q = U.randn(3, (1, m, 2, D), dt, gain)
    out, lse = U.run_attend(dict(count=1, kv=1, group=2, m=m, n=n, window=0, sinks=0, dtype=dtype), Q, K, V, None, n)
    for h in range(2):
        want = U.attention(Q[0, :, h], K[0, 0], V[0, 0], U.causal(m, n, n, 0, 0), D ** -0.5)
        U.check_attention(out[0, :, h], lse[0, h], want, dtype, n)


@pytest.mark.parametrize("m,n,window", [(1, 5000, 0), (1, 5000, 700), (600, 600, 0)])
def test_same_bits_every_time_on_another_stream_and_in_a_graph(m, n, window):
    K, V, Q = U.randn(1, (2, 2, n, D), torch.bfloat16), U.randn(2, (2, 2, n, D), torch.bfloat16), U.randn(3, (2, m, 8, D), torch.bfloat16)
    with U.context(2, 4, "bf16", n) as ctx:
        outs = [torch.empty_like(Q) for _ in range(3)]
        call = lambda o, s=None: ctx.attend(Q, K, V, 2, m, n, n, o, window=window, n_sink=4, stream=s)
        call(outs[0])
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        call(outs[1], side)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(outs[2])
        for k in range(3):
            Q.copy_(U.randn(10 + k, Q.shape, torch.bfloat16))
            graph.replay()
            torch.cuda.synchronize()
            call(outs[0])
            torch.cuda.synchronize()
            assert torch.equal(outs[0], outs[2]), k


def test_lse_is_optional_and_lengths_are_clamped():
    K, V, Q = U.randn(1, (2, 1, 50, D), torch.bfloat16), U.randn(2, (2, 1, 50, D), torch.bfloat16), U.randn(3, (2, 1, 4, D), torch.bfloat16)
    with U.context(1, 4, "bf16", 64) as ctx:
        a, b = torch.empty_like(Q), torch.empty_like(Q)
        ctx.attend(Q, K, V, 2, 1, 50, 50, a, lengths=torch.tensor([10 ** 6, -5], dtype=torch.int32, device="cuda"))
        ctx.attend(Q, K, V, 2, 1, 50, 50, b, lengths=torch.tensor([50, 0], dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
    assert torch.equal(a, b) and bool((a[1] == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m", [1, 3, 50])
def test_less_scratch_and_none(dtype, m):
    # fewer workgroups share a head; the counters at its start are left cleared
    n, dt = 5000, U.dtype_of(dtype)
    K, V, Q = U.randn(1, (2, 2, n, D), dt), U.randn(2, (2, 2, n, D), dt), U.randn(3, (2, m, 8, D), dt)
    with U.context(2, 4, dtype, n) as ctx:
        for size in (0, 16, 16384, 16384 + 520 * 40, 16384 + 520 * 700, 16384 + 520 * 5000):
            out = torch.full_like(Q, float("nan"))
            scratch = torch.zeros((max(size, 16),), dtype=torch.uint8, device="cuda")[:size]
            guard = torch.full((4096,), 77, dtype=torch.uint8, device="cuda")
            ctx.attend(Q, K, V, 2, m, n, n, out, scratch=scratch)
            torch.cuda.synchronize()
            assert bool((scratch[:16384] == 0).all()) and bool((guard == 77).all())
            for h in (0, 7):
                want = U.attention(Q[1, :, h], K[1, h // 4], V[1, h // 4], U.causal(m, n, n, 0, 0), D ** -0.5)
                U.check_attention(out[1, :, h], None, want, dtype, n, f"scratch {size}")


def test_refusals():
    K, V, Q = U.randn(1, (1, 1, 50, D), torch.bfloat16), U.randn(2, (1, 1, 50, D), torch.bfloat16), U.randn(3, (1, 2, 4, D), torch.bfloat16)
    out = torch.full_like(Q, 7.0)
    good = dict(Q=Q, K=K, V=V, count=1, m=2, n=50, stride=50, out=out)
    with U.context(1, 4, "bf16", 64) as ctx:
        for bad in (dict(Q=None), dict(K=None), dict(V=None), dict(out=None), dict(count=0), dict(m=0), dict(n=0), dict(n=51), dict(n=65, stride=65),
                    dict(stride=49), dict(window=-1), dict(n_sink=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf),
                    dict(scratch=torch.zeros(64, dtype=torch.uint8, device="cuda")[8:]), dict(Q=Q.data_ptr() + 2), dict(K=K.data_ptr() + 8), dict(out=out.data_ptr() + 4), dict(m=65)):
            with pytest.raises(B.CurdkvError) as e:
                ctx.attend(**dict(good, **bad))
            assert e.value.code == B.ERR_INVALID_ARG, bad
        with pytest.raises(B.CurdkvError) as e:
            ctx.attend(**dict(good, count=2 ** 31))
        assert e.value.code == B.ERR_UNSUPPORTED
        torch.cuda.synchronize()
        assert bool((out == 7).all())
