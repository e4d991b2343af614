"""The attention weight that cached keys got (curdkv_attend_weights) against its definition in 64 bits."""

import math

import numpy as np
import pytest
import torch

from paper_2509_15038_amd import binding as B
from tests import attend_util as U
from tests.gpu_util import Guarded

pytestmark = pytest.mark.gpu
D = 128


def lse_of(q, k, seen, scale):
    """One head in 64 bits: [m]; -infinity where a token sees nothing."""
    x = ((q.double() @ k.double().T) * scale).masked_fill(~seen, -math.inf)
    return torch.logsumexp(x, 1)


def check(dtype, count=1, kv=2, group=4, m=1, n=1, window=0, sinks=0, decay=1.0, lengths="ragged", stride=None, mass_stride=None, scale=D ** -0.5, seed=0, spoil=None,
          stream=None, scratch=None):
    dt = U.dtype_of(dtype)
    stride, mass_stride = n if stride is None else stride, n if mass_stride is None else mass_stride
    K = U.randn(seed + 1, (count, kv, stride, D), dt) * torch.exp(0.5 * U.randn(seed + 4, (count, kv, 1, D), torch.float32)).to(dt)
    Q = U.randn(seed + 3, (count, m, kv * group, D), dt)
    rng = np.random.default_rng(seed)
    if isinstance(lengths, str):
        lens = np.full(count, n) if lengths == "full" else np.concatenate([[n], rng.integers(0, n + 1, count - 1)])
    else:
        lens = np.asarray(lengths)
    lse = torch.empty((count, kv * group, m), device="cuda")
    for b in range(count):
        seen = U.causal(m, n, int(lens[b]), window, sinks)
        for h in range(kv * group):
            lse[b, h] = lse_of(Q[b, :, h], K[b, h // group, :n].nan_to_num(0, 0, 0), seen, scale).float()
        K[b, :, int(lens[b]):] = math.nan
    if spoil:
        spoil(Q, K, lse)
    old = torch.exp(U.randn(seed + 5, (count, kv, mass_stride), torch.float32))
    mass = Guarded((count * kv, mass_stride), torch.float32, float("nan"))
    mass.t.copy_(old.view(count * kv, -1) if decay else torch.full_like(mass.t, float("nan")))
    given = None if isinstance(lengths, str) and lengths == "full" else torch.from_numpy(lens.astype(np.int32)).cuda()
    with U.context(kv, group, dtype, max(n, m)) as ctx:
        ctx.attend_weights(Q, K, lse, count, m, n, stride, mass.t, mass_stride=mass_stride, lengths=given, window=window, n_sink=sinks, scale=scale, decay=decay,
                           scratch=scratch, stream=stream)
        torch.cuda.synchronize()
    mass.check("mass")
    got = mass.t.view(count, kv, mass_stride)
    for b in range(count):
        L = int(lens[b])
        rest = got[b, :, L:]
        assert torch.equal(rest, old[b, :, L:]) if decay else bool(rest.isnan().all()), f"rows behind {L} of sequence {b}"
        seen = U.causal(m, n, L, window, sinks)[:, :L]
        for h in range(kv):
            want = torch.zeros(L, dtype=torch.float64, device="cuda")
            off = torch.zeros(L, dtype=torch.float64, device="cuda")
            for i in range(group):
                q, k, z = Q[b, :, h * group + i].double(), K[b, h, :L].double(), lse[b, h * group + i].double()[:, None]
                x = (q @ k.T) * scale
                there = seen & (z != -math.inf)
                w = torch.where(there, torch.exp(torch.where(there, x - z, 0.0)), 0.0)
                want += w.sum(0)
                # a score: 128 products and sums, or what is left out of a product in parts, each below 2^-22; the difference from lse in units of log 2, four roundings of either
                # term; the exponential 2^-22; m * group summands
                size = (q.abs() @ k.abs().T) * scale
                rel = 128 * 2.0 ** -24 * size + 4 * 2.0 ** -24 * (x.abs() + z.abs()) + 2.0 ** -22
                off += torch.where(w > 0, w * rel, 0.0).sum(0)         # (no weight, as under an lse of +infinity: exactly 0)
            off += want * (m * group + 4) * 2.0 ** -24
            total = want + (decay * old[b, h, :L].double() if decay else 0.0)
            bound = off + (2 * 2.0 ** -24 * decay * old[b, h, :L].double() if decay else 0.0) + 2.0 ** -24 * total + 1e-35
            err = (got[b, h, :L].double() - total).abs()
            same = torch.isnan(total) & torch.isnan(got[b, h, :L])
            bad = ~((err <= bound) | same | (total == got[b, h, :L].double()))
            assert not bool(bad.any()), f"sequence {b} of {L}, head {h}: {int(bad.sum())} of {L} off, first at {int(bad.nonzero()[0])}, worst {float((err / bound)[~same].max()):.2f} of the bound"
    return got


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kv,group", [(1, 1), (8, 4), (2, 7), (3, 5), (1, 16), (1, 40)])
@pytest.mark.parametrize("m,n", [(1, 1), (1, 130), (2, 65), (5, 33), (17, 17)])
def test_layouts_and_sizes(dtype, kv, group, m, n):
    check(dtype, 3, kv, group, m, n)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m,n", [(64, 64), (200, 200), (257, 257), (511, 600), (1000, 1000), (33, 1500), (128, 129), (600, 100)])
def test_prompts_and_their_last_tokens(dtype, m, n):
    check(dtype, 2, 2, 4, m, n, decay=0.0, seed=m)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 4), (7, 1), (64, 0), (100, 64), (300, 500), (10 ** 6, 3), (0, 5)])
@pytest.mark.parametrize("m", [1, 40, 513])
def test_windows(dtype, window, sinks, m):
    check(dtype, 2, 1, 4, m, 513, window, sinks, decay=0.5, seed=window + sinks)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_lengths(dtype):
    for m in (1, 3, 70):
        check(dtype, 6, 2, 4, m, 200, lengths=[0, 1, 2, 69, 199, 200])
        check(dtype, 6, 2, 4, m, 200, lengths=[0, 1, 2, 69, 199, 200], decay=0.0, window=50, sinks=2)
    check(dtype, 2, 2, 4, 3, 100, lengths="full")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_strides(dtype):
    check(dtype, 2, 2, 3, 4, 100, stride=137, mass_stride=101)
    check(dtype, 2, 2, 3, 90, 100, stride=100, mass_stride=333, decay=0.0)


def test_lengths_outside_the_cache_are_clamped():
    Q, K = U.randn(1, (2, 1, 2, D), torch.bfloat16), U.randn(2, (2, 1, 40, D), torch.bfloat16)
    mass = torch.zeros((2, 1, 40), device="cuda")
    lse = torch.zeros((2, 2, 1), device="cuda")
    with U.context(1, 2, "bf16", 40) as ctx:
        ctx.attend_weights(Q, K, lse, 2, 1, 40, 40, mass, lengths=torch.tensor([-3, 99], dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
    assert bool((mass[0] == 0).all()) and bool((mass[1] > 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m", [1, 300])
def test_what_is_not_finite(dtype, m):
    # a NaN key is its own affair; a token whose lse is NaN spoils the keys that it sees; one whose lse is -infinity gives nothing, +infinity neither
    def spoil(Q, K, lse):
        K[0, 0, 5, 3] = math.nan
        lse[0, 1, 0] = -math.inf
        lse[0, 4, m - 1] = math.inf
    got = check(dtype, 1, 2, 4, m, 300, seed=3, spoil=spoil)
    assert bool(got[0, 0, 5].isnan()) and int(got.isnan().sum()) == 1

    def nan_token(Q, K, lse):
        lse[0, 4, m // 2] = math.nan                                   # (query head 0 of KV head 1)
    got = check(dtype, 1, 2, 4, m, 300, seed=4, spoil=nan_token)
    assert int(got[0, 1].isnan().sum()) == 300 - m + m // 2 + 1 and not bool(got[0, 0].isnan().any())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m", [1, 200])
def test_infinite_keys(dtype, m):
    # a key that scores -infinity has no weight; the queries are positive where it is infinite
    def spoil(Q, K, lse):
        Q[..., 7] = Q[..., 7].abs() + 0.1
        K[0, 0, 3, 7] = -math.inf
        x = (Q[0].double().transpose(0, 1) @ K[0, 0].nan_to_num(0, 0, 0).double().T) * D ** -0.5      # (any lse will do)
        lse[0] = torch.logsumexp(x, -1).float()
    got = check(dtype, 1, 1, 4, m, 200, seed=5, spoil=spoil, decay=0.0)
    assert float(got[0, 0, 3]) == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_with_the_attention_that_writes_lse(dtype):
    # every row's weights sum to 1: the mass of a call to the number of rows that see something
    for m, n, window, sinks in ((1, 700, 0, 0), (64, 700, 0, 0), (700, 700, 0, 0), (700, 700, 100, 4)):
        dt = U.dtype_of(dtype)
        Q, K, V = U.randn(1, (2, m, 8, D), dt), U.randn(2, (2, 2, n, D), dt), U.randn(3, (2, 2, n, D), dt)
        lengths = torch.tensor([n, n // 2], dtype=torch.int32, device="cuda")
        out, lse, mass = torch.empty_like(Q), torch.empty((2, 8, m), device="cuda"), torch.zeros((2, 2, n), device="cuda")
        with U.context(2, 4, dtype, n) as ctx:
            ctx.attend(Q, K, V, 2, m, n, n, out, lengths=lengths, window=window, n_sink=sinks, lse=lse)
            ctx.attend_weights(Q, K, lse, 2, m, n, n, mass, lengths=lengths, window=window, n_sink=sinks)
            torch.cuda.synchronize()
        for b, L in enumerate((n, n // 2)):
            rows = 4 * min(m, L)
            # lse is within 128 * 2^-24 * sum |q k| + (n + 20 * 14) 2^-24 of what it is (|q k| below 60 here), scores as much
            assert bool(((mass[b].double().sum(-1) - rows).abs() <= rows * 2 * (128 * 60 + n + 512) * 2.0 ** -24).all()), (m, n, b)
            assert bool((mass[b, :, L:] == 0).all())


def test_results_do_not_change_from_run_to_run_and_graphs_replay():
    for dtype, m, n in (("bf16", 1, 3000), ("bf16", 900, 900), ("fp32", 300, 300)):
        dt = U.dtype_of(dtype)
        Q, K = U.randn(1, (2, m, 8, D), dt), U.randn(2, (2, 2, n, D), dt)
        lse = torch.full((2, 8, m), 9.0, device="cuda")
        lengths = torch.tensor([n, n], dtype=torch.int32, device="cuda")
        mass = torch.zeros((2, 2, n), device="cuda")
        with U.context(2, 4, dtype, n) as ctx:
            def step():
                ctx.attend_weights(Q, K, lse, 2, m, n, n, mass, lengths=lengths, decay=0.5)
            wants = []
            for few in (n, n // 3):
                lengths.fill_(few)
                mass.zero_()
                for _ in range(3):
                    step()
                    wants.append(mass.clone())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
            for turn, few in enumerate((n, n // 3)):
                lengths.fill_(few)
                mass.zero_()
                for i in range(3):
                    graph.replay()
                    torch.cuda.synchronize()
                    assert torch.equal(mass, wants[3 * turn + i]), (dtype, m, few, i)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_scratch_that_holds_something(dtype):
    # partial sums of other calls lie in scratch: short sequences among long ones, for which there are more shares than products
    scratch = torch.zeros((B.ATTEND_SCRATCH_BYTES,), dtype=torch.uint8, device="cuda")
    scratch[16384:].view(torch.float32).fill_(1e9)
    for m, n in ((300, 300), (700, 700), (64, 1500)):
        check(dtype, 3, 2, 4, m, n, lengths=[n, n // 3, 40], decay=0.0, scratch=scratch)
        check(dtype, 3, 2, 4, m, n, lengths=[65, 1, 0], window=50, sinks=2, scratch=scratch)


def test_another_stream():
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    scratch = torch.zeros((0,), dtype=torch.uint8, device="cuda")
    check("bf16", 2, 2, 4, 100, 300, stream=side, scratch=scratch)


@pytest.mark.parametrize("m,n,kv,group,count", [(1, 20011, 8, 4, 1), (4, 20011, 8, 4, 1), (8, 20011, 2, 4, 3), (9, 20011, 2, 4, 2), (32, 9001, 2, 4, 2), (11, 9001, 2, 11, 2), (1, 40003, 8, 4, 2),
                                                (8, 40003, 8, 4, 2), (5, 40003, 8, 7, 2)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (700, 5)])
def test_which_kernel_takes_few_rows_of_long_caches(m, n, kv, group, count, window, sinks):
    # (few rows over few keys, over many, past the caches; up to 128 rows)
    check("bf16", count=count, kv=kv, group=group, m=m, n=n, window=window, sinks=sinks, decay=0.5, seed=m + n)


@pytest.mark.parametrize("dtype,m,n", [("bf16", 1, 500), ("bf16", 1, 70000), ("bf16", 8, 3000), ("bf16", 300, 300), ("bf16", 200, 5000), ("fp32", 3, 900), ("fp32", 150, 700)])
def test_recorded_calls_of_all_kernels(dtype, m, n):
    kv, group, dt = 4, 4, U.dtype_of(dtype)
    K, Q = U.randn(1, (1, kv, n, D), dt), U.randn(2, (1, m, kv * group, D), dt)
    lse = torch.full((1, kv * group, m), 6.0, device="cuda")
    recorded, eager = torch.zeros((2, 1, kv, n), device="cuda")
    with U.context(kv, group, dtype, n) as ctx:
        ctx.attend_weights(Q, K, lse, 1, m, n, n, eager, decay=0.0)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ctx.attend_weights(Q, K, lse, 1, m, n, n, recorded, decay=0.5)
        for turn in range(3):
            Q.copy_(U.randn(20 + turn, Q.shape, dt))
            eager.copy_(recorded)
            ctx.attend_weights(Q, K, lse, 1, m, n, n, eager, decay=0.5)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(recorded, eager) and bool((recorded[..., 0] > 0).all())
