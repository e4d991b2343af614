"""Attention of a few tokens where workgroups share heads: each head its own workgroups, equal shares of all of them with parts of several heads in one, more
heads than units, and the sides of the rules between these and a workgroup a head."""

import numpy as np
import pytest
import torch

from paper_2509_15038_amd import binding as B
from tests import attend_util as U
from tests.test_gpu_attend_kept import FORMS, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("count,n", [(1, 750), (1, 900), (1, 8200), (32, 383), (32, 900), (31, 1700)])
def test_heads_with_workgroups_of_their_own(dtype, count, n):
    U.check_attend(dict(count=count, kv=2, m=1, n=n, dtype=dtype), seed=n)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("count,m,n,window", [(33, 1, 2100, 0), (65, 2, 2200, 0), (150, 1, 2050, 0), (65, 1, 4200, 2500), (9, 9, 2300, 0)])
def test_equal_shares_of_all_heads(dtype, count, m, n, window):
    U.check_attend(dict(count=count, kv=2, group=2 if m > 1 else 4, m=m, n=n, window=window, sinks=4, dtype=dtype), seed=count)


@pytest.mark.parametrize("count", [128, 129])
def test_whole_turns_of_the_units(count):
    U.check_attend(dict(count=count, kv=2, group=1, m=1, n=2100), seed=count, lengths="full")


@pytest.mark.parametrize("dtype,mx", FORMS)
@pytest.mark.parametrize("heads,mean,most", [(3, 180, 300), (32, 400, 1500), (35, 700, 9000), (150, 600, 2000), (300, 600, 700), (520, 550, 2100)])
def test_kept_rows(dtype, mx, heads, mean, most):
    rng = np.random.default_rng(heads)
    budgets = np.minimum(rng.exponential(mean, heads * 2).astype(int) + mean // 4, most)
    budgets[rng.integers(0, heads * 2, 3)] = 0
    budgets[-1] = 0
    check(dtype, mx, heads, 2, 2, 1, budgets, 20, rng.integers(0, 21, heads), seed=heads)


@pytest.mark.parametrize("mx", [False, True])
def test_all_rows_in_one_head(mx):
    # 4 and 150 heads; one has all the rows, the others nothing but, some of them, a row since
    for heads in (4, 150):
        budgets = np.zeros(heads, dtype=int)
        budgets[heads // 2] = 20000
        check("bf16", mx, heads, 1, 4, 1, budgets, 1, np.arange(heads) % 2, seed=heads)


def test_the_first_call_on_another_stream():
    # the context's scratch is cleared on the current stream, which is busy; the call is on another one
    K, V, Q = (U.randn(i, (1, 2, 5000, U.D) if i < 3 else (1, 1, 8, U.D), torch.bfloat16) for i in (1, 2, 3))
    out, side = torch.empty_like(Q), torch.cuda.Stream()
    torch.cuda.synchronize()
    dirty = torch.full((B.ATTEND_SCRATCH_BYTES,), 255, dtype=torch.uint8, device="cuda")
    del dirty                                                                        # (what the allocator gives out next)
    with U.context(2, 4, "bf16", 5000) as ctx:
        torch.cuda._sleep(100_000_000)
        for _ in range(3):
            ctx.attend(Q, K, V, 1, 1, 5000, 5000, out, stream=side)
        torch.cuda.synchronize()
        assert bool((ctx._scratch_tensor[:16384] == 0).all())
    for h in range(8):
        want = U.attention(Q[0, :, h], K[0, h // 4], V[0, h // 4], U.causal(1, 5000, 5000, 0, 0), U.D ** -0.5)
        U.check_attention(out[0, :, h], None, want, "bf16", 5000)


def test_a_first_call_is_not_recorded():
    K, V, Q = (U.randn(i, (1, 2, 100, U.D) if i < 3 else (1, 1, 8, U.D), torch.bfloat16) for i in (1, 2, 3))
    out, scratch = torch.empty_like(Q), torch.zeros(B.ATTEND_SCRATCH_BYTES, dtype=torch.uint8, device="cuda")
    with U.context(2, 4, "bf16", 100) as ctx:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            with pytest.raises(RuntimeError):
                ctx.attend(Q, K, V, 1, 1, 100, 100, out)
            ctx.attend(Q, K, V, 1, 1, 100, 100, out, scratch=scratch)
        graph.replay()
        torch.cuda.synchronize()
        recorded = out.clone()
        ctx.attend(Q, K, V, 1, 1, 100, 100, out)
        torch.cuda.synchronize()
        assert torch.equal(recorded, out)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("count,n,longest", [(1, 16000, 40), (1, 16000, 700), (4, 16000, 3000), (30, 6000, 90), (30, 6000, 2000), (40, 5000, 60), (40, 5000, 1500), (200, 4200, 50), (200, 4200, 0)])
def test_lengths_far_below_what_there_may_be(dtype, count, n, longest):
    # the host shares out by the cache's size, the device by the lengths that there are
    rng = np.random.default_rng(n + longest)
    lengths = rng.integers(0, longest + 1, count)
    lengths[-1] = longest
    U.check_attend(dict(count=count, kv=2, group=2, m=1, n=n, dtype=dtype), seed=longest, lengths=lengths)


@pytest.mark.parametrize("dtype,mx", FORMS)
@pytest.mark.parametrize("heads", [3, 40, 130])
def test_a_layer_with_little_of_a_large_packed_cache(dtype, mx, heads):
    # rows not given: the host takes all rows for this layer's
    rng = np.random.default_rng(heads)
    budgets = rng.integers(0, 90, heads * 2)
    check(dtype, mx, heads, 2, 2, 1, budgets, 5, rng.integers(0, 6, heads), seed=heads, before=200000 if heads > 3 else 30000, rows_known=False)
