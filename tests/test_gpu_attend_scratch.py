"""The attention calls' scratch: a context's own is as much as they use, less is enough, nothing beyond it is touched; parts of a prompt's keys."""

import numpy as np
import pytest
import torch

from paper_2509_15038_amd import binding as B
from tests import attend_util as U

pytestmark = pytest.mark.gpu
D = 128


def scratch_of(size):
    """`size` bytes and, right behind them, 1 MB that must stay as it is."""
    whole = torch.full((size + (1 << 20),), 77, dtype=torch.uint8, device="cuda")
    whole[:size] = 0
    return whole[:size], whole[size:]


@pytest.mark.parametrize("m", [256, 512, 1024])
def test_as_much_as_prompts_use(m):
    # 64, 128 and 256 workgroups of 128 rows, their keys in 8, 4 and 2 parts; more scratch changes nothing
    n = 16000
    K, V, Q = U.randn(1, (1, 8, n, D), torch.bfloat16), U.randn(2, (1, 8, n, D), torch.bfloat16), U.randn(3, (1, m, 32, D), torch.bfloat16)
    a, b, c = (torch.empty_like(Q) for _ in range(3))
    with U.context(8, 4, "bf16", n) as ctx:
        ctx.attend(Q, K, V, 1, m, n, n, a)
        ctx.attend(Q, K, V, 1, m, n, n, b, scratch=scratch_of(100 << 20)[0])
        ctx.attend(Q, K, V, 1, m, n, n, c, scratch=scratch_of(0)[0])
        torch.cuda.synchronize()
    assert torch.equal(a, b) and not torch.equal(a, c)                  # (no parts: other roundings)
    for h in (0, 31):
        want = U.attention(Q[0, :, h], K[0, h // 4], V[0, h // 4], U.causal(m, n, n, 0, 0), D ** -0.5)
        for out in (a, c):
            U.check_attention(out[0, :, h], None, want, "bf16", n, f"head {h}")


@pytest.mark.parametrize("heads", [2100, 4096])
def test_as_much_as_few_tokens_use(heads):
    rng = np.random.default_rng(heads)
    budgets = rng.integers(900, 1500, heads)
    budgets[7] = 0
    off = np.concatenate([[0], np.cumsum(budgets)]).astype(np.int64)
    total = int(off[-1])
    K, V, Q = U.randn(1, (total, D), torch.bfloat16), U.randn(2, (total, D), torch.bfloat16), U.randn(3, (heads, 1, 4, D), torch.bfloat16)
    offsets, outs = torch.from_numpy(off).cuda(), [torch.empty_like(Q) for _ in range(3)]
    with U.context(1, 4, "bf16", 64) as ctx:
        for out, scratch in zip(outs, (None, scratch_of(100 << 20)[0], scratch_of(0)[0])):
            ctx.attend_kept(Q, K, V, offsets, heads, 1, total, out, scratch=scratch)
        torch.cuda.synchronize()
        assert bool((ctx._scratch_tensor[:16384] == 0).all())
    assert torch.equal(outs[0], outs[1]) and not torch.equal(outs[0], outs[2])
    for g in [0, 6, 7, 8, heads // 2, heads - 1, *rng.integers(0, heads, 40).tolist()]:
        k, v = K[off[g]: off[g + 1]], V[off[g]: off[g + 1]]
        for h in range(4):
            want = U.attention(Q[g, :, h], k, v, torch.ones((1, k.shape[0]), dtype=torch.bool, device="cuda"), D ** -0.5)
            for out in (outs[0], outs[2]):
                U.check_attention(out[g, :, h], None, want, "bf16", k.shape[0], f"head {g}")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("count,kv,m,n,window,sinks", [(1, 2, 300, 5000, 0, 0), (1, 8, 100, 9001, 0, 0), (2, 4, 130, 6000, 2500, 70), (3, 2, 1, 5000, 0, 0), (20, 2, 5, 3000, 0, 0)])
def test_any_size_and_nothing_behind_it(dtype, count, kv, m, n, window, sinks):
    # (prompts in parts, and few tokens; ragged lengths, the last shorter than its new tokens)
    dt = U.dtype_of(dtype)
    K, V, Q = U.randn(1, (count, kv, n, D), dt), U.randn(2, (count, kv, n, D), dt), U.randn(3, (count, m, kv * 4, D), dt)
    lens = np.random.default_rng(n).integers(n // 2, n + 1, count)
    if count > 1:
        lens[-1] = m // 2
    lengths = torch.from_numpy(lens.astype(np.int32)).cuda()
    row = 520
    with U.context(kv, 4, dtype, n) as ctx:
        for size in (0, 16, 16384, 16384 + row * 16 * 9 + 8, 16384 + row * 700, 16384 + row * 5000, 16384 + row * 20000 + 16, B.ATTEND_SCRATCH_BYTES):
            scratch, behind = scratch_of(size)
            out, lse = torch.full_like(Q, float("nan")), torch.full((count, kv * 4, m), float("nan"), device="cuda")
            ctx.attend(Q, K, V, count, m, n, n, out, lengths=lengths, window=window, n_sink=sinks, lse=lse, scratch=scratch)
            torch.cuda.synchronize()
            assert bool((behind == 77).all()) and bool((scratch[:16384] == 0).all()), size
            for b, h in {(0, 0), (count - 1, kv * 4 - 1)}:
                seen = U.causal(m, n, int(lens[b]), window, sinks)
                want = U.attention(Q[b, :, h], K[b, h // 4], V[b, h // 4], seen, D ** -0.5)
                U.check_attention(out[b, :, h], lse[b, h], want, dtype, n, f"scratch {size}, seq {b} head {h}")


@pytest.mark.parametrize("mx", [False, True])
def test_any_size_over_kept_rows(mx):
    rng = np.random.default_rng(5)
    kv, m, kept = 8, 1 if mx else 300, 3000
    off = np.concatenate([[0], np.cumsum(rng.integers(0, 2 * kept, kv))]).astype(np.int64)
    total = int(off[-1])
    K, V, Q = U.randn(1, (total, D), torch.bfloat16), U.randn(2, (total, D), torch.bfloat16), U.randn(3, (1, m, kv * 4, D), torch.bfloat16)
    Kt, Vt, offsets = U.randn(4, (1, kv, m, D), torch.bfloat16), U.randn(5, (1, kv, m, D), torch.bfloat16), torch.from_numpy(off).cuda()
    with U.context(kv, 4, "bf16", 512) as ctx:
        if mx:
            codes = [torch.empty((total, w), dtype=torch.uint8, device="cuda") for w in (64, 4, 64, 4)]
            with B.Context(1, 1, 4, D, 32, "bf16", total, 1) as one:
                one.compact_mx(K, V, total, torch.arange(total, dtype=torch.int32, device="cuda"), torch.tensor([0, total], device="cuda"), total, *codes)
            ctx.expand_mx(*codes[:2], total, K)
            ctx.expand_mx(*codes[2:], total, V)
        for size in (0, 16384, 16384 + 520 * 16 * 20, 16384 + 520 * 3000, 16384 + 520 * 30000 + 16, B.ATTEND_SCRATCH_BYTES):
            scratch, behind = scratch_of(size)
            out = torch.full_like(Q, float("nan"))
            since = dict(K_tail=Kt, V_tail=Vt, tail_n=m, tail_stride=m, scratch=scratch)
            if mx:
                ctx.attend_kept_mx(Q, *codes, offsets, 1, m, total, out, **since)
            else:
                ctx.attend_kept(Q, K, V, offsets, 1, m, total, out, **since)
            torch.cuda.synchronize()
            assert bool((behind == 77).all()) and bool((scratch[:16384] == 0).all()), size
            for h in (0, 9, 31):
                g = h // 4
                k, v = torch.cat([K[off[g]: off[g + 1]], Kt[0, g]]), torch.cat([V[off[g]: off[g + 1]], Vt[0, g]])
                seen = torch.cat([torch.ones((m, int(off[g + 1] - off[g])), dtype=torch.bool, device="cuda"), U.causal(m, m, m, 0, 0)], 1)
                U.check_attention(out[0, :, h], None, U.attention(Q[0, :, h], k, v, seen, D ** -0.5), "bf16", k.shape[0], f"scratch {size} head {h}")
