"""Attention calls whose counts are large: sums of work beyond 31 bits, and sizes that a launch does not take."""

import pytest
import torch

from paper_2509_15038_amd import binding as B
from tests import attend_util as U

pytestmark = pytest.mark.gpu
D = 128


def test_more_work_than_31_bits_count():
    # 4096 tiles of 16 queries over one head of 20 million rows in 4 bits, 2.6e9 tiles of keys in all.  All keys are zeros but 60, which score 40 and more: the others weigh
    # 2e7 e^-40 < 2^-30 together, and the result is that over the 60
    rows, m, group = 20_000_000, 16384, 4
    g = torch.Generator(device="cuda").manual_seed(1)
    at = torch.cat([torch.tensor([0, 31, 32, rows // 2, rows - 33, rows - 32, rows - 1], device="cuda"), torch.randint(0, rows, (53,), generator=g, device="cuda")]).unique()
    K_codes, K_scales = torch.zeros((rows, 64), dtype=torch.uint8, device="cuda"), torch.full((rows, 4), 125, dtype=torch.uint8, device="cuda")
    K_codes[at] = torch.randint(0, 256, (at.numel(), 64), generator=g, device="cuda").to(torch.uint8)
    K_codes[at, 0] = 7                                                  # channel 0: 6; channel 1: 0
    V_codes = torch.randint(0, 256, (rows, 64), generator=g, device="cuda", dtype=torch.uint8)
    Q = U.randn(2, (1, m, group, D), torch.bfloat16)
    Q[..., 0] = 360.0                                                   # 360 * 6 / 4 / sqrt(128) = 47.7, the other channels +-3
    out, lse = torch.empty_like(Q), torch.empty((group, m), device="cuda")
    held = [torch.empty((at.numel(), D), dtype=torch.bfloat16, device="cuda") for _ in "KV"]
    with U.context(1, group, "bf16", 64) as ctx:
        ctx.attend_kept_mx(Q, K_codes, K_scales, V_codes, K_scales, torch.tensor([0, rows], device="cuda"), 1, m, rows, out, lse=lse)
        for x, codes in zip(held, (K_codes, V_codes)):
            ctx.expand_mx(codes[at].contiguous(), K_scales[at].contiguous(), at.numel(), x)
        torch.cuda.synchronize()
    some = torch.tensor([0, 1, 3, 4, 5, 511, 4097, 8191, 12345, m - 2, m - 1], device="cuda")
    for h in range(group):
        want = U.attention(Q[0, some, h], held[0], held[1], torch.ones((some.numel(), at.numel()), dtype=torch.bool, device="cuda"), D ** -0.5)
        assert float((Q[0, some, h].double() @ held[0].double().T).min()) * D ** -0.5 > 40
        U.check_attention(out[0, some, h], lse[h, some], want, "bf16", at.numel(), f"head {h}")
    # every token's own sum, by the same 60 keys in 32 bits
    x = torch.matmul(Q[0].float(), held[0].float().T.contiguous()) * D ** -0.5
    off = (torch.logsumexp(x.double(), -1).T - lse.double()).abs().max()
    assert float(off) < 2 * 128 * 2.0 ** -24 * 200, float(off)           # (scores are sums of 128 products, of magnitudes below 200 together)


@pytest.mark.parametrize("mx", [False, True])
def test_more_rows_than_31_bits_count(mx):
    # refused before anything is launched: the arrays are small ones
    K, Q = U.randn(1, (64, D), torch.bfloat16), U.randn(3, (1, 1, 4, D), torch.bfloat16)
    codes, scales = torch.zeros((64, 64), dtype=torch.uint8, device="cuda"), torch.zeros((64, 4), dtype=torch.uint8, device="cuda")
    off, out = torch.tensor([0, 64], device="cuda"), torch.full_like(Q, 7.0)
    with U.context(1, 4, "bf16", 64) as ctx:
        call = (lambda total: ctx.attend_kept_mx(Q, codes, scales, codes, scales, off, 1, 1, total, out)) if mx else \
            (lambda total: ctx.attend_kept(Q, K, K, off, 1, 1, total, out))
        for total in (2 ** 31, 2 ** 40):
            with pytest.raises(B.CurdkvError) as e:
                call(total)
            assert e.value.code == B.ERR_UNSUPPORTED
        torch.cuda.synchronize()
        assert bool((out == 7).all())
        call(64)


def test_more_tokens_than_a_launch_has_threads_for():
    # 2^26 tokens of 3 heads and some (51 GB): the last ones, those around a launch's end and the first are looked at
    m = 2 ** 26 + 37
    qkv, Q = torch.empty((m, 3 * D), dtype=torch.bfloat16, device="cuda"), torch.empty((m, D), dtype=torch.bfloat16, device="cuda")
    K, V = (torch.full((64, D), 5.0, dtype=torch.bfloat16, device="cuda") for _ in "KV")
    some = torch.tensor([*range(40), 2 ** 25 - 1, 2 ** 25, 2 ** 25 + 1, 2 ** 26 - 1, 2 ** 26, *range(m - 30, m)], device="cuda")
    qkv[some] = U.randn(1, (some.numel(), 3 * D), torch.bfloat16)
    Q[some] = float("nan")
    angle = torch.arange(50, device="cuda")[:, None] * 0.01 * torch.arange(1, 65, device="cuda")[None]
    table = torch.stack([angle.cos(), angle.sin()], 1).contiguous()
    start = 31                                                         # (the first 33 tokens have a row of the cache; positions beyond the table are its last)
    with U.context(1, 1, "bf16", 64) as ctx:
        ctx.rotate(qkv, 1, m, table, Q, K, V, 64, starts=torch.tensor([start], dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
    x = qkv[some].double().view(-1, 3, D)
    turn = table.double()[(some + start).clamp(max=49)]
    cos, sin = turn[:, None, 0], turn[:, None, 1]
    a, b = x[:, :2, :64], x[:, :2, 64:]
    want = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    size = torch.cat([(a * cos).abs() + (b * sin).abs(), (b * cos).abs() + (a * sin).abs()], -1)
    limit = 2.0 ** -8 * 1.01 * want.abs() + 4 * 2.0 ** -24 * size      # (a bf16 significand has 8 bits; two products and a sum in 32)
    assert bool(((Q[some].double() - want[:, 0]).abs() <= limit[:, 0]).all())
    assert bool(((K[start:].double() - want[:33, 1]).abs() <= limit[:33, 1]).all()) and torch.equal(V[start:].double(), x[:33, 2])
    assert bool((K[:start] == 5).all()) and bool((V[:start] == 5).all())


@pytest.mark.parametrize("kept", [False, True])
def test_more_sequences_than_a_launch_has_workgroups_for(kept):
    # 2^24 sequences and some, of no row or one, which is the result then
    count = 2 ** 24 + 41
    Q, V = (torch.randint(-99, 99, (count, D), dtype=torch.int8, device="cuda").to(torch.bfloat16) for _ in "QV")
    have = torch.randint(0, 2, (count,), device="cuda").to(torch.int32)
    out, lse = torch.full_like(Q, 7.0), torch.full((count,), 7.0, device="cuda")
    with U.context(1, 1, "bf16", 1) as ctx:
        if kept:
            offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), have.long().cumsum(0)])
            ctx.attend_kept(Q, V, V, offsets, count, 1, count, out, lse=lse, scale=1e-9)
            want = V[(offsets[1:] - 1).clamp(min=0)]
        else:
            ctx.attend(Q, V, V, count, 1, 1, 1, out, lengths=have, lse=lse, scale=1e-9)
            want = V
        torch.cuda.synchronize()
    assert torch.equal(out, torch.where(have[:, None] > 0, want, 0.0))
    assert torch.equal(torch.isinf(lse), have == 0) and float(lse[have > 0].abs().max()) < 128 * 99 ** 2 * 1.01e-9


def test_one_sequence_of_more_than_a_launch_has_workgroups_for():
    # refused before anything is launched: the arrays are small ones
    K, Q = U.randn(1, (64, D), torch.bfloat16), U.randn(3, (1, 1, 4, D), torch.bfloat16)
    codes, scales = torch.zeros((64, 64), dtype=torch.uint8, device="cuda"), torch.zeros((64, 4), dtype=torch.uint8, device="cuda")
    off, out = torch.tensor([0, 64], device="cuda"), torch.full_like(Q, 7.0)
    with U.context(1, 4, "bf16", 64) as ctx:
        with pytest.raises(B.CurdkvError) as e:
            ctx.attend_kept_mx(Q, codes, scales, codes, scales, off, 1, 2 ** 26, 64, out)
        assert e.value.code == B.ERR_UNSUPPORTED
        torch.cuda.synchronize()
    assert bool((out == 7).all())
