"""Rows in 4 bits (curdkv_compact_mx, curdkv_expand_mx) against the format's definition, code by code."""

import math

import numpy as np
import pytest
import torch

from paper_2509_15038_amd import binding as B
from tests import attend_util as U
from tests.gpu_util import Guarded

pytestmark = pytest.mark.gpu
D = 128


def check(K, V, indices, offsets, dtype):
    """K, V [heads, n, 128]; every kept row's codes, scales and values."""
    heads, n = K.shape[:2]
    total = int(offsets[-1])
    # (pairs of bytes between canaries)
    codes = [Guarded((max(1, total), 32), torch.int16, -1) for _ in range(2)]
    scales = [Guarded((max(1, total), 2), torch.int16, -1) for _ in range(2)]
    outs = [Guarded((max(1, total), D), K.dtype, 5.0) for _ in range(2)]
    with B.Context(1, heads, 1, D, 32, dtype, n, 1) as ctx:
        ctx.compact_mx(K, V, n, indices, torch.from_numpy(offsets).cuda(), total, codes[0].t, scales[0].t, codes[1].t, scales[1].t)
        for c, s, o in zip(codes, scales, outs):
            ctx.expand_mx(c.t, s.t, total, o.t)
        torch.cuda.synchronize()
    for x in codes + scales + outs:
        x.check()
    head = np.repeat(np.arange(heads), np.diff(offsets))
    for X, c, s, o in zip((K, V), codes, scales, outs):
        rows = X[torch.from_numpy(head).cuda(), indices.long()]
        value, want_codes, want_scales = U.four_bits(rows)
        assert torch.equal(s.t[:total].contiguous().view(torch.uint8).view(-1, 4).cpu(), want_scales)
        assert torch.equal(c.t[:total].contiguous().view(torch.uint8).view(-1, 64).cpu(), want_codes)
        got = o.t[:total].double().cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(value)) and torch.equal(got.nan_to_num(7.0), value.nan_to_num(7.0))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("heads,n", [(1, 1), (1, 2), (3, 17), (2, 128), (5, 129), (2, 4099)])
def test_gathered_rows(dtype, heads, n):
    dt = U.dtype_of(dtype)
    rng = np.random.default_rng(n)
    K, V = U.randn(1, (heads, n, D), dt), U.randn(2, (heads, n, D), dt, 300.0)
    budgets = rng.integers(0, n + 1, heads)
    budgets[-1] = n
    offsets = np.concatenate([[0], np.cumsum(budgets)]).astype(np.int64)
    idx = np.concatenate([np.sort(rng.choice(n, b, replace=False)) for b in budgets]).astype(np.int32)
    check(K, V, torch.from_numpy(idx).cuda(), offsets, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_every_mantissa_and_exponent(dtype):
    # blocks whose largest value fixes the unit, the others every bf16 significand within 8 octaves below it, at units over the whole range, and
    # values just off the ties in fp32
    fine = torch.arange(128).float() / 128 + 1
    x = torch.cat([fine * 2.0 ** -k for k in range(8)])
    x = torch.cat([x, -x])
    if dtype == "fp32":
        ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]) / 4
        near = torch.cat([torch.nextafter(ties, torch.tensor(9.0)), torch.nextafter(ties, torch.tensor(0.0)), ties])
        x = torch.cat([x, near, -near])
    pad = -x.numel() % 31
    x = torch.cat([x, torch.zeros(pad)]).view(-1, 31)
    rows = []
    for top in (1.0, 1.5, 1.75, 1.9921875):
        block = torch.cat([x, torch.full((x.shape[0], 1), top)], 1)
        block = torch.cat([block, torch.zeros((-block.shape[0] % 4, 32))])
        for e in (-140, -130, -127, -126, -125, -124, -100, -1, 0, 1, 60, 126, 127):
            rows.append((block.double() * 2.0 ** e).float())
    K = torch.cat(rows).view(-1, D).to(U.dtype_of(dtype)).cuda()[None]
    n = K.shape[1]
    check(K, -K, torch.arange(n, dtype=torch.int32, device="cuda"), np.array([0, n]), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_blocks_that_are_not_finite(dtype):
    K = U.randn(1, (1, 64, D), U.dtype_of(dtype))
    K[0, 0, 0], K[0, 1, 33], K[0, 2, 127], K[0, 3, 64] = math.inf, -math.inf, math.nan, -math.nan
    K[0, 4], K[0, 5, 32:64], K[0, 6] = 0, 0, math.nan
    K[0, 7] = -0.0
    check(K, K.flip(2).contiguous(), torch.arange(64, dtype=torch.int32, device="cuda"), np.array([0, 64]), dtype)


def test_nothing_kept_and_refusals():
    K = U.randn(1, (2, 64, D), torch.bfloat16)
    c, s = torch.full((64, 64), 9, dtype=torch.uint8, device="cuda"), torch.full((64, 4), 9, dtype=torch.uint8, device="cuda")
    idx = torch.arange(64, dtype=torch.int32, device="cuda")
    out = torch.full((64, D), 3.0, dtype=torch.bfloat16, device="cuda")
    with B.Context(1, 2, 1, D, 32, "bf16", 64, 1) as ctx:
        ctx.compact_mx(K, K, 64, None, torch.zeros((3,), dtype=torch.int64, device="cuda"), 0, None, None, None, None)
        ctx.expand_mx(None, None, 0, None)
        good = dict(K=K, V=K, n=64, indices=idx, offsets=torch.tensor([0, 32, 64], device="cuda"), total=64, K_codes=c, K_scales=s, V_codes=c, V_scales=s)
        for bad in (dict(K=None), dict(V=None), dict(indices=None), dict(K_codes=None), dict(V_scales=None), dict(n=0), dict(n=65), dict(n=16),
                    dict(offsets=None), dict(total=-1), dict(total=129), dict(K=K.data_ptr() + 2), dict(V_codes=c.data_ptr() + 4)):
            with pytest.raises(B.CurdkvError) as e:
                ctx.compact_mx(**dict(good, **bad))
            assert e.value.code == B.ERR_INVALID_ARG, bad
        for bad in (dict(codes=None), dict(scales=None), dict(out=None), dict(rows=-1), dict(out=out.data_ptr() + 2)):
            with pytest.raises(B.CurdkvError) as e:
                ctx.expand_mx(**dict(dict(codes=c, scales=s, rows=64, out=out), **bad))
            assert e.value.code == B.ERR_INVALID_ARG, bad
        # indices outside the head are left out
        ctx.compact_mx(K, K, 64, torch.full((64,), 64, dtype=torch.int32, device="cuda"), torch.tensor([0, 32, 64], device="cuda"), 64, c, s, c.clone(), s.clone())
        torch.cuda.synchronize()
        assert bool((c == 9).all()) and bool((s == 9).all()) and bool((out == 3).all())


def test_more_rows_than_a_launch_has_threads_for():
    # 2^28 rows are 2^32 pieces of eight channels; the last rows alone are looked at
    rows, last = 2 ** 28 + 77, 200
    x = U.randn(9, (last, D), torch.bfloat16)
    value, codes, scales = U.four_bits(x)
    far = [torch.empty((rows, w), dtype=torch.uint8, device="cuda") for w in (64, 4)]
    far[0][-last:], far[1][-last:] = codes.cuda(), scales.cuda()
    out = torch.empty((rows, D), dtype=torch.bfloat16, device="cuda")
    with U.context(1, 4, "bf16", 64) as ctx:
        ctx.expand_mx(*far, rows, out)
        torch.cuda.synchronize()
    assert torch.equal(out[-last:].double().cpu(), value)
