"""Attention over shared kept rows whose sequences have long tails of their own (curdkv_attend_shared): many tiles of 32 keys a wave, each asked for while the one before is used."""
import math

import numpy as np
import pytest
import torch

from tests import attend_util as U
from tests.test_gpu_attend_shared import FORMS, check

pytestmark = pytest.mark.gpu
D = 128


@pytest.mark.parametrize("dtype,mx", FORMS)
@pytest.mark.parametrize("m,group", [(1, 4), (1, 1), (3, 7), (9, 4), (40, 2)])
@pytest.mark.parametrize("tail", [700, 5003])
def test_tails_of_thousands(dtype, mx, m, group, tail):
    # lengths that end inside a tile, at one, behind a wave's last round of four tiles and before it; shorter than m; none
    lens = [tail, tail - 1, tail // 128 * 128, tail // 128 * 128 + 1, 641, m - 1, 0, tail // 2]
    check(dtype, mx, 2, 4, 2, group, m, np.random.default_rng(m).integers(0, 200, 4), tail, lens, seed=tail + m)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tail", [4096, 16384])
def test_few_answers(dtype, tail):
    check(dtype, False, 1, 1, 1, 4, 1, [100], tail, None, seed=tail)
    check(dtype, False, 1, 2, 2, 4, 5, [0, 33], tail, [tail, tail - 33], seed=tail)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_long_tails_by_one_wave(dtype):
    # (2048 tails keep all waves busy: a wave each)
    lens = np.random.default_rng(5).integers(0, 701, 256)
    lens[:4] = 700, 699, 0, 672
    check(dtype, False, 2, 128, 8, 1, 1, np.full(16, 70), 700, lens, seed=3, heads=1)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_what_is_not_finite_far_into_a_tail(dtype):
    # an infinity in a token that some of a sequence's new ones see and some do not, many tiles on: it reaches those that see it, in its channel, and changes nothing else
    dt, m, n = U.dtype_of(dtype), 8, 3000
    Kk, Vk, Q = U.randn(1, (50, D), dt), U.randn(2, (50, D), dt), U.randn(5, (2, m, 4, D), dt)
    Kt, Vt = (U.randn(i, (2, 1, n, D), dt) for i in (3, 4))
    offsets, results = torch.tensor([0, 50], device="cuda"), []
    with U.context(1, 4, dtype, n) as ctx:
        for spoiled in (False, True):
            if spoiled:
                Vt[0, 0, n - 4, 5] = math.inf                          # (tokens 4 .. 7 of the eight)
                Vt[1, 0, 1500, 9] = -math.inf                          # (all of them)
            out = torch.empty_like(Q)
            ctx.attend_shared(Q, Kk, Vk, offsets, 1, 2, m, 50, out, K_tail=Kt, V_tail=Vt, tail_n=n, tail_stride=n)
            torch.cuda.synchronize()
            results.append(out)
    clean, got = results
    want = clean.clone()
    want[0, 4:, :, 5], want[1, :, :, 9] = math.inf, -math.inf
    assert torch.equal(got, want)
