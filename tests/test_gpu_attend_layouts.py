"""Attention in further layouts of heads, and kept rows that are not finite beside heads that do not hold them."""

import math

import pytest
import torch

from tests import attend_util as U
from tests.test_gpu_attend_kept import FORMS, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kv,group", [(8, 1), (16, 1), (8, 5), (2, 7)])
@pytest.mark.parametrize("count,m,n,window", [(3, 1, 700, 0), (40, 1, 2500, 0), (2, 3, 1500, 400), (2, 700, 700, 0), (3, 500, 700, 130), (1, 300, 4000, 0)])
def test_head_layouts(dtype, kv, group, count, m, n, window):
    U.check_attend(dict(count=count, kv=kv, group=group, m=m, n=n, window=window, sinks=4, dtype=dtype), seed=kv * group + m)


@pytest.mark.parametrize("dtype,mx", FORMS)
@pytest.mark.parametrize("m", [1, 700])
def test_one_query_head_for_each_of_eight(dtype, mx, m):
    budgets = [0, 1, 700, 31, 300, 2000, 33, 64, 100, 101, 102, 103, 1500, 0, 1, 16]
    check(dtype, mx, 2, 8, 1, m, budgets, 40, [40, 3], seed=m)


@pytest.mark.parametrize("dtype,mx", FORMS)
@pytest.mark.parametrize("m", [1, 5, 320])
def test_kept_rows_of_other_heads_that_are_not_finite(dtype, mx, m):
    # heads 1, 2 and 6 hold infinities and NaN, in first and last rows too; those beside them must not notice
    budgets = [90, 100, 33, 64, 1000, 17, 700, 2]

    def spoil(Kk, Vk, Kt, Vt):
        Vk[95, 3], Vk[150], Vk[189, 100] = math.nan, math.inf, -math.inf
        Kk[190], Kk[222, 7] = math.nan, math.inf
        Kk[1304:2004] = math.nan

    o, l = check(dtype, mx, 2, 4, 4, m, budgets, 20, None, seed=m, spoil=spoil)
    o, l = o.transpose(1, 2).reshape(8, 4, m, U.D), l.reshape(8, 4, m)
    for g in range(8):
        clean = g not in (1, 2, 6)
        assert bool(torch.isfinite(o[g].float()).all()) == clean, g
        assert bool(torch.isfinite(l[g]).all()) == (clean or g == 1), g
    assert bool(torch.isnan(o[6]).all()) and bool(torch.isnan(l[6]).all()) and bool(torch.isnan(o[2].float()).all())
    wide = slice(64, 128) if mx else slice(100, 101)                    # (in 4 bits the whole block is NaN)
    assert not bool(torch.isfinite(o[1, :, :, 3]).any()) and not bool(torch.isfinite(o[1, :, :, wide]).any())
