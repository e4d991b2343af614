"""Prompts over an fp32 cache: either size of workgroup, what the parts of 8 bits have to hold, infinities and NaN in tiles of either kind."""

import math

import pytest
import torch

from tests import attend_util as U

pytestmark = pytest.mark.gpu
D = 128


@pytest.mark.parametrize("count,m,n,window,sinks", [(24, 513, 513, 0, 0), (25, 512, 700, 0, 0), (26, 530, 530, 100, 40), (24, 600, 600, 257, 4)])
def test_eight_waves(count, m, n, window, sinks):
    U.check_attend(dict(count=count, kv=2, m=m, n=n, window=window, sinks=sinks, dtype="fp32"), seed=m)


@pytest.mark.parametrize("count,m,n,window,sinks", [(12, 32, 32, 0, 0), (12, 33, 33, 0, 0), (14, 250, 1021, 0, 0), (11, 511, 511, 31, 33), (11, 300, 2000, 700, 5)])
def test_four_waves(count, m, n, window, sinks):
    U.check_attend(dict(count=count, kv=16, group=4, m=m, n=n, window=window, sinks=sinks, dtype="fp32"), seed=n)


@pytest.mark.parametrize("count,m", [(24, 520), (6, 300)])
def test_a_row_alone_is_its_result(count, m):
    # a window of one and queries of zeros: every token sees its own row only, whose score is 0 and whose weight is 1, so that the parts of its value must add up to
    # it, whatever its size
    kv, n = 8, m
    g = torch.Generator(device="cuda").manual_seed(m)
    V = torch.randn((count, kv, n, D), generator=g, device="cuda") * torch.exp2(torch.randint(-90, 126, (count, kv, n, D), generator=g, device="cuda").float())
    V[:, :, ::7, ::5] = torch.finfo(torch.float32).max
    V[:, :, 3::7, 1::5] = -torch.finfo(torch.float32).max
    V[:, :, 5::7, 2::5] = 1.0 + 2.0 ** -23
    V[:, :, 6::7, 3::5] = 0.0
    K, Q = U.randn(1, (count, kv, n, D), torch.float32), torch.zeros((count, m, kv * 4, D), device="cuda")
    out = torch.empty_like(Q)
    with U.context(kv, 4, "fp32", n) as ctx:
        ctx.attend(Q, K, V, count, m, n, n, out, window=1)
        torch.cuda.synchronize()
    off = out.view(count, m, kv, 4, D) != V.transpose(1, 2)[:, :, :, None]
    assert not bool(off.any()), int(off.sum())


@pytest.mark.parametrize("count,m", [(24, 520), (3, 300)])
@pytest.mark.parametrize("window", [0, 90])
def test_values_that_are_not_finite(count, m, window):
    # rows with infinities of either sign and NaN in some channels: who sees the row has them there, whether all of its tile is seen or not, nobody else does, and
    # the other channels are right
    kv, n = 8, m
    K, V, Q = (U.randn(i, (count, kv if i < 3 else m, n if i < 3 else kv * 4, D), torch.float32) for i in (1, 2, 3))
    low = torch.tensor(0x7F800001, dtype=torch.int32).view(torch.float32).item()          # a NaN of the lowest bits
    bad = {5: math.inf, 40: -math.inf, 101: math.nan, 102: low, n - 3: math.inf}
    for row, value in bad.items():
        V[:, :, row, row % D] = value
    V[0, 0, 50, 5] = -math.inf                                                           # with row 5's: NaN
    out = torch.empty_like(Q)
    with U.context(kv, 4, "fp32", n) as ctx:
        ctx.attend(Q, K, V, count, m, n, n, out, window=window)
        torch.cuda.synchronize()
    clean = torch.where(torch.isfinite(V), V, 0.0)
    for b, h in ((0, 0), (count - 1, kv * 4 - 1)):
        seen = U.causal(m, n, n, window, 0)
        want = U.attention(Q[b, :, h], K[b, h // 4], clean[b, h // 4], seen, D ** -0.5)
        special = ~torch.isfinite(V[b, h // 4])
        touched = (seen.double() @ special.double()) > 0                                 # [m, D]
        expect = torch.zeros((m, D), device="cuda")
        for t in range(m):
            rows = special & seen[t][:, None]
            if bool(rows.any()):
                expect[t] = torch.where(rows, V[b, h // 4], 0.0).sum(0)
        got = out[b, :, h]
        assert torch.equal(torch.isnan(got), touched & torch.isnan(expect))
        inf = touched & torch.isinf(expect)
        assert torch.equal(torch.isinf(got), inf) and torch.equal(got[inf], expect[inf])
        held = torch.where(touched, want[0], got.double())
        U.check_attention(held, None, want, "fp32", n, f"seq {b} head {h}")


def test_keys_that_are_not_finite():
    # a key of infinities or NaN in a row that a token does not see leaves it alone; who sees a NaN has NaN
    count, kv, m = 6, 8, 300
    K, V, Q = (U.randn(i, (count, kv if i < 3 else m, m if i < 3 else kv * 4, D), torch.float32) for i in (1, 2, 3))
    K[:, :, 150, 3], K[:, :, 290, 7] = math.nan, math.inf
    out = torch.empty_like(Q)
    with U.context(kv, 4, "fp32", m) as ctx:
        ctx.attend(Q, K, V, count, m, m, m, out, window=100)
        torch.cuda.synchronize()
    seen = U.causal(m, m, m, 100, 0)
    sees = seen[:, 150]
    assert bool(torch.isnan(out[:, sees]).all())
    fine = ~sees & ~seen[:, 290]
    want = U.attention(Q[2, fine, 9], K[2, 2], V[2, 2], seen[fine], D ** -0.5)
    U.check_attention(out[2, fine, 9], None, want, "fp32", m)


def test_magnitudes():
    # scores of rows of 2^-60 and 2^60: nothing of the parts is lost
    count, kv, m = 6, 8, 300
    K, V, Q = (U.randn(i, (count, kv if i < 3 else m, m if i < 3 else kv * 4, D), torch.float32) for i in (1, 2, 3))
    out = torch.empty_like(Q)
    with U.context(kv, 4, "fp32", m) as ctx:
        ctx.attend(Q * 2.0 ** 60, K * 2.0 ** -60, V * 2.0 ** -40, count, m, m, m, out)
        torch.cuda.synchronize()
    want = U.attention(Q[1, :, 5], K[1, 1], V[1, 1], U.causal(m, m, m, 0, 0), D ** -0.5)
    U.check_attention(out[1, :, 5] * 2.0 ** 40, None, want, "fp32", m)
