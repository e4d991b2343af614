"""Attention over an fp32 cache of very small numbers, in either kernel: what is left of them is what the header says."""

import pytest
import torch

from tests import attend_util as U

pytestmark = pytest.mark.gpu
D = 128


@pytest.mark.parametrize("count,m", [(24, 520), (6, 300), (3, 1)])
def test_a_row_alone_of_any_size(count, m):
    # a window of one and queries of zeros: every token has its own row's value, with a weight of 1.  Parts of 8 bits end at 2^-133, half of which is what they may miss;
    # from 2^-109 on nothing
    kv, n = 8, m
    g = torch.Generator(device="cuda").manual_seed(m)
    V = torch.randn((count, kv, n, D), generator=g, device="cuda") * torch.exp2(torch.randint(-148, -95, (count, kv, n, D), generator=g, device="cuda").double()).float()
    K, Q = U.randn(1, (count, kv, n, D), torch.float32), torch.zeros((count, m, kv * 4, D), device="cuda")
    out = torch.empty_like(Q)
    with U.context(kv, 4, "fp32", n) as ctx:
        ctx.attend(Q, K, V, count, m, n, n, out, window=1)
        torch.cuda.synchronize()
    want = V.transpose(1, 2)[:, :, :, None].double()
    off = (out.view(count, m, kv, 4, D).double() - want).abs()
    assert float(off.max()) <= (2.0 ** -134 if m > 1 else 0.0)
    assert float(off[(want.abs() >= 2.0 ** -109).expand_as(off)].max()) == 0.0


@pytest.mark.parametrize("count,m", [(6, 300), (3, 1)])
def test_scores_of_small_keys_and_large_queries(count, m):
    kv, n, e = 8, 300, 118
    K, V, Q = (U.randn(i, (count, kv if i < 3 else m, n if i < 3 else kv * 4, D), torch.float32) for i in (1, 2, 3))
    K, Q = K * 2.0 ** -e, Q * 2.0 ** e
    out = torch.empty_like(Q)
    with U.context(kv, 4, "fp32", n) as ctx:
        ctx.attend(Q, K, V, count, m, n, n, out)
        torch.cuda.synchronize()
    for b, h in ((0, 0), (count - 1, 31)):
        want, _, mass, most = U.attention(Q[b, :, h], K[b, h // 4], V[b, h // 4], U.causal(m, n, n, 0, 0), D ** -0.5)
        # a score's products by 2^-22 of themselves and its sum by 128 * 2^-24, and each product by 2^-133 of its query; the weights by twice that
        score = (2.0 ** -22 + 128 * 2.0 ** -24) * most + 2.0 ** -133 * float(Q[b, :, h].double().abs().sum(-1).max()) * D ** -0.5
        rel = 2 * score + (n + 128) * 2.0 ** -24 + 2.0 ** -20
        assert bool(((out[b, :, h].double() - want).abs() <= rel * mass + 1e-30).all())
