"""Weights of calls whose queries of a tile of keys pass 2^31 bytes, so that the tile is gone over in several passes (curdkv_attend_weights)."""
import math

import pytest
import torch

from tests import attend_util as U
from tests.test_gpu_weights import lse_of

pytestmark = pytest.mark.gpu
D = 128


def chunked(seed, shape, dtype):
    """As U.randn, without 32-bit numbers for all of it at once."""
    x = torch.empty(shape, dtype=dtype, device="cuda")
    flat = x.view(-1)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    for a in range(0, flat.numel(), 1 << 27):
        part = flat[a: a + (1 << 27)]
        part.copy_(torch.randn(part.shape, generator=g, device="cuda"))
    return x


# many KV heads: a pass is four stages of rows; many query heads of each, by shares of the products
@pytest.mark.parametrize("dtype,kv,group,m,n", [("bf16", 16384, 1, 600, 600), ("fp32", 16384, 1, 300, 300), ("bf16", 256, 256, 300, 256), ("fp32", 256, 128, 300, 128)])
@pytest.mark.parametrize("window,sinks,decay", [(0, 0, 0.5), (150, 4, 0.0)])
def test_several_passes(dtype, kv, group, m, n, window, sinks, decay):
    scale, dt = D ** -0.5, U.dtype_of(dtype)
    rows = 2 ** 31 // (kv * (256 if dtype == "bf16" else 512))             # of a pass
    assert m * group > rows
    heads = sorted({0, 1, kv // 2 + 1, kv - 1})
    K, Q = chunked(1, (1, kv, n, D), dt), chunked(2, (1, m, kv * group, D), dt)
    lse = torch.full((1, kv * group, m), 7.0, device="cuda")
    seen = U.causal(m, n, n, window, sinks)
    for h in heads:
        for i in range(group):
            lse[0, h * group + i] = lse_of(Q[0, :, h * group + i], K[0, h], seen, scale).float()
    old = torch.exp(U.randn(3, (1, kv, n), torch.float32))
    mass = old.clone() if decay else torch.full_like(old, math.nan)
    with U.context(kv, group, dtype, max(m, n)) as ctx:
        ctx.attend_weights(Q, K, lse, 1, m, n, n, mass, window=window, n_sink=sinks, scale=scale, decay=decay)
        torch.cuda.synchronize()
    assert not bool(mass.isnan().any())
    for h in heads:
        want = torch.zeros(n, dtype=torch.float64, device="cuda")
        off = torch.zeros(n, dtype=torch.float64, device="cuda")
        for i in range(group):
            q, k, z = Q[0, :, h * group + i].double(), K[0, h].double(), lse[0, h * group + i].double()[:, None]
            x = (q @ k.T) * scale
            w = torch.where(seen & (z != -math.inf), torch.exp(torch.where(seen, x - z, 0.0)), 0.0)
            want += w.sum(0)
            # as in test_gpu_weights.py: 128 products and sums below 2^-24 (or what parts leave out, 2^-22), four roundings of the score and of lse, the exponential 2^-22
            rel = 128 * 2.0 ** -24 * (q.abs() @ k.abs().T) * scale + 4 * 2.0 ** -24 * (x.abs() + z.abs()) + 2.0 ** -22
            off += torch.where(w > 0, w * rel, 0.0).sum(0)
        total = want + decay * old[0, h].double()
        # (one more sum for every pass)
        bound = off + want * (m * group + 16) * 2.0 ** -24 + 4 * 2.0 ** -24 * total + 1e-35
        err = (mass[0, h].double() - total).abs()
        assert bool((err <= bound).all()), f"head {h}: {int((err > bound).sum())} of {n} off, worst {float((err / bound).max()):.2f} of the bound"
