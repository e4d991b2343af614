"""Rows in 4 bits at both ends of their powers of two: 2^-127, 2^127 and NaN, whoever wrote the codes."""

import pytest
import torch

from tests import attend_util as U

pytestmark = pytest.mark.gpu
D = 128
LEVELS = torch.tensor([*U.LEVELS, *[-x for x in U.LEVELS]], dtype=torch.float64)


def stood_for(codes, scales):
    """[rows, 128] in 64 bits: code times 2^(scale - 127), NaN where the scale is 255."""
    c = codes.cpu().long()
    value = LEVELS[torch.stack([c & 15, c >> 4], -1).view(-1, 4, 32)]
    s = scales.cpu().double()[..., None]
    return torch.where(s == 255, float("nan"), value * torch.exp2(s - 127)).view(-1, D)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_every_scale_with_every_code(dtype):
    # 256 scales in each of a row's four blocks, rows of all 16 codes in every position
    codes = torch.arange(256 * 16, device="cuda")[:, None] % 16 + torch.arange(64, device="cuda")[None]
    codes = (codes % 16 + 16 * ((codes + 5) % 16)).to(torch.uint8)
    scales = (torch.arange(256 * 16, device="cuda")[:, None] // 16 + 64 * torch.arange(4, device="cuda")[None]).to(torch.uint8)
    out = torch.empty((256 * 16, D), dtype=U.dtype_of(dtype), device="cuda")
    with U.context(1, 1, dtype, 64) as ctx:
        ctx.expand_mx(codes, scales, 256 * 16, out)
        torch.cuda.synchronize()
    want, got = stood_for(codes, scales), out.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    beyond = want.abs() >= 2.0 ** 128                                  # (of scale 2^127 and of 2^126, which no gather makes: the type has no such numbers)
    assert bool((got[beyond].abs() == float("inf")).all()) and torch.equal(got[~beyond].nan_to_num(7.0), want[~beyond].nan_to_num(7.0))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kept", [1, 40])
def test_values_of_the_smallest_scale(dtype, kept):
    # one distinct row kept: the result is its value, subnormal or not.  Scores of rows of 2^-127 times queries of 2^126 tell them apart
    g = torch.Generator(device="cuda").manual_seed(kept)
    codes = [torch.randint(0, 256, (kept, 64), generator=g, device="cuda").to(torch.uint8) for _ in "KV"]
    codes[1][:] = codes[1][0]
    scales = torch.zeros((kept, 4), dtype=torch.uint8, device="cuda")
    Q = U.randn(1, (1, 1, 2, D), U.dtype_of(dtype)) * 2.0 ** 124
    out, lse = torch.empty_like(Q), torch.empty((2, 1), device="cuda")
    with U.context(1, 2, dtype, 64) as ctx:
        ctx.attend_kept_mx(Q, codes[0], scales, codes[1], scales, torch.tensor([0, kept], device="cuda"), 1, 1, kept, out, lse=lse)
        torch.cuda.synchronize()
    K, V = (stood_for(c, scales) for c in codes)
    # (weights that add up to their sum to within 2^-8 each in bf16, 2^-22 in fp32; then one rounding, to a multiple of 2^-133 or 2^-149)
    unit = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -20
    assert bool(((out[0, 0].double().cpu() - V[0]).abs() <= unit * V[0].abs() + (2.0 ** -133 if dtype == "bf16" else 2.0 ** -148)).all())
    for h in range(2):
        x = (K @ Q[0, 0, h].double().cpu()) * D ** -0.5
        off = 128 * 2.0 ** -24 * float((K.abs() @ Q[0, 0, h].double().cpu().abs()).max()) * D ** -0.5 + 2.0 ** -18
        assert abs(float(torch.logsumexp(x, 0)) - float(lse[h, 0])) <= off


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_block_of_nan_with_codes(dtype):
    codes = torch.full((32, 64), 0x52, dtype=torch.uint8, device="cuda")
    scales = torch.full((32, 4), 127, dtype=torch.uint8, device="cuda")
    bad = scales.clone()
    bad[3, 2] = 255
    Q = U.randn(1, (1, 1, 1, D), U.dtype_of(dtype))
    out, x = torch.empty_like(Q), torch.empty((32, D), dtype=Q.dtype, device="cuda")
    with U.context(1, 1, dtype, 64) as ctx:
        ctx.attend_kept_mx(Q, codes, scales, codes, bad, torch.tensor([0, 32], device="cuda"), 1, 1, 32, out)
        ctx.expand_mx(codes, bad, 32, x)
        torch.cuda.synchronize()
    assert torch.isnan(out[0, 0, 0]).nonzero()[:, 0].tolist() == [*range(64, 96)]
    assert torch.isnan(x).nonzero().tolist() == [[3, i] for i in range(64, 96)]
