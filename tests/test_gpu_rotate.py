"""Norms of queries and keys, rotation and the cache's new rows (curdkv_rotate) against the definition in 64 bits."""

import math

import numpy as np
import pytest
import torch

from paper_2509_15038_amd import binding as B
from tests import attend_util as U
from tests.gpu_util import Guarded

pytestmark = pytest.mark.gpu
D, EPS = 128, 1e-5


def table_of(rows):
    angle = torch.arange(rows, dtype=torch.float64, device="cuda")[:, None] * 10000.0 ** (-torch.arange(0, D, 2, device="cuda", dtype=torch.float64) / D)
    return torch.stack([angle.cos(), angle.sin()], 1).float().contiguous()


def check(dtype, count, kv, group, m, stride, pairs=False, q_norm=True, k_norm=True, starts=None, positions=None, row_stride=None, scale=1.0, rows=700):
    dt = U.dtype_of(dtype)
    heads = (group + 2) * kv
    wide = heads * D if row_stride is None else row_stride
    qkv = U.randn(1, (count * m, wide), dt, scale)
    table = table_of(rows)
    qw, kw = (U.randn(i, (D,), dt) if on else None for i, on in ((2, q_norm), (3, k_norm)))
    Q = Guarded((count * m * kv * group, D), dt, float("nan"))
    K, V = (Guarded((count * kv * stride, D), dt, 5.0) for _ in range(2))
    st = None if starts is None else torch.tensor(starts, dtype=torch.int32, device="cuda")
    at = None if positions is None else torch.tensor(positions, dtype=torch.int32, device="cuda")
    with U.context(kv, group, dtype, stride) as ctx:
        ctx.rotate(qkv, count, m, table, Q.t, K.t, V.t, stride, starts=st, positions=at, q_weight=qw, k_weight=kw, eps=EPS, pairs=pairs, row_stride=row_stride)
        torch.cuda.synchronize()
    for x in (Q, K, V):
        x.check()
    x = qkv.double()[:, : heads * D].view(count, m, heads, D)
    slots = torch.arange(m).view(1, m) + (torch.zeros((count, 1), dtype=torch.long) if starts is None else torch.tensor(starts).view(count, 1))
    where = (slots if positions is None else torch.tensor(positions).view(count, m)).clamp(0, rows - 1)
    turn = table.double()[where.cuda()][:, :, None]                     # [count, m, 1, 2, 64]
    lo, hi = (slice(0, D, 2), slice(1, D, 2)) if pairs else (slice(0, D // 2), slice(D // 2, D))

    def made(y, w):
        """(value, bound of its error in 32 bits, before the rounding to the storage type)"""
        r = torch.ones_like(y[..., :1])
        if w is not None:
            r = 1 / torch.sqrt(y.square().mean(-1, keepdim=True) + EPS)
            y = y * r * w.double()
        z, size = torch.empty_like(y), torch.empty_like(y)
        a, b, c, s = y[..., lo], y[..., hi], turn[..., 0, :], turn[..., 1, :]
        z[..., lo], z[..., hi] = a * c - b * s, b * c + a * s
        size[..., lo], size[..., hi] = (a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()
        return z, size

    unit = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24               # significands of 8 and 24 bits, rounded to nearest
    q, q_size = made(x[:, :, : kv * group], qw)
    k, k_size = made(x[:, :, kv * group: kv * (group + 1)], kw)

    def near(got, want, size):
        # the norm's sum of 128 squares, its root and quotient: below 128 / 2 + 8 units of 2^-24; products and their sum: 4; then one rounding
        off = (got.double() - want).abs()
        assert bool((off <= unit * 1.01 * want.abs() + 80 * 2.0 ** -24 * size + 1e-38).all()), float(off.max())

    near(Q.t.view(count, m, -1, D), q, q_size)
    Kc, Vc = K.t.view(count, kv, stride, D), V.t.view(count, kv, stride, D)
    written = torch.zeros((count, stride), dtype=torch.bool)
    for b in range(count):
        for i in range(m):
            j = int(slots[b, i])
            if 0 <= j < stride:
                written[b, j] = True
                near(Kc[b, :, j], k[b, i], k_size[b, i])
                assert torch.equal(Vc[b, :, j].double(), x[b, i, kv * (group + 1):])
    rest = ~written.cuda()[:, None, :, None].expand_as(Kc)
    assert bool((Kc[rest] == 5).all()) and bool((Vc[rest] == 5).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("q_norm,k_norm", [(True, True), (False, False), (True, False), (False, True)])
def test_norms_and_pairings(dtype, pairs, q_norm, k_norm):
    check(dtype, 2, 2, 4, 5, 9, pairs, q_norm, k_norm, starts=[0, 4], positions=[0, 1, 2, 3, 4, 699, 5, 650, 7, 8])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kv,group", [(1, 1), (8, 4), (1, 7), (3, 5), (2, 40)])
@pytest.mark.parametrize("count,m", [(1, 1), (3, 1), (1, 33), (4, 7)])
def test_sizes_and_layouts(dtype, kv, group, count, m):
    check(dtype, count, kv, group, m, m + 3)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_many_tokens(dtype):
    # (both kernels: one token a workgroup and four)
    check(dtype, 1, 1, 1, 699, 700)
    check(dtype, 7, 1, 1, 601, 601, pairs=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_row_stride_rows_outside_the_cache_and_positions_outside_the_table(dtype):
    check(dtype, 3, 2, 2, 4, 6, starts=[-2, 3, 6], positions=[-5, 0, 1, 2, 10 ** 9, 3, 4, 5, 6, 7, 8, 9], row_stride=8 * D + 24)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("scale", [0.0, 1e-20, 1e15])
def test_small_and_large_values(dtype, scale):
    check(dtype, 1, 1, 2, 3, 4, scale=scale)


def test_infinities_and_nan_stay_in_their_head():
    kv, group, m = 2, 2, 3
    qkv = U.randn(1, (m, 8 * D), torch.bfloat16)
    qkv[1, 5], qkv[1, 4 * D + 7] = math.nan, math.inf                  # query head 0 and key head 0 of token 1
    Q, K, V = torch.empty((m, 4, D), dtype=torch.bfloat16, device="cuda"), *(torch.empty((kv, m, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    w = torch.ones((D,), dtype=torch.bfloat16, device="cuda")
    with U.context(kv, group, "bf16", m) as ctx:
        ctx.rotate(qkv, 1, m, table_of(8), Q, K, V, m, q_weight=w, k_weight=w)
        torch.cuda.synchronize()
    bad_q, bad_k = ~torch.isfinite(Q.float()).all(-1), ~torch.isfinite(K.float()).all(-1)
    assert bad_q.nonzero().tolist() == [[1, 0]] and bad_k.nonzero().tolist() == [[0, 1]] and bool(torch.isfinite(V.float()).all())


def test_graph_and_other_stream():
    qkv, table = U.randn(1, (6, 6 * D), torch.bfloat16), table_of(64)
    starts = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    bufs = [[torch.zeros((2, 3, 4, D), dtype=torch.bfloat16, device="cuda"), *(torch.zeros((2, 1, 30, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))]
            for _ in range(2)]
    with U.context(1, 4, "bf16", 64) as ctx:
        call = lambda o, s=None: ctx.rotate(qkv, 2, 3, table, *o, 30, starts=starts, stream=s)
        graph = torch.cuda.CUDAGraph()
        call(bufs[1])
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            call(bufs[1])
        side = torch.cuda.Stream()
        for k in range(3):
            starts.add_(4)
            torch.cuda.synchronize()
            graph.replay()
            call(bufs[0], side)
            torch.cuda.synchronize()
            assert all(torch.equal(a[..., 9:, :] if a.shape[-2] == 30 else a, b[..., 9:, :] if b.shape[-2] == 30 else b) for a, b in zip(*bufs))


def test_refusals():
    qkv, table = U.randn(1, (2, 6 * D), torch.bfloat16), table_of(8)
    Q = torch.full((2, 4, D), 7.0, dtype=torch.bfloat16, device="cuda")
    K, V = (torch.full((1, 8, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    good = dict(qkv=qkv, count=1, m=2, table=table, Q=Q, K=K, V=V, stride=8)
    with U.context(1, 4, "bf16", 64) as ctx:
        for bad in (dict(qkv=None), dict(Q=None), dict(K=None), dict(V=None), dict(count=0), dict(m=0), dict(stride=0), dict(stride=65),
                    dict(row_stride=6 * D - 8), dict(row_stride=6 * D + 4), dict(table=table[:0]), dict(q_weight=Q, eps=-1.0), dict(k_weight=Q, eps=math.nan),
                    dict(qkv=qkv.data_ptr() + 2), dict(K=K.data_ptr() + 8)):
            with pytest.raises(B.CurdkvError) as e:
                ctx.rotate(**dict(good, **bad))
            assert e.value.code == B.ERR_INVALID_ARG, bad
        torch.cuda.synchronize()
        assert bool((Q == 7).all()) and bool((K == 7).all()) and bool((V == 7).all())
