"""Rotation by positions on several axes (curdkv_rotate_axes) against the definition in 64 bits, and against curdkv_rotate."""

import math

import numpy as np
import pytest
import torch

from tests import attend_util as U
from tests.gpu_util import Guarded
from tests.test_gpu_rotate import table_of

pytestmark = pytest.mark.gpu
D, EPS = 128, 1e-5


def run(dtype, count, kv, group, m, stride, qkv, table, positions, axis_of, pairs=False, qw=None, kw=None, starts=None, row_stride=None, stream=None, plain=False):
    dt = U.dtype_of(dtype)
    Q = Guarded((count * m * kv * group, D), dt, float("nan"))
    K, V = (Guarded((count * kv * stride, D), dt, 5.0) for _ in range(2))
    st = None if starts is None else torch.tensor(starts, dtype=torch.int32, device="cuda")
    with U.context(kv, group, dtype, stride) as ctx:
        how = dict(starts=st, q_weight=qw, k_weight=kw, eps=EPS, pairs=pairs, row_stride=row_stride, stream=stream)
        if plain:
            ctx.rotate(qkv, count, m, table, Q.t, K.t, V.t, stride, positions=positions[0].contiguous(), **how)
        else:
            ctx.rotate_axes(qkv, count, m, table, positions, axis_of, Q.t, K.t, V.t, stride, **how)
        torch.cuda.synchronize()
    for x in (Q, K, V):
        x.check()
    return Q.t.view(count, m, -1, D), K.t.view(count, kv, stride, D), V.t.view(count, kv, stride, D)


def check(dtype, count, kv, group, m, stride, axes, axis_of, pairs=False, norms=True, starts=None, positions=None, row_stride=None, rows=700, seed=0):
    dt, heads = U.dtype_of(dtype), (group + 2) * kv
    qkv = U.randn(seed + 1, (count * m, heads * D if row_stride is None else row_stride), dt)
    table = table_of(rows)
    qw, kw = (U.randn(seed + i, (D,), dt) if norms else None for i in (2, 3))
    rng = np.random.default_rng(seed)
    at = rng.integers(0, rows, (axes, count * m)).astype(np.int32) if positions is None else np.asarray(positions, dtype=np.int32)
    Q, K, V = run(dtype, count, kv, group, m, stride, qkv, table, torch.from_numpy(at).cuda(), axis_of, pairs, qw, kw, starts, row_stride)
    x = qkv.double()[:, : heads * D].view(count, m, heads, D)
    turn = table.double()[torch.from_numpy(at).long().clamp(0, rows - 1).cuda()]      # [axes, tokens, 2, 64]
    axis = torch.from_numpy(axis_of).long().cuda()
    turn = torch.stack([turn[int(axis[i]), :, :, i] for i in range(64)], -1).view(count, m, 1, 2, 64)
    lo, hi = (slice(0, D, 2), slice(1, D, 2)) if pairs else (slice(0, D // 2), slice(D // 2, D))
    unit = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24

    def near(got, y, w, c, s):
        if w is not None:
            y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + EPS) * w.double()
        a, b = y[..., lo], y[..., hi]
        for part, want, size in ((lo, a * c - b * s, (a * c).abs() + (b * s).abs()), (hi, b * c + a * s, (b * c).abs() + (a * s).abs())):
            # (as for curdkv_rotate: the norm below 72 units of 2^-24, products and sums 4, one rounding)
            off = (got[..., part].double() - want).abs()
            assert bool((off <= unit * 1.01 * want.abs() + 80 * 2.0 ** -24 * size + 1e-38).all()), float(off.max())

    near(Q, x[:, :, : kv * group], qw, turn[..., 0, :], turn[..., 1, :])
    start = [0] * count if starts is None else starts
    written = torch.zeros((count, stride), dtype=torch.bool)
    for b in range(count):
        for i in range(m):
            j = start[b] + i
            if 0 <= j < stride:
                written[b, j] = True
                near(K[b, :, j], x[b, i, kv * group: kv * (group + 1)], kw, turn[b, i, :, 0], turn[b, i, :, 1])
                assert torch.equal(V[b, :, j].double(), x[b, i, kv * (group + 1):])
    rest = ~written.cuda()[:, None, :, None].expand_as(K)
    assert bool((K[rest] == 5).all()) and bool((V[rest] == 5).all())


SECTIONS = np.repeat([0, 1, 2], [16, 24, 24]).astype(np.uint8)
ODD = np.repeat([2, 0, 1], [13, 40, 11]).astype(np.uint8)              # stretches that end inside a lane's eight angles
MIXED = (np.arange(64) % 3).astype(np.uint8)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("axis_of", [SECTIONS, ODD, MIXED], ids=["stretches", "odd", "mixed"])
def test_layouts_of_axes(dtype, pairs, axis_of):
    check(dtype, 2, 2, 4, 5, 9, 3, axis_of, pairs, starts=[0, 4])
    check(dtype, 1, 1, 7, 33, 40, 3, axis_of, pairs, norms=False)


@pytest.mark.parametrize("axes", [1, 2, 3, 4])
def test_numbers_of_axes(axes):
    check("bf16", 1, 3, 5, 7, 8, axes, (np.arange(64) * 7 % axes).astype(np.uint8))
    check("fp32", 1, 1, 1, 1, 1, axes, np.sort(np.arange(64) % axes).astype(np.uint8)[::-1].copy())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("axis_of", [SECTIONS, MIXED], ids=["stretches", "mixed"])
def test_many_tokens(dtype, axis_of):
    check(dtype, 7, 1, 1, 601, 601, 3, axis_of, pairs=True)            # (four tokens a workgroup)


def test_row_stride_rows_outside_the_cache_and_positions_outside_the_table():
    where = [[-5, 0, 1, 2, 10 ** 9, 3, 4, 5, 6, 7, 8, 9], [0, -2 ** 31, 1, 2, 3, 3, 2 ** 31 - 1, 5, 6, 7, 699, 700]]
    check("bf16", 3, 2, 2, 4, 6, 2, (np.arange(64) % 2).astype(np.uint8), starts=[-2, 3, 6], positions=where, row_stride=8 * D + 24)
    check("fp32", 3, 2, 2, 4, 6, 2, np.repeat([0, 1], [40, 24]).astype(np.uint8), starts=[-2, 3, 6], positions=where, row_stride=8 * D + 24)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_the_same_position_on_all_axes_is_rotate(dtype):
    for m, axis_of in ((1, MIXED), (70, SECTIONS), (5000, MIXED)):
        qkv = U.randn(1, (m, 6 * D), U.dtype_of(dtype))
        w = U.randn(2, (D,), U.dtype_of(dtype))
        at = torch.randint(0, 300, (1, m), dtype=torch.int32, device="cuda").expand(3, m).contiguous()
        for pairs in (False, True):
            got = run(dtype, 1, 1, 4, m, m, qkv, table_of(300), at, axis_of, pairs, w, w)
            want = run(dtype, 1, 1, 4, m, m, qkv, table_of(300), at, axis_of, pairs, w, w, plain=True)
            for x, y in zip(got, want):
                assert torch.equal(x, y)


def test_infinities_and_nan_stay_in_their_head():
    qkv = U.randn(1, (3, 8 * D), torch.bfloat16)
    qkv[1, 5], qkv[1, 4 * D + 7] = math.nan, math.inf                  # query head 0 and key head 0 of token 1
    at = torch.zeros((3, 3), dtype=torch.int32, device="cuda")
    Q, K, V = run("bf16", 1, 2, 2, 3, 3, qkv, table_of(5), at, MIXED)
    bad_q, bad_k = ~torch.isfinite(Q), ~torch.isfinite(K)
    assert bool(bad_q[0, 1, 0].any()) and int(bad_q.sum()) == int(bad_q[0, 1, 0].sum())
    assert bool(bad_k[0, 0, 1].any()) and int(bad_k.sum()) == int(bad_k[0, 0, 1].sum())


def test_another_stream_and_the_list_of_axes_is_read_before_the_call_returns():
    qkv = U.randn(1, (50, 6 * D), torch.bfloat16)
    at = torch.randint(0, 300, (3, 50), dtype=torch.int32, device="cuda")
    table = table_of(300)
    want = run("bf16", 1, 1, 4, 50, 50, qkv, table, at, MIXED)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    Q, K, V = torch.empty_like(want[0]), torch.empty_like(want[1]), torch.empty_like(want[2])
    axis = MIXED.copy()
    with U.context(1, 4, "bf16", 50) as ctx:
        ctx.rotate_axes(qkv, 1, 50, table, at, axis, Q, K, V, 50, stream=side)
        axis[:] = 0
        side.synchronize()
        for x, y in zip((Q, K, V), want):
            assert torch.equal(x, y)
