"""Attention over kept rows and the tokens since (curdkv_attend_kept, curdkv_attend_kept_mx) against its definition in 64 bits."""

import math

import numpy as np
import pytest
import torch

from paper_2509_15038_amd import binding as B
from tests import attend_util as U
from tests.gpu_util import Guarded

pytestmark = pytest.mark.gpu
D = 128


def pack(ctx_dtype, rows):
    """Codes and scales of rows, through curdkv_compact_mx with identity indices, and the values they stand for."""
    n = max(1, rows.shape[0])
    if not rows.shape[0]:
        return torch.empty((0, 64), dtype=torch.uint8, device="cuda"), torch.empty((0, 4), dtype=torch.uint8, device="cuda"), rows.double()
    codes, scales = torch.empty((n, 64), dtype=torch.uint8, device="cuda"), torch.empty((n, 4), dtype=torch.uint8, device="cuda")
    with U.context(1, 1, ctx_dtype, n) as ctx:
        ctx.compact_mx(rows, rows, n, torch.arange(n, dtype=torch.int32, device="cuda"), torch.tensor([0, n], device="cuda"), n, codes, scales, codes.clone(), scales.clone())
        torch.cuda.synchronize()
    value, want_codes, want_scales = U.four_bits(rows)
    assert torch.equal(scales.cpu(), want_scales) and torch.equal(codes.cpu(), want_codes)
    return codes, scales, value.cuda()


def check(dtype, mx, count, kv, group, m, budgets, tail_n, tails, seed=0, before=0, spoil=None, stream=None, tail_stride=None, rows_known=True):
    """budgets: kept rows of every head; before: rows of other layers in front of them in the packed arrays; rows_known: the call is told how many are its
    heads'."""
    dt, budgets = U.dtype_of(dtype), np.asarray(budgets)
    off = before + np.concatenate([[0], np.cumsum(budgets)]).astype(np.int64)
    total = int(off[-1])
    Kk, Vk = U.randn(seed + 1, (total, D), dt), U.randn(seed + 2, (total, D), dt)
    tail_stride = tail_n if tail_stride is None else tail_stride
    Kt, Vt = (U.randn(seed + i, (count, kv, tail_stride, D), dt) for i in (3, 4))
    lens = np.full(count, tail_n) if tails is None else np.asarray(tails)
    for b in range(count):
        Kt[b, :, int(lens[b]):], Vt[b, :, int(lens[b]):] = math.nan, math.inf
    if spoil:
        spoil(Kk, Vk, Kt, Vt)
    Q = U.randn(seed + 5, (count, m, kv * group, D), dt)
    offsets = torch.from_numpy(off).cuda()
    out = Guarded((count * m * kv * group, D), dt, float("nan"))
    lse = Guarded((count * kv * group, m), torch.float32, float("nan"))
    since = dict(K_tail=Kt, V_tail=Vt, tail_n=tail_n, tail_stride=tail_stride, lse=lse.t, stream=stream, rows=int(budgets.sum()) if rows_known else None,
                 tail_lengths=None if tails is None else torch.from_numpy(lens.astype(np.int32)).cuda())
    with U.context(kv, group, dtype, max(tail_n, m, 1)) as ctx:
        if mx:
            Kc, Ks, Kk = pack(dtype, Kk)
            Vc, Vs, Vk = pack(dtype, Vk)
            ctx.attend_kept_mx(Q, Kc, Ks, Vc, Vs, offsets, count, m, total, out.t, **since)
        else:
            ctx.attend_kept(Q, Kk, Vk, offsets, count, m, total, out.t, **since)
        torch.cuda.synchronize()
    out.check("out")
    lse.check("lse")
    o, l = out.t.view(count, m, -1, D), lse.t.view(count, -1, m)
    for b in range(count):
        tail = U.causal(m, tail_n, int(lens[b]), 0, 0)
        for h in range(kv * group):
            g = b * kv + h // group
            k = torch.cat([Kk[off[g]: off[g + 1]].double(), Kt[b, h // group, :tail_n].double()])
            v = torch.cat([Vk[off[g]: off[g + 1]].double(), Vt[b, h // group, :tail_n].double()])
            seen = torch.cat([torch.ones((m, budgets[g]), dtype=torch.bool, device="cuda"), tail], 1)
            fine = ~(seen & ~(torch.isfinite(k).all(1) & torch.isfinite(v).all(1))).any(1)
            want = U.attention(Q[b, fine, h], k, v, seen[fine], D ** -0.5)
            U.check_attention(o[b, fine, h], l[b, h, fine], want, dtype, k.shape[0], f"seq {b} head {h} budget {budgets[g]} tail {lens[b]}")
            if spoil is None:
                assert bool(fine.all())
    return o, l


FORMS = [("bf16", False), ("bf16", True), ("fp32", False), ("fp32", True)]


@pytest.mark.parametrize("dtype,mx", FORMS)
@pytest.mark.parametrize("kept,tail", [(1, 1), (0, 1), (1, 0), (0, 0), (15, 3), (16, 16), (17, 31), (32, 33), (33, 1), (127, 64), (129, 65), (1000, 200), (5001, 7)])
def test_sizes(dtype, mx, kept, tail):
    check(dtype, mx, 2, 2, 4, 1, [kept] * 4, tail, None, seed=kept + tail)


@pytest.mark.parametrize("dtype,mx", FORMS)
@pytest.mark.parametrize("m", [1, 2, 3, 4, 5, 9])
def test_uneven_heads_ragged_tails_and_drafts(dtype, mx, m):
    budgets = [0, 1, 2500, 31, 300, 0, 33, 64, 700]
    check(dtype, mx, 3, 3, 4, m, budgets, 40, [40, 0, 3], seed=m, tail_stride=47)


@pytest.mark.parametrize("dtype,mx", FORMS)
@pytest.mark.parametrize("kv,group", [(1, 1), (1, 7), (2, 16), (1, 20)])
def test_head_layouts(dtype, mx, kv, group):
    check(dtype, mx, 2, kv, group, 2, [77 + 50 * i for i in range(2 * kv)], 9, None, seed=group)


@pytest.mark.parametrize("dtype,mx", FORMS)
def test_a_layer_of_a_larger_packed_cache(dtype, mx):
    check(dtype, mx, 1, 4, 2, 1, [100, 50, 0, 257], 5, None, before=333)


@pytest.mark.parametrize("dtype,mx", FORMS)
@pytest.mark.parametrize("m", [2, 5])
def test_infinities_and_nan_in_hidden_rows(dtype, mx, m):
    def spoil(Kk, Vk, Kt, Vt):
        Kt[:, :, -1], Vt[:, :, -1] = math.inf, math.nan               # the last token's own row
        Vk[:, 3] = Vk[:, 3]

    check(dtype, mx, 2, 2, 4, m, [90, 100, 33, 64], 20, None, spoil=spoil)


def test_a_block_of_nan_kept():
    # a kept row that was not finite stands for NaN and is seen by everybody of its head, and by nobody else
    K = U.randn(1, (64, D), torch.bfloat16)
    V = U.randn(2, (64, D), torch.bfloat16)
    V[5, 40] = math.inf
    Kc, Ks, Kv = pack("bf16", K)
    Vc, Vs, _ = pack("bf16", V)
    Q = U.randn(3, (1, 1, 2, D), torch.bfloat16)
    out = torch.empty_like(Q)
    with U.context(2, 1, "bf16", 64) as ctx:
        ctx.attend_kept_mx(Q, Kc, Ks, Vc, Vs, torch.tensor([0, 32, 64], device="cuda"), 1, 1, 64, out)
        torch.cuda.synchronize()
    assert bool(torch.isnan(out[0, 0, 0, 32:64]).all()) and bool(torch.isfinite(out[0, 0, 0, :32].float()).all())
    assert bool(torch.isfinite(out[0, 0, 0, 64:].float()).all()) and bool(torch.isfinite(out[0, 0, 1].float()).all())


@pytest.mark.parametrize("mx", [False, True])
def test_offsets_beyond_two_to_the_31(mx):
    # rows whose element (bf16) and byte (codes) offsets pass 32 bits; only the last rows of the array are written and kept
    rows = 2 ** 31 // D + 300 if not mx else 2 ** 32 // 64 + 300
    n, first = 250, rows - 250
    K, V, Q = U.randn(1, (n, D), torch.bfloat16), U.randn(2, (n, D), torch.bfloat16), U.randn(3, (1, 1, 4, D), torch.bfloat16)
    out = torch.empty_like(Q)
    offsets = torch.tensor([first, rows], device="cuda")
    with U.context(1, 4, "bf16", 64) as ctx:
        if mx:
            arrays = []
            for x in (K, V):
                codes, scales, value = pack("bf16", x)
                far = [torch.empty((rows, w), dtype=torch.uint8, device="cuda") for w in (64, 4)]
                far[0][first:], far[1][first:] = codes, scales
                arrays.append((far, value))
            (k, Kv), (v, Vv) = arrays
            ctx.attend_kept_mx(Q, *k, *v, offsets, 1, 1, rows, out)
        else:
            k, v = (torch.empty((rows, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
            k[first:], v[first:] = K, V
            Kv, Vv = K, V
            ctx.attend_kept(Q, k, v, offsets, 1, 1, rows, out)
        torch.cuda.synchronize()
    for h in range(4):
        want = U.attention(Q[0, :, h], Kv, Vv, torch.ones((1, n), dtype=torch.bool, device="cuda"), D ** -0.5)
        U.check_attention(out[0, :, h], None, want, "bf16", n)


@pytest.mark.parametrize("mx", [False, True])
def test_graph_and_other_stream(mx):
    total, count, kv = 6000, 2, 2
    Kk, Vk = U.randn(1, (total, D), torch.bfloat16), U.randn(2, (total, D), torch.bfloat16)
    offsets = torch.tensor([0, 3000, 3001, 4000, 6000], device="cuda")
    Kt, Vt = (U.randn(i, (count, kv, 64, D), torch.bfloat16) for i in (3, 4))
    lengths = torch.tensor([5, 64], dtype=torch.int32, device="cuda")
    Q = U.randn(5, (count, 1, 8, D), torch.bfloat16)
    packed = [pack("bf16", x)[:2] for x in (Kk, Vk)] if mx else None
    with U.context(kv, 4, "bf16", 64) as ctx:
        def call(out, stream=None):
            since = dict(K_tail=Kt, V_tail=Vt, tail_n=64, tail_stride=64, tail_lengths=lengths, stream=stream)
            if mx:
                ctx.attend_kept_mx(Q, *packed[0], *packed[1], offsets, count, 1, total, out, **since)
            else:
                ctx.attend_kept(Q, Kk, Vk, offsets, count, 1, total, out, **since)
        a, b, c = (torch.empty_like(Q) for _ in range(3))
        call(a)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        call(b, side)
        torch.cuda.synchronize()
        assert torch.equal(a, b)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(c)
        for k in range(3):                                             # tails grow between the replays, as they do while tokens are generated
            lengths.add_(torch.tensor([7, 0], dtype=torch.int32, device="cuda"))
            Q.copy_(U.randn(20 + k, Q.shape, torch.bfloat16))
            graph.replay()
            torch.cuda.synchronize()
            call(a)
            torch.cuda.synchronize()
            assert torch.equal(a, c)


def test_refusals():
    K, Q = U.randn(1, (64, D), torch.bfloat16), U.randn(3, (1, 1, 4, D), torch.bfloat16)
    codes, scales = torch.zeros((64, 64), dtype=torch.uint8, device="cuda"), torch.zeros((64, 4), dtype=torch.uint8, device="cuda")
    off, out = torch.tensor([0, 64], device="cuda"), torch.full_like(Q, 7.0)
    with U.context(1, 4, "bf16", 64) as ctx:
        good = dict(Q=Q, K_kept=K, V_kept=K, offsets=off, count=1, m=1, total=64, out=out)
        for bad in (dict(Q=None), dict(K_kept=None), dict(V_kept=None), dict(offsets=None), dict(out=None), dict(total=-1), dict(rows=-1), dict(rows=65), dict(count=0), dict(m=0),
                    dict(tail_n=1, tail_stride=1), dict(K_tail=K, V_tail=K, tail_n=2, tail_stride=1), dict(K_tail=K, V_tail=K, tail_n=-1),
                    dict(K_tail=K, V_tail=K, tail_n=65, tail_stride=65), dict(scale=0.0), dict(K_kept=K.data_ptr() + 8)):
            with pytest.raises(B.CurdkvError) as e:
                ctx.attend_kept(**dict(good, **bad))
            assert e.value.code == B.ERR_INVALID_ARG, bad
        good = dict(Q=Q, K_codes=codes, K_scales=scales, V_codes=codes, V_scales=scales, offsets=off, count=1, m=1, total=64, out=out)
        for bad in (dict(K_codes=None), dict(K_scales=None), dict(V_codes=None), dict(V_scales=None), dict(K_codes=codes.data_ptr() + 4)):
            with pytest.raises(B.CurdkvError) as e:
                ctx.attend_kept_mx(**dict(good, **bad))
            assert e.value.code == B.ERR_INVALID_ARG, bad
        torch.cuda.synchronize()
        assert bool((out == 7).all())


@pytest.mark.parametrize("mx", [False, True])
def test_more_new_tokens_than_any_cache_holds(mx):
    # max_tokens bounds caches and tails; the tokens that look at kept rows may be more
    K, V, Q = (U.randn(i, (70, D) if i < 3 else (1, 6, 4, D), torch.bfloat16) for i in (1, 2, 3))
    Kt, Vt, off, out = K[:1].clone(), V[:1].clone(), torch.tensor([0, 70], device="cuda"), torch.empty_like(Q)
    with U.context(1, 4, "bf16", 1) as ctx:
        if mx:
            (Kc, Ks, k), (Vc, Vs, v) = pack("bf16", K), pack("bf16", V)
            ctx.attend_kept_mx(Q, Kc, Ks, Vc, Vs, off, 1, 6, 70, out, K_tail=Kt, V_tail=Vt, tail_n=1, tail_stride=1)
        else:
            k, v = K, V
            ctx.attend_kept(Q, K, V, off, 1, 6, 70, out, K_tail=Kt, V_tail=Vt, tail_n=1, tail_stride=1)
        torch.cuda.synchronize()
    seen = torch.cat([torch.ones((6, 70), dtype=torch.bool, device="cuda"), U.causal(6, 1, 1, 0, 0)], 1)
    for h in range(4):
        want = U.attention(Q[0, :, h], torch.cat([k.double(), Kt.double()]), torch.cat([v.double(), Vt.double()]), seen, D ** -0.5)
        U.check_attention(out[0, :, h], None, want, "bf16", 71)


@pytest.mark.parametrize("dtype,mx", FORMS)
@pytest.mark.parametrize("count,kv,m,budgets,tail,tails", [
    (2, 2, 300, [64, 128, 1000, 0], 300, None), (2, 2, 333, [1, 63, 65, 700], 400, [400, 90]), (1, 2, 70, [6000, 3001], 70, None), (1, 1, 500, [0], 500, None),
    (1, 2, 200, [640, 6400], 0, None), (3, 2, 130, [130, 64, 0, 31, 2000, 192], 131, [131, 0, 130]), (1, 8, 1000, [300, 64, 5, 1, 0, 700, 128, 60], 1000, None)])
def test_prompts_over_kept_rows(dtype, mx, count, kv, m, budgets, tail, tails):
    check(dtype, mx, count, kv, 4, m, budgets, tail, tails, seed=m)


@pytest.mark.parametrize("row", [3, 63, 64, 127, 129])
def test_a_prompt_over_kept_rows_that_are_not_finite(row):
    # everybody sees kept rows: an infinity of a value reaches every result of its channel, in whole tiles and the last one, and no other channel
    m, kept = 300, 130
    K, V, Q = (U.randn(i, (kept, D) if i < 3 else (1, m, 4, D), torch.bfloat16) for i in (1, 2, 3))
    V[row, 17], V[row, 90] = math.inf, math.nan
    Kt, Vt = U.randn(4, (1, 1, m, D), torch.bfloat16), U.randn(5, (1, 1, m, D), torch.bfloat16)
    Kt[0, 0, -1], Vt[0, 0, -1] = math.nan, math.inf                                     # the last token's own row, hidden from the others
    out = torch.empty_like(Q)
    with U.context(1, 4, "bf16", m) as ctx:
        ctx.attend_kept(Q, K, V, torch.tensor([0, kept], device="cuda"), 1, m, kept, out, K_tail=Kt, V_tail=Vt, tail_n=m, tail_stride=m)
        torch.cuda.synchronize()
    seen = torch.cat([torch.ones((m, kept), dtype=torch.bool, device="cuda"), U.causal(m, m, m, 0, 0)], 1)[:-1]
    clean = torch.where(torch.isfinite(V), V, 0.0)
    for h in range(4):
        got = out[0, :-1, h].double()
        assert bool((got[:, 17] == math.inf).all()) and bool(torch.isnan(got[:, 90]).all())
        want = U.attention(Q[0, :-1, h], torch.cat([K, Kt[0, 0]])[:, :], torch.cat([clean, Vt[0, 0]]), seen, D ** -0.5)
        got[:, 17], got[:, 90] = want[0][:, 17], want[0][:, 90]
        U.check_attention(got, None, want, "bf16", kept + m)
