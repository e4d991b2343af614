"""Attention of sequences that share their kept rows (curdkv_attend_shared, curdkv_attend_shared_mx) against its definition in 64 bits."""

import math

import numpy as np
import pytest
import torch

from paper_2509_15038_amd import binding as B
from tests import attend_util as U
from tests.gpu_util import Guarded
from tests.test_gpu_attend_kept import pack

pytestmark = pytest.mark.gpu
D = 128


def check(dtype, mx, count, share, kv, group, m, budgets, tail_n=0, tails=None, seed=0, before=0, spoil=None, stream=None, tail_stride=None, rows_known=True, scale=D ** -0.5,
          heads=None, with_lse=True):
    """budgets: kept rows of every prefix's head; before: rows of other layers in front of them; heads: how many query heads of each sequence are checked (all)."""
    dt, budgets, every = U.dtype_of(dtype), np.asarray(budgets), count * share
    off = before + np.concatenate([[0], np.cumsum(budgets)]).astype(np.int64)
    total = int(off[-1])
    Kk, Vk = U.randn(seed + 1, (total, D), dt), U.randn(seed + 2, (total, D), dt)
    tail_stride = tail_n if tail_stride is None else tail_stride
    Kt, Vt = (U.randn(seed + i, (every, kv, tail_stride, D), dt) for i in (3, 4))
    lens = np.full(every, tail_n) if tails is None else np.asarray(tails)
    for b in range(every):
        Kt[b, :, int(lens[b]):], Vt[b, :, int(lens[b]):] = math.nan, math.inf
    if spoil:
        spoil(Kk, Vk, Kt, Vt)
    Q = U.randn(seed + 5, (every, m, kv * group, D), dt)
    out = Guarded((every * m * kv * group, D), dt, float("nan"))
    lse = Guarded((every * kv * group, m), torch.float32, float("nan"))
    since = dict(K_tail=Kt, V_tail=Vt, tail_n=tail_n, tail_stride=tail_stride, lse=lse.t if with_lse else None, stream=stream, rows=int(budgets.sum()) if rows_known else None,
                 tail_lengths=None if tails is None else torch.from_numpy(lens.astype(np.int32)).cuda(), scale=scale)
    offsets = torch.from_numpy(off).cuda()
    with U.context(kv, group, dtype, max(tail_n, m, 1)) as ctx:
        if mx:
            Kc, Ks, Kk = pack(dtype, Kk)
            Vc, Vs, Vk = pack(dtype, Vk)
            ctx.attend_shared_mx(Q, Kc, Ks, Vc, Vs, offsets, count, share, m, total, out.t, **since)
        else:
            ctx.attend_shared(Q, Kk, Vk, offsets, count, share, m, total, out.t, **since)
        torch.cuda.synchronize()
    out.check("out")
    lse.check("lse")
    got, got_lse = out.t.view(every, m, kv * group, D), lse.t.view(every, kv * group, m)
    for b in range(every):
        L = int(min(max(lens[b], 0), tail_n))
        for h in range(kv * group if heads is None else heads):
            a, z = off[b // share * kv + h // group], off[b // share * kv + h // group + 1]
            k = torch.cat([Kk[a:z].double(), Kt[b, h // group, :L].double()])
            v = torch.cat([Vk[a:z].double(), Vt[b, h // group, :L].double()])
            seen = torch.cat([torch.ones((m, z - a), dtype=torch.bool, device="cuda"), U.causal(m, L, L, 0, 0)], 1)
            want = U.attention(Q[b, :, h], k, v, seen, scale)
            U.check_attention(got[b, :, h], got_lse[b, h] if with_lse else None, want, dtype, k.shape[0] + 64, f"sequence {b}, tail {L}, head {h}")
    if not with_lse:
        assert bool(lse.t.isnan().all())
    return got, got_lse


FORMS = [("bf16", False), ("bf16", True), ("fp32", False), ("fp32", True)]


@pytest.mark.parametrize("dtype,mx", FORMS)
@pytest.mark.parametrize("kv,group", [(1, 1), (8, 4), (2, 7), (1, 40)])
@pytest.mark.parametrize("share,m", [(1, 1), (3, 1), (5, 3)])
def test_layouts(dtype, mx, kv, group, share, m):
    rng = np.random.default_rng(kv)
    check(dtype, mx, 2, share, kv, group, m, rng.integers(0, 150, 2 * kv), 37, rng.integers(0, 38, 2 * share))


@pytest.mark.parametrize("dtype,mx", FORMS)
@pytest.mark.parametrize("keep", [0, 1, 31, 32, 33, 63, 64, 65, 127, 129, 300, 1100])
@pytest.mark.parametrize("share", [2, 40])
def test_lengths_of_prefixes(dtype, mx, keep, share):
    check(dtype, mx, 1, share, 2, 4, 1, [keep, keep // 2], 5, heads=8 if share == 2 else 3)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m", [1, 2, 9, 33])
def test_lengths_of_tails(dtype, m):
    tails = [0, 1, 2, 31, 32, 33, 63, 64, 65, 128, 129, 200]
    check(dtype, False, 2, 6, 1, 4, m, [70, 0], 200, tails, tail_stride=211)
    check(dtype, False, 2, 6, 1, 4, m, [0, 0], 200, tails)


@pytest.mark.parametrize("dtype,mx", FORMS)
def test_nothing_kept_and_no_tail(dtype, mx):
    got, lse = check(dtype, mx, 2, 3, 2, 4, 2, [0, 0, 0, 0])
    assert bool((got == 0).all()) and bool((lse == -math.inf).all())
    check(dtype, mx, 2, 3, 2, 4, 2, [5, 0, 0, 70])
    check(dtype, mx, 2, 3, 2, 4, 2, [5, 0, 0, 70], 9, [0, 9, 1, 2, 0, 5], with_lse=False)


@pytest.mark.parametrize("dtype,mx", FORMS)
def test_tails_shorter_than_the_new_tokens(dtype, mx):
    # (the first tokens see no tail, and where nothing is kept, nothing)
    check(dtype, mx, 2, 4, 1, 4, 6, [0, 40], 8, [0, 2, 5, 6, 3, 8, 1, 0])


@pytest.mark.parametrize("dtype,mx", FORMS)
def test_a_layer_of_a_larger_packed_cache(dtype, mx):
    check(dtype, mx, 1, 5, 2, 4, 1, [200, 90], 20, before=333)
    check(dtype, mx, 1, 5, 2, 4, 1, [200, 90], 20, before=333, rows_known=False)


@pytest.mark.parametrize("dtype,mx", FORMS)
@pytest.mark.parametrize("share,m,group", [(8, 1, 4), (9, 1, 4), (32, 1, 4), (33, 1, 4), (64, 1, 4), (11, 5, 7)])
def test_rows_at_the_edges_of_tiles(dtype, mx, share, m, group):
    check(dtype, mx, 1, share, 1, group, m, [777], 70, np.arange(share) * 7 % 71, heads=2)


@pytest.mark.parametrize("dtype,mx", FORMS)
def test_long_prefixes_in_parts(dtype, mx):
    check(dtype, mx, 1, 16, 2, 4, 1, [9001, 40], 130, heads=5, seed=9)
    check(dtype, mx, 2, 2, 1, 4, 1, [20000, 123], 13, seed=8)


@pytest.mark.parametrize("dtype,mx", [("bf16", False), ("fp32", False), ("bf16", True)])
def test_more_rows_than_scratch_holds(dtype, mx):
    # 36864 rows of two partial results each: prefixes, sequences and tokens in turn
    check(dtype, mx, 5, 60, 8, 32, 1, np.full(40, 33), 3, heads=2)
    check(dtype, mx, 1, 200, 8, 32, 1, np.full(8, 33), 3, heads=2)
    check(dtype, mx, 1, 2, 8, 32, 150, np.full(8, 33), 151, [151, 140], heads=2)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("share,m", [(2, 1), (2, 4), (40, 3)])
def test_values_that_are_not_finite(dtype, share, m):
    # in a kept row: all tokens' channel; in a tail's: those of the tokens that see it, of that sequence alone; in rows behind the lengths: nobody's
    def spoil(Kk, Vk, Kt, Vt):
        Vk[3, 5], Vk[69, 7], Vk[40, 9] = math.inf, -math.inf, math.nan
        Vt[1, 0, 49, 11] = math.inf
        if m > 1:
            Vt[0, 0, 48, 13] = -math.inf
            Vt[0, 0, 47, 17], Vt[0, 0, 49, 17] = math.inf, -math.inf
    dt, every = U.dtype_of(dtype), share
    clean = {}
    for name, f in (("clean", None), ("spoiled", spoil)):
        Kk, Vk = U.randn(1, (70, D), dt), U.randn(2, (70, D), dt)
        Kt, Vt = (U.randn(i, (every, 1, 60, D), dt) for i in (3, 4))
        Kt[:, :, 50:], Vt[:, :, 50:] = math.nan, math.inf
        if f:
            f(Kk, Vk, Kt, Vt)
        Q = U.randn(5, (every, m, 4, D), dt)
        out = torch.empty_like(Q)
        with U.context(1, 4, dtype, 60) as ctx:
            ctx.attend_shared(Q, Kk, Vk, torch.tensor([0, 70], device="cuda"), 1, share, m, 70, out, K_tail=Kt, V_tail=Vt, tail_n=60, tail_stride=60,
                              tail_lengths=torch.full((every,), 50, dtype=torch.int32, device="cuda"))
            torch.cuda.synchronize()
        clean[name] = out.double()
    a, b = clean["clean"], clean["spoiled"]
    touched = torch.zeros_like(a, dtype=torch.bool)
    touched[..., [5, 7, 9]] = True
    touched[1, m - 1, :, 11] = True
    assert bool((b[..., 5] == math.inf).all()) and bool((b[..., 7] == -math.inf).all()) and bool(b[..., 9].isnan().all())
    assert bool((b[1, m - 1, :, 11] == math.inf).all())
    if m > 1:
        touched[0, m - 2:, :, 13] = True
        touched[0, m - 3 if m > 2 else 0:, :, 17] = True
        assert bool((b[0, m - 2:, :, 13] == -math.inf).all()) and bool(b[0, m - 1, :, 17].isnan().all())
        if m > 2:
            assert bool((b[0, m - 3:m - 1, :, 17] == math.inf).all())
    assert torch.equal(a[~touched], b[~touched])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("share", [2, 40])
def test_scores_that_are_not_finite(dtype, share):
    dt = U.dtype_of(dtype)

    def run(f, kept=70):
        Kk, Vk = U.randn(1, (kept, D), dt), U.randn(2, (kept, D), dt)
        Kt, Vt = (U.randn(i, (share, 1, 9, D), dt) for i in (3, 4))
        Q = U.randn(5, (share, 1, 4, D), dt)
        Q[..., 0] = Q[..., 0].abs() + 0.1
        f(Kk, Kt)
        out, lse = torch.empty_like(Q), torch.empty((share, 4, 1), device="cuda")
        with U.context(1, 4, dtype, 60) as ctx:
            ctx.attend_shared(Q, Kk, Vk, torch.tensor([0, kept], device="cuda"), 1, share, 1, kept, out, K_tail=Kt, V_tail=Vt, tail_n=9, tail_stride=9, lse=lse)
            torch.cuda.synchronize()
        return out, lse

    def nan_key(Kk, Kt):
        Kk[69, 3] = math.nan
    out, lse = run(nan_key)
    assert bool(out.isnan().all()) and bool(lse.isnan().all())

    def inf_key(Kk, Kt):
        Kk[1, 0] = math.inf
    out, lse = run(inf_key)
    assert bool(out.isnan().all()) and bool(lse.isnan().all())

    def nan_tail(Kk, Kt):
        Kt[1, 0, 4, 2] = math.nan
    out, lse = run(nan_tail)
    assert bool(out[1].isnan().all()) and bool(lse[1].isnan().all()) and bool(torch.isfinite(out[0]).all()) and int(lse.isnan().sum()) == 4

    # keys that score -infinity weigh nothing, wherever they are; all of them: zeros and -infinity
    def none(Kk, Kt):
        pass
    whole, whole_lse = run(none, 40)

    def first_tiles(Kk, Kt):
        Kk[: Kk.shape[0] // 2, 0] = -math.inf

    def all_kept(Kk, Kt):
        Kk[:, 0] = -math.inf

    def all_keys(Kk, Kt):
        Kk[:, 0], Kt[..., 0] = -math.inf, -math.inf
    out, lse = run(all_keys)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    out, lse = run(first_tiles, 300)
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
    out, lse = run(all_kept, 300)
    out0, lse0 = run(none, 0)
    assert torch.equal(out, out0) and torch.equal(lse, lse0)


def test_scales_of_255_make_nan():
    Kk, Vk = U.randn(1, (70, D), torch.bfloat16), U.randn(2, (70, D), torch.bfloat16)
    codes, scales, _ = pack("bf16", Kk)
    vcodes, vscales, _ = pack("bf16", Vk)
    vscales[33, 2] = 255
    for dtype in ("bf16", "fp32"):
        for share in (2, 40):
            Q = U.randn(5, (share, 1, 4, D), U.dtype_of(dtype))
            out = torch.empty_like(Q)
            with U.context(1, 4, dtype, 60) as ctx:
                ctx.attend_shared_mx(Q, codes, scales, vcodes, vscales, torch.tensor([0, 70], device="cuda"), 1, share, 1, 70, out)
                torch.cuda.synchronize()
            assert bool(out[..., 64:96].isnan().all()) and int(out.isnan().sum()) == share * 4 * 32


@pytest.mark.parametrize("dtype,mx,scale", [(*form, scale) for form in FORMS for scale in (1e-6, 1.0)] + [("bf16", False, 30.0)])
def test_scales(dtype, mx, scale):
    check(dtype, mx, 1, 12, 1, 4, 1, [200], 30, scale=scale)


def test_offsets_outside_the_arrays_are_clamped():
    Kk, Vk, Q = U.randn(1, (100, D), torch.bfloat16), U.randn(2, (100, D), torch.bfloat16), U.randn(5, (6, 1, 4, D), torch.bfloat16)
    outs = []
    with U.context(1, 4, "bf16", 60) as ctx:
        for off in ([-50, 100, 5000], [0, 100, 100]):
            out = torch.empty_like(Q)
            ctx.attend_shared(Q, Kk, Vk, torch.tensor(off, device="cuda"), 2, 3, 1, 100, out)
            outs.append(out)
        out = torch.full_like(Q, math.nan)
        ctx.attend_shared(Q, Kk, Vk, torch.tensor([90, 20, 40], device="cuda"), 2, 3, 1, 100, out)      # (falling: a head of none)
        torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and bool((out[:3] == 0).all())


def test_results_do_not_change_from_run_to_run_and_graphs_replay():
    kv, group, share, keep, tail = 2, 4, 12, 3000, 40
    for dtype, mx in FORMS:
        dt = U.dtype_of(dtype)
        Kk, Vk = U.randn(1, (2 * keep, D), dt), U.randn(2, (2 * keep, D), dt)
        Kt, Vt = (U.randn(i, (share, kv, tail, D), dt) for i in (3, 4))
        Q = U.randn(5, (share, 1, kv * group, D), dt)
        lens = torch.full((share,), tail, dtype=torch.int32, device="cuda")
        offsets = torch.tensor([0, keep, 2 * keep], device="cuda")
        out, lse = torch.empty_like(Q), torch.empty((share, kv * group, 1), device="cuda")
        kept = (*pack(dtype, Kk)[:2], *pack(dtype, Vk)[:2]) if mx else (Kk, Vk)
        with U.context(kv, group, dtype, tail) as ctx:
            def step():
                (ctx.attend_shared_mx if mx else ctx.attend_shared)(Q, *kept, offsets, 1, share, 1, 2 * keep, out, K_tail=Kt, V_tail=Vt, tail_n=tail, tail_stride=tail, tail_lengths=lens,
                                                                    lse=lse)
            wants = []
            for L in (tail, 3):
                lens.fill_(L)
                step()
                wants.append((out.clone(), lse.clone()))
                step()
                assert torch.equal(out, wants[-1][0]) and torch.equal(lse, wants[-1][1])
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
            for _ in range(3):
                for L, want in zip((tail, 3), wants):
                    lens.fill_(L)
                    out.fill_(math.nan)
                    graph.replay()
                    torch.cuda.synchronize()
                    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_two_streams_with_scratch_of_their_own():
    kv, group, share, keep = 2, 4, 12, 3000
    Kk, Vk = U.randn(1, (2 * keep, D), torch.bfloat16), U.randn(2, (2 * keep, D), torch.bfloat16)
    offsets = torch.tensor([0, keep, 2 * keep], device="cuda")
    Qs = [U.randn(5 + i, (share, 1, kv * group, D), torch.bfloat16) for i in range(2)]
    with U.context(kv, group, "bf16", 10) as ctx:
        wants, outs, streams = [], [torch.empty_like(q) for q in Qs], [torch.cuda.Stream() for _ in Qs]
        for q in Qs:
            o = torch.empty_like(q)
            ctx.attend_shared(q, Kk, Vk, offsets, 1, share, 1, 2 * keep, o)
            wants.append(o)
        scratches = [torch.zeros((B.ATTEND_SCRATCH_BYTES,), dtype=torch.uint8, device="cuda") for _ in Qs]
        torch.cuda.synchronize()
        for _ in range(20):
            for q, o, scratch, s in zip(Qs, outs, scratches, streams):
                ctx.attend_shared(q, Kk, Vk, offsets, 1, share, 1, 2 * keep, o, scratch=scratch, stream=s)
        torch.cuda.synchronize()
        for o, w in zip(outs, wants):
            assert torch.equal(o, w)


def test_scratch_serves_the_other_attention_calls_in_turn():
    # one scratch for both: the counters that the others rely on stay cleared
    kv, group, keep = 2, 4, 3000
    Kk, Vk, Q = U.randn(1, (2 * keep, D), torch.bfloat16), U.randn(2, (2 * keep, D), torch.bfloat16), U.randn(5, (1, 1, kv * group, D), torch.bfloat16)
    offsets = torch.tensor([0, keep, 2 * keep], device="cuda")
    with U.context(kv, group, "bf16", 10) as ctx:
        a, b, c = (torch.empty_like(Q) for _ in range(3))
        ctx.attend_kept(Q, Kk, Vk, offsets, 1, 1, 2 * keep, a)
        many = U.randn(6, (40, 1, kv * group, D), torch.bfloat16)
        ctx.attend_shared(many, Kk, Vk, offsets, 1, 40, 1, 2 * keep, torch.empty_like(many))
        ctx.attend_kept(Q, Kk, Vk, offsets, 1, 1, 2 * keep, b)
        ctx.attend_shared(Q, Kk, Vk, offsets, 1, 1, 1, 2 * keep, c)
        torch.cuda.synchronize()
    assert torch.equal(a, b)
    # two ways to the same: each within 2^-7 of sum w |v| (its bf16 weights and result), which is below 2 here
    assert float((a.double() - c.double()).abs().max()) <= 2 * 2.0 ** -7 * 2


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("share,kv", [(33, 1), (65, 1), (37, 3)])
def test_odd_numbers_of_tails_beside_many_rows(mx, share, kv):
    # (two tails share a workgroup there; one of the last two is none)
    rng = np.random.default_rng(share)
    check("bf16", mx, 1, share, kv, 4, 1, rng.integers(1, 400, kv), 70, rng.integers(0, 71, share))


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("share,kv,keep,m", [(33, 1, 200000, 1), (37, 3, 70001, 1), (80, 2, 100100, 2), (64, 8, 25000, 1)])
def test_many_rows_over_long_prefixes(mx, share, kv, keep, m):
    # (tiles of 256 rows, two tails a workgroup, an odd number of them)
    rng = np.random.default_rng(share)
    check("bf16", mx, 1, share, kv, 4, m, keep - rng.integers(0, 70, kv), 40, rng.integers(0, 41, share), heads=2, seed=share)


@pytest.mark.parametrize("dtype,mx", FORMS)
@pytest.mark.parametrize("count,share,kv,m,tail", [(3, 60, 4, 2, 9), (5, 60, 4, 1, 130), (2, 130, 8, 1, 33), (9, 33, 7, 1, 20)])
def test_many_tails(dtype, mx, count, share, kv, m, tail):
    # (a wave a tail, and of the last workgroup's waves some that have none)
    rng = np.random.default_rng(share)
    check(dtype, mx, count, share, kv, 4, m, rng.integers(0, 90, count * kv), tail, rng.integers(0, tail + 1, count * share), heads=2)


@pytest.mark.parametrize("dtype,mx", FORMS)
@pytest.mark.parametrize("kv,group,share,m", [(1024, 16, 2, 1), (1024, 1, 3, 2), (500, 17, 2, 2), (128, 128, 1, 1), (126, 129, 2, 1), (1, 16384, 1, 2)])
def test_as_many_heads_as_there_may_be(dtype, mx, kv, group, share, m):
    # (parts of rows fill what scratch there is: nothing beside the outputs is written, and the last heads' are right)
    rng = np.random.default_rng(kv)
    scratch = Guarded((B.ATTEND_SCRATCH_BYTES // 4,), torch.int32, 0)
    dt, budgets = U.dtype_of(dtype), rng.integers(0, 70, kv)
    off = np.concatenate([[0], np.cumsum(budgets)]).astype(np.int64)
    total = int(off[-1])
    Kk, Vk = U.randn(1, (total, D), dt), U.randn(2, (total, D), dt)
    Kt, Vt = (U.randn(i, (share, kv, 6, D), dt) for i in (3, 4))
    Q = U.randn(5, (share, m, kv * group, D), dt)
    out = Guarded((share * m * kv * group, D), dt, float("nan"))
    lse = Guarded((share * kv * group, m), torch.float32, float("nan"))
    since = dict(K_tail=Kt, V_tail=Vt, tail_n=6, tail_stride=6, lse=lse.t, scratch=scratch.t)
    with U.context(kv, group, dtype, 64) as ctx:
        if mx:
            Kc, Ks, Kk = pack(dtype, Kk)
            Vc, Vs, Vk = pack(dtype, Vk)
            ctx.attend_shared_mx(Q, Kc, Ks, Vc, Vs, torch.from_numpy(off).cuda(), 1, share, m, total, out.t, **since)
        else:
            ctx.attend_shared(Q, Kk, Vk, torch.from_numpy(off).cuda(), 1, share, m, total, out.t, **since)
        torch.cuda.synchronize()
    for x in (scratch, out, lse):
        x.check()
    got, got_lse = out.t.view(share, m, kv * group, D), lse.t.view(share, kv * group, m)
    assert not bool(got.isnan().any()) and not bool(got_lse.isnan().any())
    for h in sorted({0, 1, kv * group // 2, kv * group - 2, kv * group - 1} & set(range(kv * group))):
        k = torch.cat([Kk[off[h // group]:off[h // group + 1]].double(), Kt[share - 1, h // group].double()])
        v = torch.cat([Vk[off[h // group]:off[h // group + 1]].double(), Vt[share - 1, h // group].double()])
        seen = torch.cat([torch.ones((m, k.shape[0] - 6), dtype=torch.bool, device="cuda"), U.causal(m, 6, 6, 0, 0)], 1)
        want = U.attention(Q[share - 1, :, h], k, v, seen, D ** -0.5)
        U.check_attention(got[share - 1, :, h], got_lse[share - 1, h], want, dtype, k.shape[0] + 64, f"head {h}")
