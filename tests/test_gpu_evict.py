"""Eviction by accumulated weight (curdkv_evict) against its definition."""

import math

import numpy as np
import pytest
import torch

from paper_2509_15038_amd import binding as B
from tests import attend_util as U
from tests.gpu_util import Guarded

pytestmark = pytest.mark.gpu
D = 128


def want_rows(mass, positions, L, keep, n_sink, recent):
    """One head, by the definition: the row that each place's row comes from."""
    stays = min(L, keep)
    if L <= keep:
        return np.arange(L)
    with np.errstate(invalid="ignore"):             # (signalling NaN)
        w, p = mass[:L].astype(np.float64), positions[:L].astype(np.int64)
    first = (p < n_sink) | (p > p.max() - recent)
    order = sorted(range(L), key=lambda i: (not first[i], 0 if math.isnan(w[i]) else 1, 0.0 if math.isnan(w[i]) else -w[i], i))
    chosen = np.zeros(L, dtype=bool)
    chosen[order[:stays]] = True
    rows = np.arange(stays)
    rows[~chosen[:stays]] = np.flatnonzero(chosen[stays:]) + stays
    return rows


def check(dtype, count, kv, n, keep, n_sink=0, recent=0, lengths=None, stride=None, place=True, mass=None, positions="own", out_stride=None, seed=0, moves_mass=True, stream=None):
    dt = U.dtype_of(dtype)
    stride = n if stride is None else stride
    out_stride = stride if place else (min(n, keep) + 3 if out_stride is None else out_stride)
    rng = np.random.default_rng(seed)
    K0, V0 = (U.randn(seed + i, (count, kv, stride, D), dt) for i in (1, 2))
    lens = np.full(count, n) if lengths is None else np.asarray(lengths)
    M0 = np.exp(rng.standard_normal((count, kv, stride))).astype(np.float32) if mass is None else np.asarray(mass(rng, (count, kv, stride)), dtype=np.float32)
    P0 = None
    if isinstance(positions, str) and positions == "own":
        P0 = np.argsort(rng.random((count, kv, stride)), -1).astype(np.int32) * 2
    elif positions is not None:
        P0 = np.asarray(positions(rng, (count, kv, stride)), dtype=np.int32)
    kinds = [(K0, dt), (V0, dt), (torch.from_numpy(M0).cuda(), torch.float32)] + ([(torch.from_numpy(P0).cuda(), torch.int32)] if P0 is not None else [])
    given = []
    for x, t in kinds:
        g = Guarded((count * kv * stride * (D if x.dim() == 4 else 1),), t, 0)
        g.t.copy_(x.reshape(-1))
        given.append(g)
    if place:
        outs = list(given)
        if P0 is None:
            outs.append(Guarded((count * kv * out_stride,), torch.int32, -7))
    else:
        outs = [Guarded((count * kv * out_stride * D,), dt, 5.0) for _ in "KV"] + [Guarded((count * kv * out_stride,), torch.float32, 5.0), Guarded((count * kv * out_stride,), torch.int32, -7)]
    before = [o.t.clone() for o in outs]
    rows = Guarded((count * kv * keep,), torch.int32, -9)
    with U.context(kv, 1, dtype, n) as ctx:
        ctx.evict(given[0].t, given[1].t, given[2].t, count, n, stride, keep, rows.t, positions=None if P0 is None else given[3].t,
                  lengths=None if lengths is None else torch.from_numpy(lens.astype(np.int32)).cuda(), n_sink=n_sink, recent=recent, K_out=outs[0].t, V_out=outs[1].t,
                  mass_out=outs[2].t if moves_mass else None, positions_out=outs[3].t if moves_mass else None, out_stride=out_stride, stream=stream)
        torch.cuda.synchronize()
    for g in given + outs + [rows]:
        g.check()
    got_rows = rows.t.view(count, kv, keep).cpu().numpy()
    shapes = [(count, kv, out_stride, D)] * 2 + [(count, kv, out_stride)] * 2
    wants = [b.clone().view(s) for b, s in zip(before, shapes)]
    P = np.broadcast_to(np.arange(stride, dtype=np.int32), (count, kv, stride)) if P0 is None else P0
    sources = [K0, V0, torch.from_numpy(M0).cuda(), torch.from_numpy(np.ascontiguousarray(P)).cuda()]
    for b in range(count):
        L = int(min(max(lens[b], 0), n))
        for h in range(kv):
            want = want_rows(M0[b, h], P[b, h], L, keep, n_sink, recent)
            got = got_rows[b, h]
            assert (got[: len(want)] == want).all(), f"sequence {b} of {L}, head {h}: places {np.flatnonzero(got[: len(want)] != want)[:5]}, {got[: len(want)][got[: len(want)] != want][:5]}, " \
                                                     f"not {want[got[: len(want)] != want][:5]}"
            assert (got[len(want):] == -1).all()
            at = torch.from_numpy(want).cuda()
            for w, x, moved in zip(wants, sources, (True, True, moves_mass, moves_mass)):
                if moved:
                    w[b, h, : len(want)] = x[b, h, at]
    for o, w, what in zip(outs, wants, ("K", "V", "mass", "positions")):
        x, y = o.t.view(w.shape), w
        assert torch.equal(x.view(torch.int32) if x.dtype == torch.float32 else x, y.view(torch.int32) if y.dtype == torch.float32 else y), what


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("place", [True, False])
@pytest.mark.parametrize("n,keep", [(1, 1), (2, 1), (5, 9), (64, 64), (65, 64), (130, 63), (1000, 1), (1025, 1024), (1500, 1000), (3277, 3276), (4096, 100), (5000, 4999)])
def test_sizes(dtype, place, n, keep):
    check(dtype, 2, 2, n, keep, min(4, keep // 2), min(16, keep // 3), place=place, seed=n + keep)


@pytest.mark.parametrize("place", [True, False])
@pytest.mark.parametrize("n_sink,recent", [(0, 0), (1, 0), (0, 1), (40, 60), (100, 0), (0, 100), (37, 63)])
def test_protected_rows(place, n_sink, recent):
    check("bf16", 2, 2, 300, 100, n_sink, recent, place=place, seed=n_sink)
    check("bf16", 2, 2, 300, 100, n_sink, recent, place=place, seed=n_sink, positions=None)


def test_more_protected_rows_than_stay():
    # positions more than once: the weight decides among the protected
    same = lambda rng, shape: rng.integers(0, 20, shape)
    for n_sink, recent in ((50, 50), (0, 100), (100, 0), (3, 2)):
        check("bf16", 2, 2, 300, 100, n_sink, recent, positions=same, seed=n_sink)
    check("bf16", 1, 2, 300, 100, 0, 100, positions=lambda rng, s: np.zeros(s))


@pytest.mark.parametrize("mass", [lambda r, s: np.zeros(s), lambda r, s: np.full(s, 3.5), lambda r, s: r.integers(0, 3, s), lambda r, s: r.integers(0, 2, s) * 1e-42,
                                  lambda r, s: -r.random(s), lambda r, s: r.standard_normal(s) * 1e30, lambda r, s: 1 + r.integers(0, 5, s) * 2.0 ** -23,
                                  lambda r, s: np.where(r.random(s) < 0.5, 0.0, -0.0),
                                  lambda r, s: np.select([r.random(s) < 0.1, r.random(s) < 0.1, r.random(s) < 0.1], [np.nan, np.inf, -np.inf], r.random(s)),
                                  lambda r, s: np.full(s, np.nan)],
                         ids=["zeros", "equal", "few values", "smallest", "negative", "large", "last bits", "signed zeros", "not finite", "all NaN"])
@pytest.mark.parametrize("n,keep", [(700, 300), (2100, 2000)])
def test_weights(mass, n, keep):
    check("bf16", 2, 2, n, keep, 4, 30, mass=mass, seed=1)
    check("bf16", 2, 2, n, keep, 0, 0, mass=mass, seed=2, place=False)


def test_nan_of_either_sign():
    def mass(r, s):
        x = r.random(s).astype(np.float32)
        x.view(np.uint32)[..., ::7] = 0xFFC00000
        x.view(np.uint32)[..., ::11] = 0x7F800001
        return x
    check("bf16", 1, 2, 500, 100, mass=mass)
    check("bf16", 1, 2, 500, 30, mass=mass)


@pytest.mark.parametrize("place", [True, False])
def test_lengths(place):
    lens = [0, 1, 99, 100, 101, 128, 199, 200, 777, -4, 5]
    for dtype in ("bf16", "fp32"):
        check(dtype, 11, 2, 200, 100, 4, 20, lengths=lens, place=place)
    check("bf16", 11, 1, 200, 100, 4, 20, lengths=lens, place=place, positions=None)


def test_strides_and_what_is_not_asked_for():
    check("bf16", 2, 3, 150, 70, 2, 9, stride=201)
    check("fp32", 2, 3, 150, 70, 2, 9, stride=201, place=False, out_stride=70)
    check("bf16", 2, 3, 150, 70, 2, 9, moves_mass=False)
    check("bf16", 2, 3, 150, 200, 2, 9, place=False, out_stride=150)


def test_positions_of_all_sizes():
    check("bf16", 1, 2, 300, 100, 4, 50, positions=lambda r, s: r.integers(-2 ** 31, 2 ** 31 - 1, s))
    check("bf16", 1, 2, 300, 100, 2 ** 5, 2 ** 6, positions=lambda r, s: r.integers(-2 ** 31, -2 ** 31 + 100, s))


@pytest.mark.parametrize("n,keep", [(32768, 3276), (40000, 39000), (131072, 13107), (200000, 100000)])
def test_long_heads(n, keep):
    check("bf16", 1, 2, n, keep, 4, 64, seed=n)
    check("bf16", 1, 1, n, keep, 4, 64, seed=n, mass=lambda r, s: r.integers(0, 40, s), place=False)


def test_longest_head():
    check("bf16", 1, 1, 2 ** 19, 1000, 4, 64, place=False)
    with U.context(1, 1, "bf16", 2 ** 19 + 1) as ctx, pytest.raises(B.CurdkvError) as e:
        z = torch.zeros(16, device="cuda")
        ctx.evict(z, z[4:], z, 1, 2 ** 19 + 1, 2 ** 19 + 1, 5, z)
    assert e.value.code == B.ERR_UNSUPPORTED


def test_weights_and_positions_with_places_of_their_own_while_rows_stay():
    # in place, but the old weights are kept: a second call finds the same rows
    n, keep = 130, 100
    K, V = U.randn(1, (1, 2, n, D), torch.bfloat16), U.randn(2, (1, 2, n, D), torch.bfloat16)
    mass = torch.rand((1, 2, n), device="cuda")
    at = torch.arange(n, dtype=torch.int32, device="cuda").expand(1, 2, n).contiguous()
    to, at_to, rows = torch.zeros_like(mass), torch.zeros_like(at), torch.empty((1, 2, keep), dtype=torch.int32, device="cuda")
    old = mass.clone()
    with U.context(2, 1, "bf16", n) as ctx:
        ctx.evict(K, V, mass, 1, n, n, keep, rows, positions=at, mass_out=to, positions_out=at_to)
        first = [x.clone() for x in (K, V, to, at_to, rows)]
        ctx.evict(K, V, mass, 1, n, n, keep, rows, positions=at, mass_out=to, positions_out=at_to)
        torch.cuda.synchronize()
        for x, y in zip(first, (K, V, to, at_to, rows)):
            assert torch.equal(x, y)
        assert torch.equal(mass, old)
        want = [want_rows(old[0, h].cpu().numpy(), np.arange(n), n, keep, 0, 0) for h in range(2)]
        assert (rows.cpu().numpy()[0] == np.stack(want)).all()


def test_generation_keeps_the_heaviest_and_graphs_replay():
    # one token comes, one row leaves, replayed: the same as the definition step by step
    kv, keep, steps, sinks, recent = 3, 50, 40, 2, 8
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    K, V = torch.zeros((1, kv, keep + 1, D), device="cuda"), torch.zeros((1, kv, keep + 1, D), device="cuda")
    mass, at = torch.zeros((1, kv, keep + 1), device="cuda"), torch.zeros((1, kv, keep + 1), dtype=torch.int32, device="cuda")
    for i in range(keep):
        K[:, :, i], V[:, :, i], at[:, :, i] = i, -i, i
    mass[..., :keep] = torch.rand((1, kv, keep), generator=g, device="cuda")
    new_mass, now = torch.zeros((1, kv), device="cuda"), torch.zeros((1,), dtype=torch.int32, device="cuda")
    rows = torch.empty((1, kv, keep), dtype=torch.int32, device="cuda")
    with U.context(kv, 1, "fp32", keep + 1) as ctx:
        def step():
            K[:, :, keep], V[:, :, keep], at[:, :, keep], mass[:, :, keep] = now.float(), -now.float(), now, new_mass
            ctx.evict(K, V, mass, 1, keep + 1, keep + 1, keep, rows, positions=at, n_sink=sinks, recent=recent)
        held = [[(i, float(mass[0, h, i])) for i in range(keep)] for h in range(kv)]
        now.fill_(keep - 1)
        graph = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream()
        keepers = [x.clone() for x in (K, V, mass, at)]
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        for x, y in zip((K, V, mass, at), keepers):
            x.copy_(y)
        with torch.cuda.graph(graph):
            step()
        for t in range(keep, keep + steps):
            now.fill_(t)
            new_mass.copy_(torch.rand((1, kv), generator=g, device="cuda"))
            graph.replay()
            torch.cuda.synchronize()
            for h in range(kv):
                have = held[h] + [(t, float(new_mass[0, h]))]
                source = want_rows(np.array([w for _, w in have], dtype=np.float32), np.array([p for p, _ in have]), keep + 1, keep, sinks, recent)
                held[h] = [have[i] for i in source]
                assert at[0, h, :keep].tolist() == [p for p, _ in held[h]] and mass[0, h, :keep].tolist() == pytest.approx([w for _, w in held[h]], abs=0)
                assert K[0, h, :keep, 77].tolist() == [p for p, _ in held[h]] and V[0, h, :keep, 0].tolist() == [-p for p, _ in held[h]]


def test_another_stream():
    torch.cuda.synchronize()
    check("bf16", 2, 2, 500, 200, 4, 20, stream=torch.cuda.Stream())


def test_many_heads():
    check("bf16", 300, 4, 70, 64, 2, 8, lengths=np.arange(300) % 71)


@pytest.mark.parametrize("n,keep", [(900, 100), (5000, 4998), (40000, 4000), (220000, 50000)])
def test_recorded_calls_of_all_sizes(n, keep):
    # (short heads, few that leave, a long head, one whose bitmaps need more LDS than a launch has by itself), weights changed between the replays
    K, V = (U.randn(i, (1, 2, n, D), torch.bfloat16) for i in (1, 2))
    mass = torch.empty((1, 2, n), device="cuda")
    outs = [[torch.zeros((1, 2, keep, D), dtype=torch.bfloat16, device="cuda") for _ in "KV"] + [torch.zeros((1, 2, keep), device="cuda"),
                                                                                                   torch.zeros((1, 2, keep), dtype=torch.int32, device="cuda"),
                                                                                                   torch.zeros((1, 2, keep), dtype=torch.int32, device="cuda")] for _ in range(2)]
    with U.context(2, 1, "bf16", n) as ctx:
        def call(out):
            ctx.evict(K, V, mass, 1, n, n, keep, out[4], n_sink=4, recent=16, K_out=out[0], V_out=out[1], mass_out=out[2], positions_out=out[3], out_stride=keep)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(outs[0])
        for turn in range(3):
            mass.copy_(U.randn(10 + turn, (1, 2, n), torch.float32).exp())
            call(outs[1])
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(*outs):
                assert torch.equal(a, b)
            rows = want_rows(mass[0, 1].cpu().numpy(), np.arange(n), n, keep, 4, 16)
            assert np.array_equal(outs[0][4][0, 1].cpu().numpy(), rows)
