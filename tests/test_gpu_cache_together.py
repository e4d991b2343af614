"""A cache that stays at its size and one that serves several answers, as a program uses them: rotation by several positions, attention, the weights that keys got, eviction by them, and
answers over what is left, each step against its definition in 64 bits; recorded steps against eager ones; and the small decoder's."""

import math

import numpy as np
import pytest
import torch

from tests import attend_util as U
from tests.test_gpu_evict import want_rows
from tests.test_gpu_rotate import table_of

pytestmark = pytest.mark.gpu
D = 128


class Run:
    """A prompt of n tokens on a grid, `steps` tokens over a cache that stays at `room`, and then `share` answers of one token each over what it holds."""

    def __init__(self, dtype, kv, group, n, room, seed=0):
        self.dt, self.kv, self.group, self.n, self.room = U.dtype_of(dtype), kv, group, n, room
        self.axis_of = np.repeat(np.arange(3, dtype=np.uint8), (16, 24, 24))
        self.table = table_of(n + 64)
        self.qkv = U.randn(seed + 1, (n, (group + 2) * kv * D), self.dt)
        token = torch.arange(n, dtype=torch.int32, device="cuda")
        self.positions = torch.stack([token // 64, token // 8 % 8, token % 8]).contiguous()
        self.ctx = U.context(kv, group, dtype, n + 64)

    def prompt(self, window):
        n, heads = self.n, self.kv * self.group
        self.Q = torch.empty((n, heads, D), dtype=self.dt, device="cuda")
        self.K, self.V = (torch.empty((self.kv, n, D), dtype=self.dt, device="cuda") for _ in "KV")
        self.out, self.lse = torch.empty_like(self.Q), torch.empty((heads, n), device="cuda")
        self.mass = torch.full((self.kv, n), math.nan, device="cuda")
        self.ctx.rotate_axes(self.qkv, 1, n, self.table, self.positions, self.axis_of, self.Q, self.K, self.V, n)
        self.ctx.attend(self.Q, self.K, self.V, 1, n, n, n, self.out, lse=self.lse)
        self.ctx.attend_weights(self.Q[n - window:], self.K, self.lse[:, n - window:].contiguous(), 1, window, n, n, self.mass, decay=0.0)

    def evict(self, n_sink, recent):
        shape = (self.kv, self.room + 1)
        self.held = [torch.zeros((*shape, D), dtype=self.dt, device="cuda") for _ in "KV"] + [torch.zeros(shape, device="cuda"), torch.zeros(shape, dtype=torch.int32, device="cuda")]
        self.rows = torch.empty((self.kv, self.room), dtype=torch.int32, device="cuda")
        K, V, mass, tokens = self.held
        self.ctx.evict(self.K, self.V, self.mass, 1, self.n, self.n, self.room, self.rows, n_sink=n_sink, recent=recent, K_out=K, V_out=V, mass_out=mass, positions_out=tokens,
                       out_stride=self.room + 1)

    def begin(self, seed):
        heads = self.kv * self.group
        self.x = U.randn(seed, (1, (self.group + 2) * self.kv * D), self.dt)
        self.at = torch.full((3, 1), 9, dtype=torch.int32, device="cuda")
        self.place = torch.full((1,), self.room, dtype=torch.int32, device="cuda")
        self.tokens = torch.full((1,), self.n, dtype=torch.int32, device="cuda")
        self.q1, self.o1, self.l1 = torch.empty((1, heads, D), dtype=self.dt, device="cuda"), torch.empty((1, heads, D), dtype=self.dt, device="cuda"), torch.empty(heads, device="cuda")

    def step(self, decay, n_sink, recent):
        K, V, mass, tokens = self.held
        n = self.room + 1
        mass[:, self.room] = 0
        tokens[:, self.room] = self.tokens
        self.ctx.rotate_axes(self.x, 1, 1, self.table, self.at, self.axis_of, self.q1, K, V, n, starts=self.place)
        self.ctx.attend(self.q1, K, V, 1, 1, n, n, self.o1, lse=self.l1)
        self.ctx.attend_weights(self.q1, K, self.l1, 1, 1, n, n, mass, decay=decay)
        self.before = mass.clone()
        self.ctx.evict(K, V, mass, 1, n, n, self.room, self.rows, positions=tokens, n_sink=n_sink, recent=recent)
        self.at += 1
        self.tokens += 1

    def answer(self, share, seed):
        """`share` answers, whose own tokens lie in tails, over the first `room` rows of the held cache."""
        heads, room = self.kv * self.group, self.room
        Q = U.randn(seed, (share, 1, heads, D), self.dt)
        Kt, Vt = (U.randn(seed + i, (share, self.kv, 4, D), self.dt) for i in (1, 2))
        lengths = torch.arange(share, dtype=torch.int32, device="cuda") % 5
        kept = [t[:, :room].reshape(-1, D).contiguous() for t in self.held[:2]]
        offsets = torch.arange(self.kv + 1, device="cuda") * room
        out, lse = torch.empty_like(Q), torch.empty((share, heads, 1), device="cuda")
        self.ctx.attend_shared(Q, *kept, offsets, 1, share, 1, self.kv * room, out, K_tail=Kt, V_tail=Vt, tail_n=4, tail_stride=4, tail_lengths=lengths, lse=lse)
        return Q, kept, Kt, Vt, lengths, out, lse


def near_weights(got, q, k, lse, seen, old, scale):
    """One KV head's summed weights: q [heads, m, D], k [n, D], lse [heads, m]; `old` already decayed."""
    x = torch.matmul(q.double(), k.double().T) * scale
    z = lse.double()[..., None]
    w = torch.where(seen, torch.exp(x - z), 0.0)
    size = torch.matmul(q.double().abs(), k.double().abs().T) * scale
    # a score: 128 products and sums; its difference from lse, four roundings of either term; the exponential 2^-22; the sum of all weights, and one more with `old`
    rel = 128 * 2.0 ** -24 * size + 4 * 2.0 ** -24 * (x.abs() + z.abs()) + 2.0 ** -22
    want = w.sum((0, 1)) + old
    off = (w * rel).sum((0, 1)) + (w.shape[0] * w.shape[1] + 6) * 2.0 ** -24 * want + 1e-35
    assert bool(((got.double() - want).abs() <= off).all())


@pytest.mark.parametrize("dtype,kv,group,n,room,window", [("bf16", 2, 4, 700, 200, 8), ("bf16", 1, 7, 333, 333, 333), ("fp32", 2, 4, 520, 97, 16), ("bf16", 8, 4, 4096, 1000, 32)])
def test_a_cache_that_stays_at_its_size(dtype, kv, group, n, room, window):
    scale, decay, n_sink, recent = D ** -0.5, 0.75, 4, 16
    r = Run(dtype, kv, group, n, room)
    r.prompt(window)
    r.evict(n_sink, recent)
    torch.cuda.synchronize()
    seen = U.causal(window, n, n, 0, 0)
    for h in range(kv):
        q = r.Q[n - window:, h * group:(h + 1) * group].transpose(0, 1)
        near_weights(r.mass[h], q, r.K[h], r.lse[h * group:(h + 1) * group, n - window:], seen, 0.0, scale)
        rows = want_rows(r.mass[h].cpu().numpy(), np.arange(n), n, room, n_sink, recent)
        assert np.array_equal(r.rows[h].cpu().numpy(), rows)
        for held, came in zip(r.held, (r.K[h], r.V[h], r.mass[h], torch.arange(n, dtype=torch.int32, device="cuda"))):
            assert torch.equal(held[h, :room], came[torch.from_numpy(rows).cuda()])
    r.begin(50)
    for i in range(4):
        K0, V0, m0, t0 = (t.clone() for t in r.held)
        r.x = U.randn(60 + i, r.x.shape, r.dt)
        r.step(decay, n_sink, recent)
        torch.cuda.synchronize()
        # the token's own row is where the rotation put it until it has gone: what the others are is known from before
        last_k, last_v = K0.clone(), V0.clone()
        y = r.x.view(-1, D)
        r.ctx.rotate_axes(r.x, 1, 1, r.table, r.at - 1, r.axis_of, r.q1, last_k, last_v, room + 1, starts=r.place)
        assert torch.equal(last_v[:, room], y[kv * (group + 1):])
        for h in range(kv):
            q = r.q1[:, h * group:(h + 1) * group].transpose(0, 1)
            all_seen = torch.ones((1, room + 1), dtype=torch.bool, device="cuda")
            for g in range(group):
                want = U.attention(q[g], last_k[h], last_v[h], all_seen, scale)
                U.check_attention(r.o1[:, h * group + g], r.l1[h * group + g][None], want, dtype, room + 65)
            old = m0[h].double() * decay
            old[room] = 0
            near_weights(r.before[h], q, last_k[h], r.l1[h * group:(h + 1) * group, None], all_seen, old, scale)
            t = t0[h].clone()
            t[room] = n + i
            rows = want_rows(r.before[h].cpu().numpy(), t.cpu().numpy(), room + 1, room, n_sink, recent)
            assert np.array_equal(r.rows[h].cpu().numpy(), rows)
            for held, came in zip(r.held, (last_k[h], last_v[h], r.before[h], t)):
                assert torch.equal(held[h, :room], came[torch.from_numpy(rows).cuda()])
    for share in (1, 3, 40):
        Q, kept, Kt, Vt, lengths, out, lse = r.answer(share, 70)
        torch.cuda.synchronize()
        for b in range(share):
            L = int(lengths[b])
            for h in range(kv * group):
                k = torch.cat([r.held[0][h // group, :room].double(), Kt[b, h // group, :L].double()])
                v = torch.cat([r.held[1][h // group, :room].double(), Vt[b, h // group, :L].double()])
                want = U.attention(Q[b, :, h], k, v, torch.ones((1, room + L), dtype=torch.bool, device="cuda"), scale)
                U.check_attention(out[b, :, h], lse[b, h], want, dtype, room + 68, f"answer {b}, head {h}")
    r.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_recorded_steps(dtype):
    # two graphs of one context, whose steps share its scratch, replayed in turn with eager work between: every replay is the eager step
    def fresh():
        r = Run(dtype, 2, 4, 600, 150)
        r.prompt(8)
        r.evict(2, 8)
        r.begin(50)
        return r

    eager, recorded = fresh(), fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        recorded.step(0.5, 2, 8)
        recorded.answer(5, 70)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    fixed = [t.clone() for t in fresh().held]
    for t, was in zip(recorded.held, fixed):
        t.copy_(was)
    recorded.at.fill_(9)
    recorded.tokens.fill_(recorded.n)
    step, answers = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(step):
        recorded.step(0.5, 2, 8)
    heads, share = 8, 5
    Q = U.randn(70, (share, 1, heads, D), recorded.dt)
    kept = [torch.empty((2 * 150, D), dtype=recorded.dt, device="cuda") for _ in "KV"]
    offsets, out = torch.arange(3, device="cuda") * 150, torch.empty_like(Q)

    def answer(r, out):
        for to, t in zip(kept, r.held):
            to.view(2, 150, D).copy_(t[:, :150])
        r.ctx.attend_shared(Q, *kept, offsets, 1, share, 1, 300, out)

    with torch.cuda.graph(answers):
        answer(recorded, out)
    for i in range(5):
        x = U.randn(80 + i, eager.x.shape, eager.dt)
        eager.x.copy_(x)
        recorded.x.copy_(x)
        eager.step(0.5, 2, 8)
        want = torch.empty_like(Q)
        answer(eager, want)
        torch.cuda.synchronize()
        step.replay()
        answers.replay()
        torch.cuda.synchronize()
        for a, b in zip([*eager.held, eager.rows, eager.o1, eager.l1, want], [*recorded.held, recorded.rows, recorded.o1, recorded.l1, out]):
            assert torch.equal(a, b)
    eager.ctx.close()
    recorded.ctx.close()


def prompt_of(model, n, seed):
    return torch.randn((n, 1024), generator=torch.Generator().manual_seed(seed)).to("cuda", model.dtype)


# a layer rounds projections, queries, keys, weights, results and sums in bf16, about ten roundings of 2^-9 relative (2^-8 at most) to values of size 1 to 3; two layers, and two results
# that are compared
TOLERANCE = {"bf16": 2 * 2 * 10 * 3 * 2.0 ** -9, "fp32": 2e-3}


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_decoder_with_several_answers(dtype):
    from paper_2509_15038_amd.example import Decoder
    model = Decoder(2, 2, 4, 512, 8, dtype=dtype, sketch_dim=16, seed=3)
    model.prompt(prompt_of(model, 300, 4))
    tokens = [prompt_of(model, 3, 5 + i) for i in range(4)]
    for choose in (model.keep_all, lambda answers: model.keep(0.3, False, answers), lambda answers: model.keep(0.3, True, answers)):
        choose(answers=3)
        together = [model.step(x) for x in tokens]
        for b in range(3):
            choose(answers=1)
            for x, y in zip(tokens, together):
                assert (model.step(x[b:b + 1])[0].double() - y[b].double()).abs().max() < TOLERANCE[dtype]
        choose(answers=3)
        recorded, _ = model.generate(tokens[0], 3)
        choose(answers=3)
        assert recorded.shape == (3, 3, 1024) and torch.equal(model.step(tokens[0]), recorded[0])
    model.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_decoder_that_holds_its_size(dtype):
    from paper_2509_15038_amd.example import Decoder
    model = Decoder(2, 2, 4, 512, 8, dtype=dtype, sketch_dim=16, seed=3)
    x = prompt_of(model, 300, 4)
    first = model.prompt(x, watch=16)[-1:].clone()
    model.keep_all()
    whole = model.step(first)
    model.hold(300)                                                 # (room for all of them: its first token is the whole cache's)
    assert (model.step(first).double() - whole.double()).abs().max() < TOLERANCE[dtype]
    model.hold(100, recent=10)
    recorded, _ = model.generate(first, 6)
    model.hold(100, recent=10)
    y = first
    for i in range(6):
        z = model.step(y)
        torch.cuda.synchronize()
        assert torch.equal(z[0], recorded[i])
        y = (z.float() * torch.rsqrt(z.float().square().mean(-1, keepdim=True) + 1e-6)).to(model.dtype)
        for tokens in model.held[3][:, :, :100].reshape(-1, 100).tolist():
            assert len(set(tokens)) == 100 and set(range(4)) | set(range(291 + i, 301 + i)) <= set(tokens)
    model.close()


def test_decoder_on_a_grid():
    from paper_2509_15038_amd.example import Decoder
    # (the same position on every axis is one position)
    plain, grid = Decoder(2, 2, 4, 256, 8, sketch_dim=16, seed=3), Decoder(2, 2, 4, 256, 8, sketch_dim=16, seed=3, axes=(16, 24, 24))
    x = prompt_of(plain, 200, 4)
    same = torch.arange(200, dtype=torch.int32, device="cuda").expand(3, -1).contiguous()
    assert torch.equal(plain.prompt(x), grid.prompt(x, same))
    for model in (plain, grid):
        model.keep_all(answers=2)
    y = prompt_of(plain, 2, 9)
    assert torch.equal(plain.step(y), grid.step(y))
    token = torch.arange(200, dtype=torch.int32, device="cuda")
    other = grid.prompt(x, torch.stack([token // 100, token // 10 % 10, token % 10]).contiguous())
    assert grid.last == 9 and not torch.equal(other, plain.prompt(x))
    for model, positions in ((plain, same), (grid, None)):
        with pytest.raises(ValueError):
            model.prompt(x, positions)
    for model in (plain, grid):
        model.close()


def test_decoder_refuses():
    from paper_2509_15038_amd.example import Decoder
    model = Decoder(1, 2, 4, 256, 8, sketch_dim=16, seed=3)
    x = prompt_of(model, 50, 4)
    model.prompt(x)
    with pytest.raises(ValueError, match="watched"):
        model.hold(20)
    model.prompt(x, watch=8)
    with pytest.raises(ValueError, match="shorter"):
        model.hold(51)
    model.close()
    model = Decoder(1, 2, 4, 256, 8, sketch_dim=16, seed=3, window=20)
    model.prompt(x, watch=8)
    with pytest.raises(ValueError, match="window"):
        model.hold(20)
    with pytest.raises(ValueError, match="window"):
        model.keep_all(answers=2)
    model.close()


def test_command_with_all_of_it(capsys):
    from paper_2509_15038_amd import example
    example.main(["--layers", "2", "--kv-heads", "2", "--tokens", "2000", "--new", "3", "--hold", "300", "--answers", "5", "--axes", "32", "32"])
    assert capsys.readouterr().out.count("\n") == 7
