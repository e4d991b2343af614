"""A small decoder around a compressed cache: every entry point of the attention side in the place where a program calls it.

    python -m paper_2509_15038_amd.example --layers 8 --tokens 32768 --keep 0.1 --new 64

A stack of attention layers with random weights (x + Wo attention(Wqkv x), grouped heads, rotary positions, RMS norms of a head's queries and
keys) takes a prompt, chooses the tokens whose keys and values it keeps, holds those in 4 bits and generates over them and the tokens since, one
step a HIP graph replay; beside it the same over the whole prompt's cache.  With a window it generates over the whole cache alone: kept rows have no
positions that a window could pass.  With --hold the cache also stays at a size while it generates: after every token the one that got the least
attention goes.  With --answers several answers follow the prompt at once, its rows read once for all.  With --axes the prompt's tokens stand on a
square grid.  The products with weights are torch's, all else is the library's."""
import argparse
import time

import numpy as np
import torch

from . import binding as B
from . import workloads as wl

D = 128                                             # channels of a head


def rotary_table(rows: int, base: float = 500000.0, device="cuda") -> torch.Tensor:
    """[rows, 2, 64]: cosines and sines of position * base^(-i / 64)."""
    angle = torch.arange(rows, dtype=torch.float64)[:, None] * base ** (-torch.arange(D // 2, dtype=torch.float64) / (D // 2))
    return torch.stack([angle.cos(), angle.sin()], dim=1).float().to(device).contiguous()


class Decoder:
    def __init__(self, layers: int, kv_heads: int, group: int, max_tokens: int, new_tokens: int, dtype: str = "bf16", window: int = 0, n_sink: int = 4,
                 sketch_dim: int = 64, seed: int = 1, axes=()):
        """axes: how many of the 64 angles turn by each axis' position, as (16, 24, 24); empty: a token has one position."""
        self.layers, self.kv, self.group, self.window, self.n_sink, self.stride = layers, kv_heads, group, window, n_sink, new_tokens
        self.dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.ctx = B.Context(layers, kv_heads, group, D, sketch_dim, dtype, max_tokens + (new_tokens if window else 0), seed=seed)
        self.table = rotary_table(max_tokens + new_tokens)
        self.axis_of = np.repeat(np.arange(len(axes), dtype=np.uint8), axes) if axes else None
        width = kv_heads * group * D
        draw = torch.Generator().manual_seed(seed)

        def weight(rows, columns):
            return (torch.randn((rows, columns), generator=draw) * rows ** -0.5).to("cuda", self.dtype)
        self.qkv = [weight(width, width + 2 * kv_heads * D) for _ in range(layers)]
        self.out = [weight(width, width) for _ in range(layers)]
        self.norms = [[(1 + 0.1 * torch.randn(D, generator=draw)).to("cuda", self.dtype) for _ in "qk"] for _ in range(layers)]

    def close(self):
        self.ctx.close()

    def _rotate(self, layer, x, K, V, stride, count=1, positions=None, **where):
        """The queries of the tokens x, [count * m, kv * group, D]; their keys and values go to K and V, [count, kv, stride, D]."""
        m = x.shape[0] // count
        Q = torch.empty((count * m, self.kv * self.group, D), dtype=self.dtype, device="cuda")
        where.update(q_weight=self.norms[layer][0], k_weight=self.norms[layer][1])
        if self.axis_of is None:
            self.ctx.rotate(x @ self.qkv[layer], count, m, self.table, Q, K, V, stride, positions=positions, **where)
        else:
            self.ctx.rotate_axes(x @ self.qkv[layer], count, m, self.table, positions, self.axis_of, Q, K, V, stride, **where)
        return Q

    def prompt(self, x: torch.Tensor, positions=None, watch: int = 0) -> torch.Tensor:
        """x: [n, width]; fills the cache, [layers, kv, n, D].  positions: int32 [axes, n], with axes alone.  watch: how many of the last tokens' attention
        weights are summed, for hold."""
        self.n = n = x.shape[0]
        if (positions is None) != (self.axis_of is None):
            raise ValueError("axes need positions, and positions axes")
        self.last, w = n - 1 if positions is None else int(positions.max()), min(watch, n)
        self.K = torch.empty((self.layers, self.kv, n, D), dtype=self.dtype, device="cuda")
        self.V = torch.empty_like(self.K)
        self.mass = torch.empty((self.layers, self.kv, n), device="cuda") if w else None
        lse = torch.empty((self.kv * self.group, n), device="cuda") if w else None
        for i in range(self.layers):
            Q = self._rotate(i, x, self.K[i], self.V[i], n, positions=positions)
            o = torch.empty_like(Q)
            self.ctx.attend(Q, self.K[i], self.V[i], 1, n, n, n, o, window=self.window, n_sink=self.n_sink, lse=lse)
            if w:
                self.ctx.attend_weights(Q[n - w:], self.K[i], lse[:, n - w:].contiguous(), 1, w, n, n, self.mass[i], window=self.window, n_sink=self.n_sink,
                                        decay=0.0)
            x = x + o.view(n, -1) @ self.out[i]
        return x

    def hold(self, room: int, recent: int = 16, decay: float = 1.0) -> None:
        """The cache stays at `room` tokens (before the next one comes): the first ones, the last `recent`, and those that the most attention went to, from the
        prompt's watched tokens and, old attention counting `decay` of what it did a token before, from those since."""
        if self.window or self.mass is None:
            raise ValueError("hold takes a prompt whose last tokens were watched, and no window")
        if self.n < room:
            raise ValueError("the prompt is shorter than the room: keep_all")
        self.room, self.recent, self.decay = room, recent, decay
        shape = (self.layers, self.kv, room + 1)                    # (the token at hand comes last, until one has gone)
        self.held = [torch.zeros((*shape, D), dtype=self.dtype, device="cuda") for _ in "KV"]
        self.held += [torch.zeros(shape, device="cuda"), torch.zeros(shape, dtype=torch.int32, device="cuda")]
        self.rows_held = torch.empty((self.layers, self.kv, room), dtype=torch.int32, device="cuda")
        K, V, mass, tokens = self.held
        self.ctx.evict(self.K, self.V, self.mass, self.layers, self.n, self.n, room, self.rows_held, n_sink=self.n_sink, recent=recent, K_out=K, V_out=V,
                       mass_out=mass, positions_out=tokens, out_stride=room + 1)
        self.kept = self.held[:2]
        self._begin()
        self.place.fill_(room)                                      # (it does not move: the step puts a token there)
        self.counters = self.position, self.tokens

    def keep(self, share: float, bits4: bool = True, answers: int = 1) -> None:
        """Chooses the share of every head's tokens that stays, and holds their rows in 4 bits (or as they are).  answers: how many follow the prompt."""
        if self.window:
            raise ValueError("kept rows have no positions: with a window, keep_all")
        heads, n = self.layers * self.kv, self.n
        budgets = np.full(heads, max(min(n, self.n_sink), int(n * share)), dtype=np.int32)
        offsets = wl.offsets_for(budgets)
        total = int(offsets[-1])
        scores = torch.empty((heads, n), device="cuda")
        indices = torch.empty(total, dtype=torch.int32, device="cuda")
        self.ctx.scores(self.K, self.V, n, scores)
        self.ctx.select(scores, n, budgets, min(n, self.n_sink), offsets, indices)
        self.offsets, self.total, self.rows = torch.from_numpy(offsets).cuda(), total, int(budgets[0]) * self.kv
        if bits4:
            self.kept = [torch.empty((total, w), dtype=torch.uint8, device="cuda") for w in (64, 4, 64, 4)]
            self.ctx.compact_mx(self.K, self.V, n, indices, self.offsets, total, *self.kept)
        else:
            self.kept = [torch.empty((total, D), dtype=self.dtype, device="cuda") for _ in "KV"]
            self.ctx.compact(self.K, self.V, n, indices, offsets, *self.kept)
        self._begin(answers)

    def keep_all(self, answers: int = 1) -> None:
        """The whole prompt's cache is what is kept, where it lies; with a window, in a cache that has room for the tokens since."""
        if self.window and answers > 1:
            raise ValueError("kept rows have no positions: with a window, one answer")
        if self.window:
            self.kept = [torch.zeros((self.layers, self.kv, self.n + self.stride, D), dtype=self.dtype, device="cuda") for _ in "KV"]
            for whole, rows in zip(self.kept, (self.K, self.V)):
                whole[:, :, :self.n] = rows
            self._begin()
            return
        self.offsets = torch.arange(self.layers * self.kv + 1, device="cuda") * self.n
        self.total, self.rows = self.layers * self.kv * self.n, self.kv * self.n
        self.kept = [self.K.view(-1, D), self.V.view(-1, D)]
        self._begin(answers)

    def _begin(self, answers: int = 1) -> None:
        self.answers, self.holds = answers, self.kept[0].dim() == 4 and not self.window
        shape = (self.layers, answers, self.kv, 0 if self.window or self.holds else self.stride, D)
        self.K_new, self.V_new = torch.zeros(shape, dtype=self.dtype, device="cuda"), torch.zeros(shape, dtype=self.dtype, device="cuda")
        # (on the device, so that a recorded step finds the present ones: tokens since the prompt, with the one at hand, its place among them and its position, tokens in all)
        self.length = torch.zeros(answers, dtype=torch.int32, device="cuda")
        self.place = torch.full((answers,), -1, dtype=torch.int32, device="cuda")
        self.position = torch.full((1 if self.axis_of is None else int(self.axis_of[-1]) + 1, answers), self.last, dtype=torch.int32, device="cuda")
        self.tokens = torch.full((1,), self.n, dtype=torch.int32, device="cuda")
        self.counters = self.length, self.place, self.position, self.tokens

    def step(self, x: torch.Tensor) -> torch.Tensor:
        """One generated token of every answer, x: [answers, width]."""
        for counter in self.counters:
            counter += 1
        if self.holds:
            K, V, mass, tokens = self.held
            mass[:, :, self.room] = 0
            tokens[:, :, self.room] = self.tokens - 1
        attend = self._in_window if self.window else self._in_room if self.holds else self._over_kept
        for i in range(self.layers):
            x = x + attend(i, x).view(self.answers, -1) @ self.out[i]
        if self.holds:
            self.ctx.evict(K, V, mass, self.layers, self.room + 1, self.room + 1, self.room, self.rows_held, positions=tokens, n_sink=self.n_sink, recent=self.recent)
        return x

    def _over_kept(self, i, x):
        Q = self._rotate(i, x, self.K_new[i], self.V_new[i], self.stride, self.answers, starts=self.place, positions=self.position)
        o = torch.empty_like(Q)
        since = dict(K_tail=self.K_new[i], V_tail=self.V_new[i], tail_n=self.stride, tail_stride=self.stride, tail_lengths=self.length, rows=self.rows)
        if self.answers > 1:
            attend = self.ctx.attend_shared if len(self.kept) == 2 else self.ctx.attend_shared_mx
            attend(Q, *self.kept, self.offsets[i * self.kv:], 1, self.answers, 1, self.total, o, **since)
        else:
            attend = self.ctx.attend_kept if len(self.kept) == 2 else self.ctx.attend_kept_mx
            attend(Q, *self.kept, self.offsets[i * self.kv:], 1, 1, self.total, o, **since)
        return o

    def _in_room(self, i, x):
        (K, V, mass), n = [t[i] for t in self.held[:3]], self.room + 1
        Q = self._rotate(i, x, K, V, n, starts=self.place, positions=self.position)
        o, lse = torch.empty_like(Q), torch.empty(self.kv * self.group, device="cuda")
        self.ctx.attend(Q, K, V, 1, 1, n, n, o, lse=lse)
        self.ctx.attend_weights(Q, K, lse, 1, 1, n, n, mass, decay=self.decay)
        return o

    def _in_window(self, i, x):
        K, V, room = self.kept[0][i], self.kept[1][i], self.n + self.stride
        Q = self._rotate(i, x, K, V, room, starts=self.position, positions=self.position)
        o = torch.empty_like(Q)
        self.ctx.attend(Q, K, V, 1, 1, room, room, o, lengths=self.tokens, window=self.window, n_sink=self.n_sink)
        return o

    def generate(self, x: torch.Tensor, count: int):
        """`count` tokens of every answer, each the one before made into unit length, by replays of one recorded step.  Returns them, [count, width] or
        [count, answers, width], and the seconds a replay took."""
        def following(y):
            return (y.float() * torch.rsqrt(y.float().square().mean(-1, keepdim=True) + 1e-6)).to(self.dtype)
        given = x.clone()
        side = torch.cuda.Stream()                  # (libraries set themselves up in a call that is not recorded)
        side.wait_stream(torch.cuda.current_stream())
        changed = [*self.counters, *(self.held if self.holds else [])]
        with torch.cuda.stream(side):
            before = [t.clone() for t in changed]
            self.step(given)
            for t, was in zip(changed, before):
                t.copy_(was)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = self.step(given)
            given.copy_(following(y))
        out = torch.empty((count, *x.shape[x.shape[0] == 1:]), dtype=self.dtype, device="cuda")
        torch.cuda.synchronize()
        begin = time.perf_counter()
        for i in range(count):
            graph.replay()
            out[i] = y[0] if y.shape[0] == 1 else y
        torch.cuda.synchronize()
        return out, (time.perf_counter() - begin) / count


def main(argv=None) -> None:
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--layers", type=int, default=8)
    p.add_argument("--kv-heads", type=int, default=8)
    p.add_argument("--group", type=int, default=4)
    p.add_argument("--tokens", type=int, default=32768)
    p.add_argument("--new", type=int, default=64)
    p.add_argument("--keep", type=float, default=0.1)
    p.add_argument("--window", type=int, default=0)
    p.add_argument("--hold", type=int, default=0, help="tokens that the cache stays at")
    p.add_argument("--answers", type=int, default=1, help="answers that follow the prompt at once")
    p.add_argument("--axes", type=int, nargs="*", default=[], help="how many of the 64 angles turn by each of two axes' positions")
    a = p.parse_args(argv)
    if a.axes and (len(a.axes) != 2 or sum(a.axes) != D // 2):
        p.error(f"--axes takes two numbers that add up to {D // 2}")
    if a.window and (a.hold or a.answers > 1):
        p.error("--hold and --answers go without a window")
    model = Decoder(a.layers, a.kv_heads, a.group, a.tokens, a.new + 1, window=a.window, axes=a.axes)
    x = torch.randn((a.tokens, a.kv_heads * a.group * D), generator=torch.Generator().manual_seed(2)).to("cuda", model.dtype)
    token, side = torch.arange(a.tokens, dtype=torch.int32, device="cuda"), int(a.tokens ** 0.5)
    positions, watch = torch.stack([token // side, token % side]) if a.axes else None, 32 if a.hold else 0
    model.prompt(x[:64], positions[:, :64].contiguous() if a.axes else None, watch)         # (first calls load code)
    torch.cuda.synchronize()
    begin = time.perf_counter()
    y = model.prompt(x, positions, watch)
    torch.cuda.synchronize()
    print(f"prompt of {a.tokens} tokens, {a.layers} layers: {(time.perf_counter() - begin) * 1e3:.1f} ms", flush=True)
    first = y[-1:].clone()
    results = {}
    runs = [("whole cache, bf16", model.keep_all), (f"{a.keep:.0%}, bf16", lambda: model.keep(a.keep, False)), (f"{a.keep:.0%}, 4 bits", lambda: model.keep(a.keep))]
    if a.hold:
        runs.append((f"held at {a.hold} tokens", lambda: model.hold(a.hold, min(16, a.hold // 2))))
    if a.answers > 1:
        runs.append((f"{a.answers} answers over the whole cache", lambda: model.keep_all(a.answers)))
        runs.append((f"{a.answers} answers over {a.keep:.0%}, 4 bits", lambda: model.keep(a.keep, True, a.answers)))
    for name, choose in runs:
        if model.window and name != "whole cache, bf16":
            print(f"{name}: left out, kept rows have no positions that the window could pass", flush=True)
            continue
        choose()
        results[name], seconds = model.generate(first.expand(model.answers, -1).contiguous(), a.new)
        held = sum(t.numel() * t.element_size() for t in model.kept)
        whole = results["whole cache, bf16"].double()
        likeness = torch.nn.functional.cosine_similarity(results[name].double().view(a.new, model.answers, -1)[:, 0], whole, dim=-1)
        print(f"{name}: {held / 1e6:.1f} MB held, {seconds * 1e6:.0f} us a token, first token's cosine with the whole cache's {likeness[0]:.4f}", flush=True)
    model.close()


if __name__ == "__main__":
    main()
