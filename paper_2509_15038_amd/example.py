"""A small decoder around a compressed cache: every entry point of the attention side in the place where a program calls it.

    python -m paper_2509_15038_amd.example --layers 8 --tokens 32768 --keep 0.1 --new 64

A stack of attention layers with random weights (x + Wo attention(Wqkv x), grouped heads, rotary positions, RMS norms of a head's queries and
keys) takes a prompt, chooses the tokens whose keys and values it keeps, holds those in 4 bits and generates over them and the tokens since, one
step a HIP graph replay; beside it the same over the whole prompt's cache.  With a window it generates over the whole cache alone: kept rows have no
positions that a window could pass.  The products with weights are torch's, all else is the library's."""
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
                 sketch_dim: int = 64, seed: int = 1):
        self.layers, self.kv, self.group, self.window, self.n_sink, self.stride = layers, kv_heads, group, window, n_sink, new_tokens
        self.dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.ctx = B.Context(layers, kv_heads, group, D, sketch_dim, dtype, max_tokens + (new_tokens if window else 0), seed=seed)
        self.table = rotary_table(max_tokens + new_tokens)
        width = kv_heads * group * D
        draw = torch.Generator().manual_seed(seed)

        def weight(rows, columns):
            return (torch.randn((rows, columns), generator=draw) * rows ** -0.5).to("cuda", self.dtype)
        self.qkv = [weight(width, width + 2 * kv_heads * D) for _ in range(layers)]
        self.out = [weight(width, width) for _ in range(layers)]
        self.norms = [[(1 + 0.1 * torch.randn(D, generator=draw)).to("cuda", self.dtype) for _ in "qk"] for _ in range(layers)]

    def close(self):
        self.ctx.close()

    def _rotate(self, layer, x, K, V, stride, **where):
        """The queries of the tokens x, [m, kv * group, D]; their keys and values go to K and V, [kv, stride, D]."""
        m = x.shape[0]
        Q = torch.empty((m, self.kv * self.group, D), dtype=self.dtype, device="cuda")
        self.ctx.rotate(x @ self.qkv[layer], 1, m, self.table, Q, K, V, stride, q_weight=self.norms[layer][0], k_weight=self.norms[layer][1], **where)
        return Q

    def prompt(self, x: torch.Tensor) -> torch.Tensor:
        """x: [n, width]; fills the cache, [layers, kv, n, D]."""
        self.n = n = x.shape[0]
        self.K = torch.empty((self.layers, self.kv, n, D), dtype=self.dtype, device="cuda")
        self.V = torch.empty_like(self.K)
        for i in range(self.layers):
            Q = self._rotate(i, x, self.K[i], self.V[i], n)
            o = torch.empty_like(Q)
            self.ctx.attend(Q, self.K[i], self.V[i], 1, n, n, n, o, window=self.window, n_sink=self.n_sink)
            x = x + o.view(n, -1) @ self.out[i]
        return x

    def keep(self, share: float, bits4: bool = True) -> None:
        """Chooses the share of every head's tokens that stays, and holds their rows in 4 bits (or as they are)."""
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
        self._begin()

    def keep_all(self) -> None:
        """The whole prompt's cache is what is kept, where it lies; with a window, in a cache that has room for the tokens since."""
        if self.window:
            self.kept = [torch.zeros((self.layers, self.kv, self.n + self.stride, D), dtype=self.dtype, device="cuda") for _ in "KV"]
            for whole, rows in zip(self.kept, (self.K, self.V)):
                whole[:, :, :self.n] = rows
            self._begin()
            return
        self.offsets = torch.arange(self.layers * self.kv + 1, device="cuda") * self.n
        self.total, self.rows = self.layers * self.kv * self.n, self.kv * self.n
        self.kept = [self.K.view(-1, D), self.V.view(-1, D)]
        self._begin()

    def _begin(self) -> None:
        shape = (self.layers, self.kv, 0 if self.window else self.stride, D)
        self.K_new, self.V_new = torch.zeros(shape, dtype=self.dtype, device="cuda"), torch.zeros(shape, dtype=self.dtype, device="cuda")
        # (on the device, so that a recorded step finds the present ones: tokens since the prompt, with the one at hand, its place among them and its position, tokens in all)
        self.length = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.place = torch.full((1,), -1, dtype=torch.int32, device="cuda")
        self.position = torch.full((1,), self.n - 1, dtype=torch.int32, device="cuda")
        self.tokens = torch.full((1,), self.n, dtype=torch.int32, device="cuda")
        self.counters = self.length, self.place, self.position, self.tokens

    def step(self, x: torch.Tensor) -> torch.Tensor:
        """One generated token, x: [1, width]."""
        for counter in self.counters:
            counter += 1
        for i in range(self.layers):
            x = x + (self._in_window(i, x) if self.window else self._over_kept(i, x)).view(1, -1) @ self.out[i]
        return x

    def _over_kept(self, i, x):
        attend = self.ctx.attend_kept if len(self.kept) == 2 else self.ctx.attend_kept_mx
        Q = self._rotate(i, x, self.K_new[i], self.V_new[i], self.stride, starts=self.place, positions=self.position)
        o = torch.empty_like(Q)
        attend(Q, *self.kept, self.offsets[i * self.kv:], 1, 1, self.total, o, K_tail=self.K_new[i], V_tail=self.V_new[i], tail_n=self.stride,
               tail_stride=self.stride, tail_lengths=self.length, rows=self.rows)
        return o

    def _in_window(self, i, x):
        K, V, room = self.kept[0][i], self.kept[1][i], self.n + self.stride
        Q = self._rotate(i, x, K, V, room, starts=self.position, positions=self.position)
        o = torch.empty_like(Q)
        self.ctx.attend(Q, K, V, 1, 1, room, room, o, lengths=self.tokens, window=self.window, n_sink=self.n_sink)
        return o

    def generate(self, x: torch.Tensor, count: int):
        """`count` tokens, each the one before made into unit length, by replays of one recorded step.  Returns them, [count, width], and the seconds a
        replay took."""
        def following(y):
            return (y.float() * torch.rsqrt(y.float().square().mean(-1, keepdim=True) + 1e-6)).to(self.dtype)
        given = x.clone()
        side = torch.cuda.Stream()                  # (libraries set themselves up in a call that is not recorded)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            self.step(given)
            for c in self.counters:
                c -= 1
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = self.step(given)
            given.copy_(following(y))
        out = torch.empty((count, x.shape[1]), dtype=self.dtype, device="cuda")
        torch.cuda.synchronize()
        begin = time.perf_counter()
        for i in range(count):
            graph.replay()
            out[i] = y[0]
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
    a = p.parse_args(argv)
    model = Decoder(a.layers, a.kv_heads, a.group, a.tokens, a.new + 1, window=a.window)
    x = torch.randn((a.tokens, a.kv_heads * a.group * D), generator=torch.Generator().manual_seed(2)).to("cuda", model.dtype)
    model.prompt(x[:64])                            # (first calls load code)
    torch.cuda.synchronize()
    begin = time.perf_counter()
    y = model.prompt(x)
    torch.cuda.synchronize()
    print(f"prompt of {a.tokens} tokens, {a.layers} layers: {(time.perf_counter() - begin) * 1e3:.1f} ms", flush=True)
    first = y[-1:].clone()
    results = {}
    for name, choose in (("whole cache, bf16", model.keep_all), (f"{a.keep:.0%}, bf16", lambda: model.keep(a.keep, False)), (f"{a.keep:.0%}, 4 bits", lambda: model.keep(a.keep))):
        if model.window and name != "whole cache, bf16":
            print(f"{name}: left out, kept rows have no positions that the window could pass", flush=True)
            continue
        choose()
        results[name], seconds = model.generate(first, a.new)
        held = sum(t.numel() * t.element_size() for t in model.kept)
        whole = results["whole cache, bf16"].double()
        likeness = torch.nn.functional.cosine_similarity(results[name].double(), whole, dim=-1)
        print(f"{name}: {held / 1e6:.1f} MB held, {seconds * 1e6:.0f} us a token, first token's cosine with the whole cache's {likeness[0]:.4f}", flush=True)
    model.close()


if __name__ == "__main__":
    main()
