"""The small decoder that runs the entry points together, against a plain one in 64 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def plain(model, x):
    """The stack over all tokens x at once in 64 bits."""
    import math
    D = 128
    x = x.double().cpu()
    n = x.shape[0]
    table = model.table.double().cpu()
    for i in range(model.layers):
        w, wo = model.qkv[i].double().cpu(), model.out[i].double().cpu()
        y = (x @ w).view(n, -1, D)
        queries = model.kv * model.group
        q, k, v = y[:, :queries], y[:, queries:queries + model.kv], y[:, queries + model.kv:]

        def turned(z, g):
            z = z / torch.sqrt(z.square().mean(-1, keepdim=True) + 1e-5) * g.double().cpu()
            a, b = z[..., :64], z[..., 64:]
            c, s = table[:n, 0][:, None], table[:n, 1][:, None]
            return torch.cat([a * c - b * s, b * c + a * s], -1)
        q, k = turned(q, model.norms[i][0]), turned(k, model.norms[i][1])
        k, v = k.repeat_interleave(model.group, 1), v.repeat_interleave(model.group, 1)
        s = torch.matmul(q.transpose(0, 1), k.permute(1, 2, 0).contiguous()) / math.sqrt(D)
        t = torch.arange(n)
        hidden = t[None, :] > t[:, None]
        p = s.masked_fill(hidden, -math.inf).softmax(-1)
        x = x + torch.matmul(p, v.transpose(0, 1).contiguous()).transpose(0, 1).reshape(n, -1) @ wo
    return x


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_prompt_and_steps(dtype):
    from paper_2509_15038_amd.example import Decoder
    n, new = 203, 5
    model = Decoder(2, 2, 4, 256, new + 1, dtype=dtype, sketch_dim=16, seed=3)
    x = torch.randn((n + new, 1024), generator=torch.Generator().manual_seed(4)).to("cuda", model.dtype)
    want = plain(model, x)
    got = model.prompt(x[:n])
    # bf16: a layer rounds projections, queries, keys, weights, results and sums, about ten roundings of 2^-9 relative (2^-8 at most) to values of size 1 to 3
    tolerance = 2 * 10 * 3 * 2.0 ** -9 if dtype == "bf16" else 1e-3
    assert (got.double().cpu() - want[:n]).abs().max() < tolerance
    model.keep_all()
    for i in range(new):
        y = model.step(x[n + i:n + i + 1])
        assert (y[0].double().cpu() - want[n + i]).abs().max() < tolerance
    model.close()


def test_recorded_steps_are_the_eager_ones():
    from paper_2509_15038_amd.example import Decoder
    n, new = 1000, 6
    model = Decoder(3, 2, 4, 1024, new + 2, sketch_dim=16, seed=5)
    x = torch.randn((n, 1024), generator=torch.Generator().manual_seed(6)).to("cuda", model.dtype)
    first = model.prompt(x)[-1:].clone()
    for choose in (model.keep_all, lambda: model.keep(0.3, False), lambda: model.keep(0.3)):
        choose()
        recorded, _ = model.generate(first, new)
        choose()
        y = first
        for i in range(new):
            z = model.step(y)
            torch.cuda.synchronize()
            assert torch.equal(z[0], recorded[i])
            y = (z.float() * torch.rsqrt(z.float().square().mean(-1, keepdim=True) + 1e-6)).to(model.dtype)
    model.close()


def test_what_is_kept_in_4_bits():
    from paper_2509_15038_amd.example import Decoder
    model = Decoder(2, 2, 4, 512, 4, sketch_dim=16, seed=7)
    model.prompt(torch.randn((400, 1024), generator=torch.Generator().manual_seed(8)).to("cuda", model.dtype))
    model.keep(0.25, False)
    rows = [t.clone() for t in model.kept]
    model.keep(0.25)
    for codes, scales, row in zip(model.kept[::2], model.kept[1::2], rows):
        out = torch.empty_like(row)
        model.ctx.expand_mx(codes, scales, model.total, out)
        most = row.double().view(-1, 4, 32).abs().amax(-1, keepdim=True)
        # the step between codes is at most 2 of 4 to 8 units that the largest one is; what lies beyond 6 of them goes to 6
        assert ((out - row).double().view(-1, 4, 32).abs() <= most / 4).all()
    model.close()


def test_command(capsys):
    from paper_2509_15038_amd import example
    example.main(["--layers", "2", "--kv-heads", "2", "--tokens", "2000", "--new", "3", "--window", "500"])
    assert capsys.readouterr().out.count("\n") == 4
