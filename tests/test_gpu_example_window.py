"""The small decoder with a window: the tokens that it generates see what the prompt's see."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
D = 128


def plain(model, x, window, sinks):
    """The stack over all tokens x at once in 64 bits, every token seeing the `window` last ones and the first `sinks`."""
    x, table = x.double().cpu(), model.table.double().cpu()
    n, queries = x.shape[0], model.kv * model.group
    p, j = torch.arange(n)[:, None], torch.arange(n)[None]
    seen = (j <= p) & ((p - j < window) | (j < sinks))

    def turned(z, g):
        z = z / torch.sqrt(z.square().mean(-1, keepdim=True) + 1e-5) * g.double().cpu()
        a, b, c, s = z[..., :64], z[..., 64:], table[:n, 0][:, None], table[:n, 1][:, None]
        return torch.cat([a * c - b * s, b * c + a * s], -1)

    for i in range(model.layers):
        y = (x @ model.qkv[i].double().cpu()).view(n, -1, D)
        q, k, v = turned(y[:, :queries], model.norms[i][0]), turned(y[:, queries:queries + model.kv], model.norms[i][1]), y[:, queries + model.kv:]
        heads = []
        for h in range(queries):
            s = (q[:, h] @ k[:, h // model.group].T) / math.sqrt(D)
            heads.append(s.masked_fill(~seen, -math.inf).softmax(-1) @ v[:, h // model.group])
        x = x + torch.cat(heads, 1) @ model.out[i].double().cpu()
    return x


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("window,sinks", [(30, 4), (64, 0), (1, 0)])
def test_prompt_and_steps(dtype, window, sinks):
    from paper_2509_15038_amd.example import Decoder
    n, new = 203, 5
    model = Decoder(2, 2, 4, n, new + 1, dtype=dtype, window=window, n_sink=sinks, sketch_dim=16, seed=3)
    x = torch.randn((n + new, 1024), generator=torch.Generator().manual_seed(4)).to("cuda", model.dtype)
    want = plain(model, x, window, sinks)
    # (as without a window: about ten roundings a layer of 2^-9 relative to values of size 1 to 3 in bf16)
    tolerance = 2 * 10 * 3 * 2.0 ** -9 if dtype == "bf16" else 1e-3
    assert (model.prompt(x[:n]).double().cpu() - want[:n]).abs().max() < tolerance
    model.keep_all()
    for i in range(new):
        y = model.step(x[n + i:n + i + 1])
        assert (y[0].double().cpu() - want[n + i]).abs().max() < tolerance, i
    with pytest.raises(ValueError):
        model.keep(0.5)
    model.close()


def test_recorded_steps_are_the_eager_ones():
    from paper_2509_15038_amd.example import Decoder
    n, new = 1000, 6
    model = Decoder(3, 2, 4, n, new + 2, window=300, sketch_dim=16, seed=5)
    first = model.prompt(torch.randn((n, 1024), generator=torch.Generator().manual_seed(6)).to("cuda", model.dtype))[-1:].clone()
    model.keep_all()
    recorded, _ = model.generate(first, new)
    model.keep_all()
    y = first
    for i in range(new):
        z = model.step(y)
        torch.cuda.synchronize()
        assert torch.equal(z[0], recorded[i])
        y = (z.float() * torch.rsqrt(z.float().square().mean(-1, keepdim=True) + 1e-6)).to(model.dtype)
    model.close()


def test_command_with_a_window(capsys):
    from paper_2509_15038_amd import example
    example.main(["--layers", "2", "--kv-heads", "2", "--tokens", "2000", "--new", "3", "--window", "500"])
    lines = capsys.readouterr().out.splitlines()
    assert lines[1].startswith("whole cache") and "us a token" in lines[1] and all("left out" in line for line in lines[2:])
