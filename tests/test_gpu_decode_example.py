"""The decoding example: the operators together, on real caches."""

import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

from examples import decode as ex  # noqa: E402


def _plain_forward(decoder, x):
    """The decoder on one sequence bf16 [n,dim], causal, in 64 bits with the weights that were packed."""
    c = decoder.c
    x, r = x.double(), 0.0
    n = x.shape[0]

    def norm(v, w):
        return v / torch.sqrt((v * v).mean(-1, keepdim=True) + 1e-6) * w.double()

    def rotate(v):
        a, b = v.chunk(2, -1)
        cos, sin = decoder.cos[:n, None].double(), decoder.sin[:n, None].double()
        return torch.cat((a * cos - b * sin, a * sin + b * cos), -1)

    seen = torch.tril(torch.ones((n, n), dtype=torch.bool, device="cuda"))
    for layer in decoder.layers:
        w = {k: v.double() for k, v in layer.plain.items()}
        r = r + x
        qkv = (norm(r, layer.norms[0]) @ w["qkv"].T).view(n, -1, c.head_dim)
        q, k, v = qkv.split((c.heads, c.key_heads, c.key_heads), dim=1)
        g = c.heads // c.key_heads
        q, k, v = rotate(q), rotate(k).repeat_interleave(g, 1), v.repeat_interleave(g, 1)
        z = (q.transpose(0, 1).contiguous() @ k.permute(1, 2, 0).contiguous()) * c.head_dim ** -0.5
        p = torch.softmax(z.masked_fill(~seen, -math.inf), -1)
        x = (p @ v.transpose(0, 1).contiguous()).transpose(0, 1).reshape(n, -1) @ w["o"].T
        r = r + x
        gate, up = (norm(r, layer.norms[1]) @ w["gate_up"].T).chunk(2, -1)
        x = (gate * torch.sigmoid(gate) * up) @ w["down"].T
    return norm(r + x, decoder.final)


def _off(a, b):
    return float((a.double() - b.double()).norm() / b.double().norm())


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
def test_decode_against_plain(cache):
    """A prompt, then a token at a time from a replayed graph, against the whole sequence in 64 bits and in one pass.

    An int4 code stands for its value to a step / sqrt(12), a step being the row's largest / 7, about 4 sigma / 7: 0.17
    of sigma on W4A4 inputs, as much again on their weights.  The two W4A4 products of a layer are a part of what it
    adds to a residual stream, whose own share grows with every layer: outputs stay within 0.35 of their norm.  A step
    and the whole pass differ only where another order of a sum moves a bf16 rounding (2^-9 of a value) and that a code:
    one in a hundred by a step, 0.1 * 4 / 7 of sigma; 0.15 is asked.
    """
    print(f"decode {cache}", flush=True)
    c = ex.Config(layers=3, dim=512, heads=8, key_heads=2, ffn=1408, cache=cache)
    steps, lens = 6, [61, 40, 1]
    decoder = ex.Decoder(c, 128)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    inputs = [torch.randn((n + steps, c.dim), generator=g, device="cuda").bfloat16() for n in lens]
    kv = ex.Cache(c, 3, 80)
    got = [decoder.prefill([x[:n] for x, n in zip(inputs, lens)], kv)]
    x = torch.zeros((3, 1, c.dim), dtype=torch.bfloat16, device="cuda")
    graph, y = ex.graph_of(decoder, kv, x, 80)
    assert kv.lens.tolist() == lens
    eager_kv = ex.Cache(c, 3, 80)
    decoder.prefill([x[:n] for x, n in zip(inputs, lens)], eager_kv)
    for i in range(steps):
        x.copy_(torch.stack([s[n + i] for s, n in zip(inputs, lens)])[:, None])
        graph.replay()
        got.append(y[:, 0].clone())
        assert torch.equal(decoder.step(x, eager_kv, 80)[:, 0], got[-1]), "the graph and eager calls differ"
        torch.cuda.synchronize()
    assert kv.lens.tolist() == [n + steps for n in lens]
    got = torch.stack(got)
    whole = ex.Cache(c, 3, 80)
    for b, n in enumerate(lens):
        plain = _plain_forward(decoder, inputs[b])[n - 1:]
        assert _off(got[:, b], plain) < 0.35
        for i in range(steps + 1):
            one = decoder.prefill([s[: m + i] for s, m in zip(inputs, lens)], whole)[b]
            assert _off(got[i, b], one) < 0.15


def test_decode_block():
    """A block of tokens at once, as block diffusion decodes."""
    print("decode block", flush=True)
    c = ex.Config(layers=1, dim=512, heads=8, key_heads=2, ffn=1408)
    decoder = ex.Decoder(c, 256)
    kv = ex.Cache(c, 2, 160)
    decoder.prefill([torch.randn((n, c.dim), device="cuda").bfloat16() for n in (70, 33)], kv)
    y = decoder.step(torch.randn((2, 64, c.dim), device="cuda").bfloat16(), kv, 160)
    assert y.shape == (2, 64, c.dim) and bool(y.isfinite().all()) and kv.lens.tolist() == [134, 97]
