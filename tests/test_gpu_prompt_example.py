"""The decoding example's packed prompts and chunks: the prompts' operators together, on real caches."""

import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

from examples import decode as ex  # noqa: E402


def _plain_forward(decoder, x):
    """The decoder with head norms on one sequence bf16 [n,dim], causal, in 64 bits with the weights that were packed."""
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
        q, k = rotate(norm(q, layer.head_norms[0])), rotate(norm(k, layer.head_norms[1])).repeat_interleave(g, 1)
        z = (q.transpose(0, 1).contiguous() @ k.permute(1, 2, 0).contiguous()) * c.head_dim ** -0.5
        p = torch.softmax(z.masked_fill(~seen, -math.inf), -1)
        x = (p @ v.repeat_interleave(g, 1).transpose(0, 1).contiguous()).transpose(0, 1).reshape(n, -1) @ w["o"].T
        r = r + x
        gate, up = (norm(r, layer.norms[1]) @ w["gate_up"].T).chunk(2, -1)
        x = (gate * torch.sigmoid(gate) * up) @ w["down"].T
    return norm(r + x, decoder.final)


def _off(a, b):
    return float((a.double() - b.double()).norm() / b.double().norm())


def _inputs(c, lens, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return [torch.randn((n, c.dim), generator=g, device="cuda").bfloat16() for n in lens]


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
def test_packed_prompts_against_plain(cache):
    """All prompts in one pass, against each in 64 bits, and a chunk at a time against that pass.

    As for the decoding steps: an int4 code is 0.17 of sigma off, on W4A4 inputs and on their weights; with the residual
    stream's own share outputs stay within 0.35 of their norm.  Packed prompts and chunks differ in which keys attention
    reads, the rotated bf16 ones or the cache's, and by bf16 roundings that move a code here and there: 0.15 with a bf16
    cache.  An 8-bit cache's keys and values are 2^-4 / sqrt(12) = 0.02 to 0.04 off besides, below the int4 codes' own
    0.17: 0.2.
    """
    print(f"packed prompts {cache}", flush=True)
    c = ex.Config(layers=3, dim=512, heads=8, key_heads=2, ffn=1408, cache=cache, head_norm=True, fused=True)
    lens = [61, 40, 1, 130]
    decoder = ex.Decoder(c, 160)
    inputs = _inputs(c, lens, 7)
    kv = ex.Cache(c, 4, 144)
    whole = decoder.extend(inputs, kv)
    assert kv.lens.tolist() == lens
    for b, x in enumerate(inputs):
        assert _off(whole[b], _plain_forward(decoder, x)[-1]) < 0.35
    parts = ex.Cache(c, 4, 144)
    last = torch.zeros_like(whole)
    for i in range(0, max(lens), 32):
        y = decoder.extend([x[i: i + 32] for x in inputs], parts)
        for b, n in enumerate(lens):
            assert (i < n) or not y[b].any()
            if i < n:
                last[b] = y[b]
    assert parts.lens.tolist() == lens
    assert _off(last, whole) < (0.15 if cache == "bf16" else 0.2)


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
def test_chunks_beside_single_tokens(cache):
    """A pass that holds one sequence's next token and another's prompt gives each what it gets alone."""
    print(f"chunks beside tokens {cache}", flush=True)
    c = ex.Config(layers=2, dim=512, heads=8, key_heads=2, ffn=1408, cache=cache, fused=True)
    decoder = ex.Decoder(c, 160)
    a, b = _inputs(c, [50, 70], 9)
    mixed, apart = ex.Cache(c, 2, 96), ex.Cache(c, 2, 96)
    apart.table.copy_(mixed.table)
    for kv in (mixed, apart):
        decoder.extend([a[:49], b[:0]], kv)
    got = decoder.extend([a[49:], b], mixed)
    one = decoder.extend([a[49:], b[:0]], apart)
    two = decoder.extend([a[:0], b], apart)
    assert mixed.lens.tolist() == apart.lens.tolist() == [50, 70]
    assert not one[1].any() and not two[0].any()
    # other tiles, and so other orders of a product's sums, move bf16 roundings and with them a code here and there
    assert _off(got[0], one[0]) < 0.15 and _off(got[1], two[1]) < 0.15
    assert _off(two[1], decoder.prefill([b], ex.Cache(c, 1, 96))[0]) < 0.15
