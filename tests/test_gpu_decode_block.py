"""The decoding example's block step (block diffusion: new tokens see the whole cache and each other) against 64 bits."""

import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

from examples import decode as ex  # noqa: E402

E4M3 = torch.float8_e4m3fn
OFF = 0.03


def _bf16(x):
    return x.bfloat16().double()


def _int4(y):
    """The values that int4 codes of y's rows stand for."""
    s = y.abs().amax(1, keepdim=True) / 7
    return torch.where(s > 0, (y / s).round().clamp(-8, 7), 0.0) * s


def _e4m3(y):
    """The values that e4m3 codes of y's last dimension, with a scale for each 128, stand for."""
    n = y.shape[-1]
    pad = torch.nn.functional.pad(y, (0, -n % 128)).view(*y.shape[:-1], -1, 128)
    s = pad.abs().amax(-1, keepdim=True) / 448
    return (torch.where(s > 0, pad / s, 0.0).float().to(E4M3).double() * s).flatten(-2)[..., :n]


def _int4_weight(wq, ws):
    lo, hi = (wq & 15).to(torch.int8), (wq >> 4).to(torch.int8)
    q = torch.stack((lo, hi), 2).flatten(1)
    return torch.where(q > 7, q - 16, q).double() * ws.double()[:, None]


def _fp8_weight(wq, ws):
    return wq.double() * ws.double().repeat_interleave(128, 0)[:wq.shape[0]].repeat_interleave(128, 1)[:, :wq.shape[1]]


def _attention(decoder, layer, x, r, seen):
    """What a layer's attention gives, 64 bits [n, heads * head_dim], on the sums x + r of a sequence that enter the layer,
    token i seeing the tokens that seen[i] names; packed weights, and a rounding wherever the operators state one."""
    c, n = decoder.c, x.shape[0]

    def rotate(v):
        a, b = v.chunk(2, -1)
        cos, sin = decoder.cos[:n, None].double(), decoder.sin[:n, None].double()
        return torch.cat((a * cos - b * sin, a * sin + b * cos), -1)

    def cached(v):
        return _bf16(v) if c.cache == "bf16" else _e4m3(v)  # heads are no longer than 128

    h = _norm(x.double() + r.double(), layer.norms[0])
    qkv = _bf16(_int4(h) @ _int4_weight(*layer.qkv).t()).view(n, -1, c.head_dim)
    q, k, v = qkv.split((c.heads, c.key_heads, c.key_heads), dim=1)
    g = c.heads // c.key_heads
    q, k, v = _bf16(rotate(q)), cached(rotate(k)).repeat_interleave(g, 1), cached(v).repeat_interleave(g, 1)
    z = torch.matmul(q.transpose(0, 1).contiguous(), k.permute(1, 2, 0).contiguous()) * c.head_dim ** -0.5
    p = torch.softmax(z.masked_fill(~seen, -math.inf), -1)
    return torch.matmul(p, v.transpose(0, 1).contiguous()).transpose(0, 1).reshape(n, -1)


def _rest(layer, x, r, attended):
    """What leaves the layer, as the sum x + r, from what entered it and its attention's outputs."""
    r = _bf16(x.double() + r.double())
    h = _bf16(_int4(attended.double()) @ _int4_weight(*layer.o).t()) + r
    gate, up = _bf16(_e4m3(_norm(h, layer.norms[1])) @ _fp8_weight(*layer.gate_up).t()).chunk(2, 1)
    x = _bf16(_bf16(gate * torch.sigmoid(gate)) * up)
    return _bf16(_e4m3(x) @ _fp8_weight(*layer.down).t()) + _bf16(h)


def _norm(h, w):
    return h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6) * w.double()


def _off(a, b):
    return float((a.double() - b.double()).norm() / b.double().norm())


class Recorder:
    """The sums that enter the norms and the attention's outputs, of every pass, kept for each layer and sequence."""

    def __init__(self, monkeypatch, layers, batch):
        self.norms, self.attends, self.layers = [], [], layers
        self.entered = [[[] for _ in range(batch)] for _ in range(layers + 1)]  # (x, r) of the last: the final norm's
        self.attended = [[[] for _ in range(batch)] for _ in range(layers)]
        norm, attend = ex.jb.jq_rmsnorm, ex.jb.jq_paged_attention

        def recorded_norm(x, w, residual=None, **kw):
            self.norms.append((x.clone(), residual.clone()))
            return norm(x, w, residual=residual, **kw)

        def recorded_attend(*args, **kw):
            out = attend(*args, **kw)
            self.attends.append(out.flatten(2).clone())
            return out

        monkeypatch.setattr(ex.jb, "jq_rmsnorm", recorded_norm)
        monkeypatch.setattr(ex.jb, "jq_paged_attention", recorded_attend)

    def deal(self, sequences):
        """The passes since the last call, of which each had the same number of tokens of these sequences."""
        per = len(sequences)
        for i in range(self.layers + 1):
            x, r = self.norms[2 * i]
            for b, xs, rs in zip(sequences, x.chunk(per), r.chunk(per)):
                self.entered[i][b].append((xs, rs))
        for i in range(self.layers):
            for b, o in zip(sequences, self.attends[i]):
                self.attended[i][b].append(o)
        self.norms, self.attends = [], []

    def entering(self, layer, b):
        return [torch.cat(t) for t in zip(*self.entered[layer][b])]


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("block", [64, 5])
def test_block_steps_against_plain(block, cache, monkeypatch):
    """Two block steps after prompts of different lengths: every layer on the sums that entered it, for each sequence.

    Attention's inputs and the plain pass's differ by the bf16 outputs that fall on the other side of a tie, its outputs by
    their rounding, 2^-9 each in rms: below 0.01.  Behind it e4m3 and int4 codes fall on the other side of a tie where
    their input does; a difference of d in rms changes sqrt(0.09 d) of what a product of e4m3 codes gives (a step is 0.09
    of a value), so d = 0.001 becomes 0.01, and 0.03 of the second product, which is a third of what leaves the layer.
    0.03 is asked of both.  A causal block, a block that does not see the cache and another sequence's lie outside it.
    """
    print(f"[gpu-decode] block {block} {cache}", flush=True)
    c = ex.Config(layers=2, dim=512, heads=8, key_heads=2, ffn=1408, cache=cache)
    decoder = ex.Decoder(c, 256)
    g = torch.Generator(device="cuda")
    g.manual_seed(31)
    lens = [70, 33, 1]
    inputs = [torch.randn((n + 2 * block, c.dim), generator=g, device="cuda").bfloat16() for n in lens]
    kv = ex.Cache(c, 3, 208)
    rec = Recorder(monkeypatch, 2, 3)
    for b in range(3):
        one = ex.Cache(c, 1, 208)
        one.kv, one.scales, one.table, one.lens = kv.kv, kv.scales, kv.table[b:b + 1], kv.lens[b:b + 1]
        decoder.prefill([inputs[b][:lens[b]]], one)
        rec.deal([b])
    for step in range(2):
        at = [n + step * block for n in lens]
        y = decoder.step(torch.stack([x[i: i + block] for x, i in zip(inputs, at)]), kv, 208)
        rec.deal([0, 1, 2])
        assert kv.lens.tolist() == [i + block for i in at]
        for b, n in enumerate(at):
            total = n + block
            causal = torch.tril(torch.ones((total, total), dtype=torch.bool, device="cuda"))
            seen = causal.clone()
            for s in range(step + 1):  # every block that has been taken sees all of itself
                first = lens[b] + s * block
                seen[first: first + block, first: first + block] = True
            alone = seen.clone()
            alone[n:, :n] = False
            for i, layer in enumerate(decoder.layers):
                x, r = rec.entering(i, b)
                assert x.shape[0] == total and (i or torch.equal(x, inputs[b][:total]))
                got = torch.cat(rec.attended[i][b])
                plain = _attention(decoder, layer, x, r, seen)
                assert _off(got[n:], plain[n:]) < OFF, (step, b, i)
                for other in (causal, alone):
                    assert _off(_attention(decoder, layer, x, r, other)[n:], plain[n:]) > OFF, (step, b, i)
                assert _off(rec.attended[i][(b + 1) % 3][-1], plain[n:]) > OFF
                x2, r2 = (t[n:].double() for t in rec.entering(i + 1, b))
                assert _off(x2 + r2, _rest(layer, x, r, got)[n:]) < OFF, (step, b, i)
            x, r = (t[n:].double() for t in rec.entering(2, b))
            assert _off(y[b], _norm(x + r, decoder.final)) < OFF
