"""A small decoder served with the library's operators: prompts of different
lengths go through one causal pass, packed (or a chunk of each at a time), then
every sequence gets new tokens, one at a time (or a block at a time, as block
diffusion decodes), from a replayed HIP graph.

    python -m examples.decode [--batch 8] [--prompt 500] [--chunk 0] [--new 32] [--block 1] [--cache fp8]

Weights are random and the embedding of the next token is the block's last
output, so what it shows is the operators at work and what they take, not text.

A layer, on rows of tokens with the residual stream r:

    h, r = norm(x, r) as int4        -> W4A4 product: q, k, v
    (norm each head of q and k,) rotate q and k, append k and v to the paged cache
    attention over the cache, or the packed prompts' own keys -> W4A4 linear
    h, r = norm(., r) as e4m3        -> 8-bit product: gate, up
    silu(gate) * up                  -> 8-bit linear (as e4m3 at once, with `fused`)
"""

import argparse
import dataclasses
import time

import torch
import torch.nn.functional as F

from paper_2609_33601_amd import jq
from paper_2609_33601_amd import jq_block as jb


@dataclasses.dataclass
class Config:
    layers: int = 4
    dim: int = 1024
    heads: int = 16
    key_heads: int = 4
    head_dim: int = 64
    ffn: int = 2816
    page: int = 16
    base: float = 10000.0
    cache: str = "fp8"  # or "bf16"
    head_norm: bool = False  # an RMS norm of each head of q and k before the rotation
    fused: bool = False  # the gated activation written as the 8-bit product's codes


class Layer:
    def __init__(self, c, gen):
        def randn(n, k, scale=1.0):
            return (torch.randn((n, k), generator=gen, device="cuda") * scale * k ** -0.5).bfloat16()

        qkv = (c.heads + 2 * c.key_heads) * c.head_dim
        self.plain = {  # what the packed weights stand for
            "qkv": randn(qkv, c.dim), "o": randn(c.dim, c.heads * c.head_dim, 0.5),
            "gate_up": randn(2 * c.ffn, c.dim), "down": randn(c.dim, c.ffn, 0.5),
        }
        self.norms = [(1 + 0.1 * torch.randn((c.dim,), generator=gen, device="cuda")).bfloat16() for _ in range(2)]
        self.head_norms = [(1 + 0.1 * torch.randn((c.head_dim,), generator=gen, device="cuda")).bfloat16()
                           for _ in range(2)] if c.head_norm else None
        self.qkv, self.o = (jq.jq_pack_weight_int4(self.plain[n]) for n in ("qkv", "o"))
        self.gate_up, self.down = (jb.jq_pack_weight_fp8(self.plain[n]) for n in ("gate_up", "down"))


class Cache:
    """Pages for every layer, dealt to sequences in order; a serving program would keep a free list."""

    def __init__(self, c, batch, tokens):
        self.page, self.columns = c.page, -(-tokens // c.page)
        pages = batch * self.columns
        kind = torch.float8_e4m3fn if c.cache == "fp8" else torch.bfloat16
        shape = (pages, c.key_heads, c.page, c.head_dim)
        self.kv = [[torch.zeros(shape, dtype=kind, device="cuda") for _ in range(2)] for _ in range(c.layers)]
        self.scales = [[torch.zeros(shape[:3], device="cuda") if c.cache == "fp8" else None for _ in range(2)]
                       for _ in range(c.layers)]
        self.table = torch.randperm(pages, device="cuda").int().view(batch, self.columns)
        self.lens = torch.zeros((batch,), dtype=torch.int32, device="cuda")

    def slots(self, sequences, positions):
        at = self.table[sequences, (positions // self.page).long()].long()
        return at * self.page + positions % self.page


class Decoder:
    def __init__(self, config, max_tokens, seed=0):
        self.c = c = config
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.layers = [Layer(c, gen) for _ in range(c.layers)]
        self.final = torch.ones((c.dim,), dtype=torch.bfloat16, device="cuda")
        freq = c.base ** (-torch.arange(0, c.head_dim, 2, device="cuda", dtype=torch.float64) / c.head_dim)
        angle = torch.arange(max_tokens, device="cuda", dtype=torch.float64)[:, None] * freq
        self.cos, self.sin = angle.cos().float(), angle.sin().float()

    def forward(self, x, positions, slots, attend, cache, dense=False):
        """x bf16 [T,dim], the new tokens of all sequences; attend(layer, q [T,heads,head_dim], k, v) is their attention
        (k, rotated, only if `dense`, which takes head norms; else None)."""
        c, T = self.c, x.shape[0]
        r = torch.zeros_like(x)
        for i, layer in enumerate(self.layers):
            q4, s4, r = jb.jq_rmsnorm(x, layer.norms[0], residual=r, out="int4")
            qkv = jq.jq_w4a4_gemm(q4, s4, *layer.qkv).view(T, c.heads + 2 * c.key_heads, c.head_dim)
            q, k, v = qkv.split((c.heads, c.key_heads, c.key_heads), dim=1)
            where = (positions, self.cos, self.sin, slots, *cache.kv[i], *cache.scales[i])
            if c.head_norm:
                q, k = jb.jq_qk_norm_rope_append(q, k, v, *layer.head_norms, *where, dense_k=dense)
            else:
                q, k = jb.jq_rope_append(q, k, v, *where), None
            x = jq.jq_w4a4_linear(attend(i, q, k, v).reshape(T, -1), *layer.o)
            q8, s8, r = jb.jq_rmsnorm(x, layer.norms[1], residual=r, out="fp8")
            gate, up = jb.jq_fp8_gemm(q8, s8, *layer.gate_up).chunk(2, dim=1)
            if c.fused:
                x = jb.jq_fp8_gemm(*jb.jq_gated_act(gate, up, out="fp8"), *layer.down)
            else:
                x = jb.jq_fp8_linear(F.silu(gate) * up, *layer.down)
        return jb.jq_rmsnorm(x, self.final, residual=r)[0]

    def prefill(self, prompts, cache):
        """Each prompt bf16 [n,dim] in a causal pass of its own; returns its last token's output, [batch,dim]."""
        last = []
        for b, x in enumerate(prompts):
            n = x.shape[0]
            at = torch.arange(n, dtype=torch.int32, device="cuda")
            cache.lens[b] = n
            lens, table = cache.lens[b:b + 1], cache.table[b:b + 1]

            def attend(i, q, k, v):
                return jb.jq_paged_attention(q[None], *cache.kv[i], table, lens, *cache.scales[i], max_len=n)[0]

            last.append(self.forward(x, at, cache.slots(b, at), attend, cache)[-1])
        return torch.stack(last)

    def extend(self, chunks, cache):
        """A chunk bf16 [n,dim] (n may be 0) of new tokens of each sequence, packed into one causal pass: prompts, parts of
        prompts and single tokens side by side.  Returns each chunk's last output, [batch,dim] (0 for an empty one)."""
        c, new = self.c, [x.shape[0] for x in chunks]
        before = cache.lens.tolist()
        sequences = torch.repeat_interleave(torch.arange(len(new)), torch.tensor(new)).cuda()
        starts = torch.tensor([0] + new).cumsum(0).int()
        ends = starts[1:].long() - 1
        at = torch.cat([torch.arange(m, m + n, dtype=torch.int32) for n, m in zip(new, before)]).cuda()
        starts = starts.cuda()
        cache.lens += torch.tensor(new, dtype=torch.int32).cuda()
        # prompts from their first token on see their own keys alone, as they come out of the rotation
        dense, max_len = c.head_norm and not any(before), max(n + m for n, m in zip(new, before))

        def attend(i, q, k, v):
            if dense:
                return jb.jq_prompt_attention(q, k, v, starts)
            return jb.jq_chunk_attention(q, *cache.kv[i], cache.table, starts, cache.lens, *cache.scales[i],
                                         max_len=max_len)

        y = self.forward(torch.cat(chunks), at, cache.slots(sequences, at), attend, cache, dense)
        return torch.where(torch.tensor(new)[:, None].cuda() > 0, y[ends.clamp_min(0).cuda()], 0.0).to(y.dtype)

    def step(self, x, cache, max_len):
        """Appends a block x bf16 [batch,n,dim] to every sequence and returns its output; a block sees all of itself.
        Nothing here depends on a length that the host knows, so that a graph of it can be replayed."""
        B, n, dim = x.shape
        positions = (cache.lens[:, None] + torch.arange(n, dtype=torch.int32, device="cuda")).view(-1)
        sequences = torch.arange(B, device="cuda").repeat_interleave(n)
        slots = cache.slots(sequences, positions)
        cache.lens += n

        def attend(i, q, k, v):
            return jb.jq_paged_attention(q.view(B, n, *q.shape[1:]), *cache.kv[i], cache.table, cache.lens,
                                         *cache.scales[i], max_len=max_len, causal=False)

        return self.forward(x.reshape(B * n, dim), positions, slots, attend, cache).view(B, n, dim)


def graph_of(decoder, cache, x, max_len):
    """A graph of one step on x; capturing it leaves the cache's lengths as they were."""
    lens = cache.lens.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        decoder.step(x, cache, max_len)
    torch.cuda.current_stream().wait_stream(side)
    cache.lens.copy_(lens)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = decoder.step(x, cache, max_len)
    return graph, y


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--batch", type=int, default=8)
    p.add_argument("--prompt", type=int, default=500, help="longest prompt; the others are shorter")
    p.add_argument("--chunk", type=int, default=0, help="tokens of a prompt at a time (0: all of them)")
    p.add_argument("--new", type=int, default=32, help="steps")
    p.add_argument("--block", type=int, default=1, help="tokens of a step")
    p.add_argument("--cache", choices=("fp8", "bf16"), default="fp8")
    a = p.parse_args()
    if a.prompt < 0 or a.chunk < 0:
        p.error("--prompt and --chunk must not be negative")
    c = Config(cache=a.cache, head_norm=True, fused=True)
    tokens = a.prompt + (a.new + 1) * a.block
    decoder, cache = Decoder(c, tokens), Cache(c, a.batch, tokens)
    prompts = [torch.randn((max(1, a.prompt - 37 * b), c.dim), device="cuda").bfloat16() for b in range(a.batch)]

    torch.cuda.synchronize()
    t = time.perf_counter()
    longest = max(len(x) for x in prompts)
    chunk = a.chunk or longest
    last = torch.zeros((a.batch, c.dim), dtype=torch.bfloat16, device="cuda")
    for i in range(0, longest, chunk):
        y = decoder.extend([x[i: i + chunk] for x in prompts], cache)
        last = torch.where(torch.tensor([[i < len(x)] for x in prompts], device="cuda"), y, last)
    torch.cuda.synchronize()
    print(f"prompts: {sum(len(x) for x in prompts)} tokens in {1e3 * (time.perf_counter() - t):.2f} ms (first calls)")

    x = last[:, None].repeat(1, a.block, 1)
    graph, y = graph_of(decoder, cache, x, tokens)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(a.new):
        graph.replay()
        x.copy_(y)
    torch.cuda.synchronize()
    t = time.perf_counter() - t
    print(f"{a.new} steps of {a.batch} x {a.block} tokens: {1e6 * t / a.new:.1f} us a step, "
          f"{a.new * a.batch * a.block / t:.0f} tokens/s; lengths {cache.lens.tolist()}")


if __name__ == "__main__":
    main()
