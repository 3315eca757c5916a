"""Performance cases of the operators that take whole prompts through a decoder block.

perf/operators.py measures what a decoding step runs; these are the operators
that a prompt, a chunk of one, or the tokens of an image run besides:

  rotate  per-head RMS norm of the queries and keys with their rotation, in one
          pass, the keys and values written into a paged cache (bf16 or e4m3),
          returned densely, or both;
  act     the gated activation between a block's two linears, act(gate) * up,
          written as bf16, or as e4m3 codes with a scale for each 128 columns
          (what the 8-bit linear reads);
  prompt  attention over packed sequences of different lengths, causal or not,
          with grouped heads, from the projections' own rows;
  chunk   attention of chunks of new tokens, packed, of different lengths,
          single tokens among them, over each sequence's paged cache.

With `own` false, run() computes an operator from elementary torch operations
in 32 bits; with `own` true it makes a user's calls.
"""

import math

import torch

own = False

DEV = "cuda"
E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
EPS = 1e-6

LISTED = [
    # one new token on its way into the cache: all latency
    dict(name="rotate_one_token", op="rotate", T=1, Hq=32, Hk=8, D=128, R=128, page=16, cache="bf16", dense=False,
         interleaved=False),
    # the tokens of an image: no cache, the keys are returned, neighbouring pairs turn together
    dict(name="rotate_image", op="rotate", T=4608, Hq=24, Hk=24, D=128, R=128, page=16, cache="none", dense=True,
         interleaved=True),
    # a prefill, half of each head rotated, into an 8-bit cache and densely for the prompt's own attention
    dict(name="rotate_prefill_fp8", op="rotate", T=8191, Hq=32, Hk=8, D=128, R=64, page=64, cache="fp8", dense=True,
         interleaved=False),
    # one token between the gate projection and the 8-bit down projection
    dict(name="act_one_token", op="act", M=1, N=12288, act="silu", gated=True, out="fp8"),
    # a ragged batch of an uneven width, plain bf16
    dict(name="act_ragged_bf16", op="act", M=2747, N=2816, act="gelu", gated=True, out="bf16"),
    # a prefill's, between the projections of an 8B model
    dict(name="act_prefill", op="act", M=8192, N=12288, act="silu", gated=True, out="fp8"),
    # a few short prompts, the first tokens of conversations: latency
    dict(name="prompt_short", op="prompt", B=3, Hq=32, Hk=8, D=64, length=77, keys=0, ragged=True, causal=True,
         lse=False),
    # the tokens of an image see each other
    dict(name="prompt_image", op="prompt", B=1, Hq=24, Hk=24, D=128, length=4608, keys=0, ragged=False, causal=False,
         lse=False),
    # a prefill batch of prompts of all lengths, packed
    dict(name="prompt_packed", op="prompt", B=8, Hq=32, Hk=8, D=128, length=4096, keys=0, ragged=True, causal=True,
         lse=True),
    # sixteen drafted tokens checked against a conversation of two thousand
    dict(name="chunk_draft", op="chunk", B=1, Hq=32, Hk=8, D=128, page=16, new=16, mix="equal", length=2080,
         ragged=False, cache="bf16", causal=True),
    # a serving batch: most sequences decode one token while two are at a chunk of their prompt, 8-bit cache
    dict(name="chunk_mixed_fp8", op="chunk", B=16, Hq=32, Hk=8, D=128, page=16, new=512, mix="mostly_one", length=8192,
         ragged=True, cache="fp8", causal=True),
    # a chunk of a long document
    dict(name="chunk_long", op="chunk", B=1, Hq=32, Hk=8, D=128, page=64, new=2048, mix="equal", length=32768,
         ragged=False, cache="bf16", causal=True),
]


def listed():
    return [dict(c) for c in LISTED]


def _log(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


HEADS = [(32, 32), (32, 8), (16, 16), (24, 24), (28, 4), (64, 8), (12, 2), (8, 1), (40, 8)]
ACTS = ("silu", "gelu", "gelu_tanh")
PAIRS = 2048 * 32 * 32768  # scores of the largest listed case, unmasked


def draw(rng):
    op = rng.choice(("rotate", "act", "prompt", "chunk"))
    if op == "act":
        N = 16 * _log(rng, 8, 1024)
        M = _log(rng, 1, max(1, min(16384, 8192 * 12288 // N)))
        return dict(op=op, M=M, N=N, act=rng.choice(ACTS), gated=rng.random() < 0.7, out=rng.choice(("bf16", "fp8")))
    Hq, Hk = rng.choice(HEADS)
    D = rng.choice((64, 128, 128, 256))
    page = rng.choice((16, 32, 64, 128))
    if op == "rotate":
        T = _log(rng, 1, max(1, 8191 * 48 * 128 // ((Hq + 2 * Hk) * D)))
        cache = rng.choice(("bf16", "fp8", "none"))
        return dict(op=op, T=T, Hq=Hq, Hk=Hk, D=D, R=rng.choice((D, D // 2)), page=page, cache=cache,
                    dense=cache == "none" or rng.random() < 0.5, interleaved=rng.random() < 0.5)
    B = _log(rng, 1, 16)
    room = PAIRS * 128 // (D * B * Hq)  # scores of a sequence and head
    if op == "prompt":
        length = _log(rng, 8, min(8192, math.isqrt(room)))
        keys = _log(rng, 8, max(8, min(8192, room // length))) if rng.random() < 0.2 else 0
        return dict(op=op, B=B, Hq=Hq, Hk=Hk, D=D, length=length, keys=keys, ragged=rng.random() < 0.7,
                    causal=rng.random() < 0.6, lse=rng.random() < 0.3)
    new = _log(rng, 1, 2048)
    length = _log(rng, max(16, new), max(16, new, min(32768, room // new, 8 * 32768 * 128 // (B * Hk * D))))
    return dict(op=op, B=B, Hq=Hq, Hk=Hk, D=D, page=page, new=new, mix=rng.choice(("equal", "ragged", "mostly_one")),
                length=length, ragged=rng.random() < 0.7, cache=rng.choice(("bf16", "fp8")), causal=rng.random() < 0.8)


# ---------------------------------------------------------------------------
# inputs


def _blocks(n):
    return -(-n // 128)


def lengths(case):
    """(new tokens, keys) of each sequence: the new tokens' own among the keys, but where a prompt has keys apart."""
    B, n = case["B"], case["length"]
    spread = [n] + [1 + (i * 7919 + n // 3) % n for i in range(1, B)]
    total = spread if case["ragged"] else [n] * B
    if case["op"] == "prompt":
        m = case["keys"]
        return total, ([m] + [1 + (i * 6151 + m // 2) % m for i in range(1, B)] if m else total)
    m = case["new"]
    new = {"equal": [m] * B, "ragged": [m] + [1 + (i * 5003 + m // 2) % m for i in range(1, B)],
           "mostly_one": [m if i % 8 == 0 else 1 for i in range(B)]}[case["mix"]]
    return [min(a, b) for a, b in zip(new, total)], total


def _starts(lens):
    return torch.tensor([0] + lens, device=DEV).cumsum(0).int()


def _cache(pages, Hk, page, D, kind, g):
    """A cache as an append leaves it: [pages, heads, page, D], and its scales or None."""
    x = torch.randn((pages, Hk, page, D), generator=g, device=DEV, dtype=torch.bfloat16)
    if kind == "bf16":
        return x, None
    s = x.abs().amax(-1).float() / E4M3_MAX
    x /= s.bfloat16().unsqueeze(-1)
    return x.clamp_(-E4M3_MAX, E4M3_MAX).to(E4M3), s


def _heads(tokens, counts, D, g, scale=1.0):
    """Views [tokens, heads, D] of one fused projection's rows."""
    x = torch.randn((tokens, sum(counts) * D), generator=g, device=DEV, dtype=torch.bfloat16) * scale
    return [p.view(tokens, -1, D) for p in x.split([c * D for c in counts], dim=1)]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = dict(case)
    if case["op"] == "act":
        M, N = case["M"], case["N"]
        x = torch.randn((M, 2 * N), generator=g, device=DEV, dtype=torch.bfloat16) * 2
        s["gate"], up = x.chunk(2, dim=1)  # views of the fused projection's rows
        s["up"] = up if case["gated"] else None
        return s
    Hq, Hk, D = case["Hq"], case["Hk"], case["D"]
    if case["op"] == "rotate":
        T, page = case["T"], case["page"]
        s["q"], s["k"], s["v"] = _heads(T, (Hq, Hk, Hk), D, g, 3.0)
        s["qw"], s["kw"] = ((1 + 0.2 * torch.randn((D,), generator=g, device=DEV)).bfloat16() for _ in range(2))
        P = 2 * T + 64
        s["pos"] = torch.randint(0, P, (T,), generator=g, device=DEV, dtype=torch.int32)
        freq = 10000.0 ** (-torch.arange(0, case["R"], 2, device=DEV, dtype=torch.float64) / case["R"])
        at = torch.arange(P, device=DEV, dtype=torch.float64)[:, None] * freq
        s["cos"], s["sin"] = at.cos().float(), at.sin().float()
        s["slots"] = s["kc"] = s["vc"] = s["ks"] = s["vs"] = None
        if case["cache"] != "none":
            pages = -(-T // page) + 3
            order = torch.randperm(pages, generator=g, device=DEV)
            t = torch.arange(T, device=DEV)
            s["slots"] = order[t // page] * page + t % page
            dt = torch.bfloat16 if case["cache"] == "bf16" else E4M3
            s["kc"], s["vc"] = (torch.zeros((pages, Hk, page, D), device=DEV).to(dt) for _ in range(2))
            if case["cache"] == "fp8":
                s["ks"], s["vs"] = (torch.zeros((pages, Hk, page), device=DEV) for _ in range(2))
        return s
    new, total = lengths(case)
    s["starts"], s["max_new"], s["max_len"] = _starts(new), max(new), max(total)
    if case["op"] == "prompt":
        if case["keys"]:
            s["q"], = _heads(sum(new), (Hq,), D, g, 1.5)
            s["k"], s["v"] = _heads(sum(total), (Hk, Hk), D, g)
            s["k_starts"] = _starts(total)
        else:
            s["q"], s["k"], s["v"] = _heads(sum(new), (Hq, Hk, Hk), D, g, 1.25)
            s["k_starts"] = None
        return s
    page = case["page"]
    s["q"] = torch.randn((sum(new), Hq, D), generator=g, device=DEV, dtype=torch.bfloat16) * 1.5
    need = [-(-n // page) for n in total]
    pages = sum(need) + 5
    s["kc"], s["ks"] = _cache(pages, Hk, page, D, case["cache"], g)
    s["vc"], s["vs"] = _cache(pages, Hk, page, D, case["cache"], g)
    order = torch.randperm(pages, generator=g, device=DEV).int()
    first = torch.tensor([0] + need[:-1], device=DEV).cumsum(0)[:, None]
    col = torch.arange(max(need), device=DEV)[None, :]
    used = col < torch.tensor(need, device=DEV)[:, None]
    s["table"] = torch.where(used, order[torch.where(used, first + col, 0)], 0).int()
    s["lens"] = torch.tensor(total, dtype=torch.int32, device=DEV)
    return s


# ---------------------------------------------------------------------------
# plain forms


def _scale(y):
    a = y.abs().amax(-1, keepdim=True)
    return torch.where(a > 0, (a / E4M3_MAX).clamp_min(2.0 ** -126), torch.zeros_like(a))


def _coded(y):
    """y's last axis under one scale -> (e4m3 codes, scale)."""
    f = _scale(y)
    return torch.where(f > 0, y / f, torch.zeros_like(y)).to(E4M3), f[..., 0]


def _act(s):
    x = s["gate"].float()
    if s["act"] == "silu":
        y = x / (1 + torch.exp(-x))
    elif s["act"] == "gelu":
        y = 0.5 * x * (1 + torch.erf(x * 0.5 ** 0.5))
    else:
        y = 0.5 * x * (1 + torch.tanh((2 / math.pi) ** 0.5 * (x + 0.044715 * x * x * x)))
    if s["up"] is not None:
        y = y * s["up"].float()
    if s["out"] == "bf16":
        return [y.bfloat16()]
    M, N = y.shape
    q, f = _coded(torch.nn.functional.pad(y, (0, -N % 128)).view(M, -1, 128))
    return [q.view(M, -1)[:, :N].contiguous(), f]


def _turned(x, w, s):
    """Norm over each head, then the rotation of its first R elements, fp32."""
    x = x.float()
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
    c, sn = (t[s["pos"].long()][:, None, :] for t in (s["cos"], s["sin"]))
    R = s["R"]
    r, rest = x[..., :R], x[..., R:]
    if s["interleaved"]:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack((a * c - b * sn, a * sn + b * c), -1).flatten(-2)
    else:
        a, b = r[..., : R // 2], r[..., R // 2 :]
        r = torch.cat((a * c - b * sn, a * sn + b * c), -1)
    return torch.cat((r, rest), -1)


def _put(cache, scales, slots, x):
    """x fp32 [T, heads, D] into the cache's slots."""
    page = cache.shape[2]
    at = (slots // page, slice(None), slots % page)
    if scales is None:
        cache[at] = x.to(cache.dtype)
    else:
        q, f = _coded(x)
        cache.view(torch.uint8)[at] = q.view(torch.uint8)
        scales[at] = f


def _rotate(s):
    q, k = _turned(s["q"], s["qw"], s).bfloat16(), _turned(s["k"], s["kw"], s)
    if s["kc"] is not None:
        _put(s["kc"], s["ks"], s["slots"], k)
        _put(s["vc"], s["vs"], s["slots"], s["v"].float())
    return [q, k.bfloat16() if s["dense"] else None, s["kc"], s["vc"], s["ks"], s["vs"]]


def _gather(cache, scales, table):
    """The cached rows of each sequence, fp32 [B, heads, tokens, D]."""
    B = table.shape[0]
    _, H, page, D = cache.shape
    if scales is None:
        x = cache[table.long()].float()
    else:
        x = cache.view(torch.uint8)[table.long()].view(E4M3).float() * scales[table.long()][..., None]
    return x.permute(0, 2, 1, 3, 4).reshape(B, H, -1, D)


def _padded(x, starts, most):
    """Packed rows [T, heads, D] as fp32 [B, heads, most, D]; places past a sequence's end hold some other row."""
    at = starts[:-1, None].long() + torch.arange(most, device=DEV)
    return x[at.clamp_max(x.shape[0] - 1)].float().permute(0, 2, 1, 3)


def _attend(q, k, v, starts, lens, most, causal):
    """q packed [T,Hq,D] over fp32 k, v [B,Hk,tokens,D] of `lens` tokens -> out [T,Hq,D], log-sum-exp [T,Hq], fp32."""
    T, Hq, D = q.shape
    B, Hk, n, _ = k.shape
    G = Hq // Hk
    new = starts.diff()
    x = _padded(q, starts, most).reshape(B, Hk, G * most, D)
    p = torch.matmul(x, k.transpose(2, 3)).mul_(D ** -0.5).view(B, Hk, G, most, n)
    last = lens[:, None].expand(B, most)
    if causal:
        last = last - new[:, None] + 1 + torch.arange(most, device=DEV)
    p.masked_fill_((torch.arange(n, device=DEV) >= last[:, :, None])[:, None, None], -math.inf)
    m = p.amax(-1, keepdim=True).clamp_min(-3e38)
    p.sub_(m).exp_()
    z = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hk, G * most, n), v).view(B, Hk, G, most, D) / z.clamp_min(1e-38)
    t = torch.arange(T, device=DEV)
    b = torch.searchsorted(starts[1:].contiguous(), t, right=True)
    i = t - starts[b]
    o, lse = o.view(B, Hq, most, D), (m + torch.log(z)).view(B, Hq, most)
    return o[b, :, i], lse[b, :, i]


def _prompt(s):
    k_starts = s["starts"] if s["k_starts"] is None else s["k_starts"]
    k, v = (_padded(s[n], k_starts, s["max_len"]) for n in ("k", "v"))
    o, lse = _attend(s["q"], k, v, s["starts"], k_starts.diff(), s["max_new"], s["causal"])
    return [o.bfloat16(), lse] if s["lse"] else [o.bfloat16()]


def _chunk(s):
    k, v = _gather(s["kc"], s["ks"], s["table"]), _gather(s["vc"], s["vs"], s["table"])
    return [_attend(s["q"], k, v, s["starts"], s["lens"], s["max_new"], s["causal"])[0].bfloat16()]


def run(s):
    op = s["op"]
    if not own:
        return {"rotate": _rotate, "act": _act, "prompt": _prompt, "chunk": _chunk}[op](s)
    from paper_2609_33601_amd import jq_block as jb

    if op == "act":
        return list(jb.jq_gated_act(s["gate"], s["up"], act=s["act"], out=s["out"]))
    if op == "rotate":
        q, k = jb.jq_qk_norm_rope_append(s["q"], s["k"], s["v"], s["qw"], s["kw"], s["pos"], s["cos"], s["sin"],
                                         s["slots"], s["kc"], s["vc"], k_scale=s["ks"], v_scale=s["vs"], eps=EPS,
                                         interleaved=s["interleaved"], dense_k=s["dense"])
        return [q, k, s["kc"], s["vc"], s["ks"], s["vs"]]
    if op == "prompt":
        lse = torch.empty(s["q"].shape[:2], dtype=torch.float32, device=DEV) if s["lse"] else None
        o = jb.jq_prompt_attention(s["q"], s["k"], s["v"], s["starts"], k_starts=s["k_starts"], causal=s["causal"],
                                   lse=lse)
        return [o, lse] if s["lse"] else [o]
    return [jb.jq_chunk_attention(s["q"], s["kc"], s["vc"], s["table"], s["starts"], s["lens"], k_scale=s["ks"],
                                  v_scale=s["vs"], max_len=s["max_len"], causal=s["causal"])]


# ---------------------------------------------------------------------------
# what a pass cannot do without, and its results from the definition in 64 bits


def work(case):
    op = case["op"]
    if op == "act":
        M, N = case["M"], case["N"]
        n = M * N
        out = 2 * n if case["out"] == "bf16" else n + 4 * M * _blocks(N)
        return {"bytes": (4 if case["gated"] else 2) * n + out, "flops": 8 * n}
    Hq, Hk, D = case["Hq"], case["Hk"], case["D"]
    if op == "rotate":
        T = case["T"]
        kv = {"none": 0, "bf16": 4 * D, "fp8": 2 * (D + 4)}[case["cache"]] * T * Hk
        read = Hq + (Hk if case["cache"] == "none" else 2 * Hk)
        return {"bytes": 2 * T * D * (read + Hq + (Hk if case["dense"] else 0)) + kv + 4 * T * case["R"] + 4 * D
                + (4 if case["cache"] == "none" else 12) * T,
                "flops": T * (Hq + Hk) * (5 * D + 3 * case["R"])}
    pairs = 0
    new, total = lengths(case)
    for a, n in zip(new, total):
        if case["causal"]:  # the last token sees n keys, each one before it one key less
            seen = min(a, n)
            pairs += seen * n - seen * (seen - 1) // 2
        else:
            pairs += a * n
    row = 2 * D if op == "prompt" or case["cache"] == "bf16" else D + 4
    lse = 4 * sum(new) * Hq if op == "prompt" and case["lse"] else 0
    return {"bytes": 2 * sum(total) * Hk * row + 4 * sum(new) * Hq * D + lse, "flops": 4 * pairs * Hq * D}


def _e_turned(x, w, s):
    """Norm and rotation, the rotation as a complex product."""
    x = x.double()
    n = torch.linalg.vector_norm(x, dim=-1, keepdim=True)
    x = x * w.double() / torch.sqrt(n * n / x.shape[-1] + EPS)
    R = s["R"]
    z = torch.complex(s["cos"].double(), s["sin"].double())[s["pos"].long()][:, None]
    even, odd = (slice(0, R, 2), slice(1, R, 2)) if s["interleaved"] else (slice(0, R // 2), slice(R // 2, R))
    t = torch.complex(x[..., even], x[..., odd]) * z
    x[..., even], x[..., odd] = t.real, t.imag
    return x


def _e_act(s):
    x = s["gate"].double()
    if s["act"] == "silu":
        y = x * torch.sigmoid(x)
    elif s["act"] == "gelu":
        y = x * torch.special.ndtr(x)
    else:
        y = x * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3))
    if s["up"] is not None:
        y = y * s["up"].double()
    if s["out"] == "bf16":
        return [y]
    a = torch.zeros((s["M"], _blocks(s["N"])), dtype=torch.float64, device=DEV)
    at = torch.arange(s["N"], device=DEV) // 128
    a.scatter_reduce_(1, at.expand(y.shape), y.abs(), "amax")
    f = a / E4M3_MAX
    return [y / f.clamp_min(1e-300)[:, at], f]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "act":
        return _e_act(s)
    Hq, Hk, D = case["Hq"], case["Hk"], case["D"]
    if op == "rotate":
        q, k, v = _e_turned(s["q"], s["qw"], s), _e_turned(s["k"], s["kw"], s), s["v"].double()
        caches, scales = [None, None], [None, None]
        for j, x in enumerate((k, v) if s["kc"] is not None else ()):
            pages, _, page, _ = s["kc"].shape
            c = torch.zeros((pages * page, Hk, D), dtype=torch.float64, device=DEV)
            f = x.abs().amax(-1) / E4M3_MAX
            c[s["slots"]] = x if s["ks"] is None else x / f.clamp_min(1e-300)[..., None]
            caches[j] = c.view(pages, page, Hk, D).transpose(1, 2).contiguous()
            if s["ks"] is not None:
                z = torch.zeros((pages * page, Hk), dtype=torch.float64, device=DEV)
                z[s["slots"]] = f
                scales[j] = z.view(pages, page, Hk).transpose(1, 2).contiguous()
        return [q, k if case["dense"] else None, *caches, *scales]
    new, total = lengths(case)
    out = torch.zeros((sum(new), Hq, D), dtype=torch.float64, device=DEV)
    lse = torch.zeros((sum(new), Hq), dtype=torch.float64, device=DEV)
    t0 = k0 = 0
    for b, (a, n) in enumerate(zip(new, total)):
        if op == "prompt":
            k, v = s["k"][k0 : k0 + n], s["v"][k0 : k0 + n]
        else:
            pages = s["table"][b].long()[: -(-n // case["page"])]
            k, v = (c.view(torch.uint8)[pages].view(c.dtype).transpose(1, 2).reshape(-1, Hk, D)[:n]
                    for c in (s["kc"], s["vc"]))
            fk, fv = (None if f is None else f[pages].transpose(1, 2).reshape(-1, Hk)[:n] for f in (s["ks"], s["vs"]))
        hidden = torch.ones((a, n), dtype=torch.bool, device=DEV).triu(n - a + 1) if case["causal"] else None
        for h in range(Hk):
            kh, vh = k[:, h].double(), v[:, h].double()
            if op == "chunk" and fk is not None:
                kh, vh = kh * fk[:, h, None].double(), vh * fv[:, h, None].double()
            for j in range(h * (Hq // Hk), (h + 1) * (Hq // Hk)):
                z = torch.mm(s["q"][t0 : t0 + a, j].double(), kh.t()) / math.sqrt(D)
                if hidden is not None:
                    z.masked_fill_(hidden, -math.inf)
                e = torch.logsumexp(z, 1)
                z = torch.exp(z - torch.where(e > -math.inf, e, 0.0)[:, None])
                out[t0 : t0 + a, j] = torch.mm(z, vh)
                lse[t0 : t0 + a, j] = e
        t0, k0 = t0 + a, k0 + n
    return [out, lse] if op == "prompt" and case["lse"] else [out]
