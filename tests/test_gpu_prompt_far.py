"""The prompts' operators where offsets pass 32 bits: far pages, far rows, far strides."""

import pytest
import torch

from paper_2609_33601_amd import jq_block as jb
from tests import block_reference as block
from tests import prompt_reference as ref

pytestmark = pytest.mark.gpu

DEV = "cuda"


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_far_pages(kind):
    """Append to, and attention over, pages whose elements lie past 2^32 bytes and 2^31 elements."""
    Hk, D, page, g = 8, 128, 64, gen(1)
    per = Hk * page * D
    pages = (2 ** 32 + 2 ** 30) // (per * (2 if kind == "bf16" else 1)) + 5
    dt = torch.bfloat16 if kind == "bf16" else torch.float8_e4m3fn
    kv = [torch.empty((pages, Hk, page, D), dtype=dt, device=DEV) for _ in range(2)]
    scales = [torch.empty((pages, Hk, page), device=DEV) if kind == "fp8" else None for _ in range(2)]
    n = 150
    table = i32(pages - 1, 0, pages - 3)[None]
    t = torch.arange(n, device=DEV)
    slots = table[0, t // page].long() * page + t % page
    q, k, v = (torch.randn((n, h, D), generator=g, device=DEV).bfloat16() for h in (32, Hk, Hk))
    one = torch.ones((D,), device=DEV).bfloat16()
    at = torch.outer(t.double(), 10000.0 ** (-torch.arange(0, D, 2, device=DEV).double() / D))
    q2, _ = jb.jq_qk_norm_rope_append(q, k, v, one, one, t.int(), at.cos().float(), at.sin().float(), slots, *kv, *scales)
    out = jb.jq_chunk_attention(q2, *kv, table, i32(0, n), i32(n), *scales)
    kk, vv = [block.cached(c, s, table[0], n).transpose(0, 1) for c, s in zip(kv, scales)]
    ref.check_attention(out, None, q2, kk, vv)
    assert float((vv - v.double()).norm() / v.double().norm()) < (2.0 ** -9 if kind == "bf16" else 0.04)


def test_far_rows():
    """Keys and values with the widest rows that are allowed, in one allocation past 2^32 bytes."""
    n, D, g = 70, 64, gen(2)
    room = torch.empty((n * 2 ** 25,), dtype=torch.bfloat16, device=DEV)
    k = room.as_strided((n, 2, D), (2 ** 25, D, 1))
    v = room.as_strided((n, 2, D), (2 ** 25, D, 1), 2 ** 24)
    for x in (k, v):
        x.copy_(torch.randn((n, 2, D), generator=g, device=DEV))
    q = torch.randn((n, 4, D), generator=g, device=DEV).bfloat16()
    for causal in (True, False):
        out = jb.jq_prompt_attention(q, k, v, i32(0, 40, n), causal=causal)
        for a, b in ((0, 40), (40, n)):
            ref.check_attention(out[a:b], None, q[a:b], k[a:b], v[a:b], causal)


def test_far_elements():
    """An activation of more than 2^32 bytes in and 2^31 codes out; and heads beyond 2^31 elements."""
    M, N, g = 140000, 16384, gen(3)
    gate = torch.zeros((M, N), dtype=torch.bfloat16, device=DEV)
    gate[-3:] = torch.randn((3, N), generator=g, device=DEV).bfloat16() * 3
    q, s = jb.jq_gated_act(gate, None, act="gelu_tanh", out="fp8")
    block.check_fp8(q[-3:], s[-3:], ref.activation(gate[-3:], None, "gelu_tanh"))
    assert not q[:2].float().any() and not s[:2].any()
    del q, s
    T = M * N // (8 * 128)
    k = gate.view(T, 8, 128)
    w = torch.ones((128,), device=DEV).bfloat16()
    _, y = jb.jq_qk_norm_rope_append(None, k, None, None, w, torch.zeros((T,), dtype=torch.int32, device=DEV), None, None)
    want, e = ref.head_norm(k[-48:], w, 1e-6)
    assert torch.all((y[-48:].double() - want).abs() <= ref.BF16 * want.abs() + 1.02 * e)
    assert not y[:2].any()
