"""What the binding of the prompts' operators refuses, and that a refused call writes nothing."""

import pytest
import torch

from paper_2609_33601_amd import jq, jq_block as jb

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF = torch.bfloat16
E4M3 = torch.float8_e4m3fn


def z(*shape, dtype=BF):
    return torch.zeros(shape, dtype=dtype, device=DEV)


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def refused(error, call, out=None, match=None):
    if out is not None:
        out.fill_(7.0)
    with pytest.raises(error, match=match):
        call()
    torch.cuda.synchronize()
    assert out is None or bool((out == 7.0).all())


@pytest.mark.parametrize("error,match,kw", [
    (TypeError, "q must be", lambda: dict(q=z(8, 4, 64, dtype=torch.float16))), (ValueError, "q must be", lambda: dict(q=z(8, 256))),
    (ValueError, "on the GPU", lambda: dict(q=torch.zeros((8, 4, 64), dtype=BF))), (ValueError, "k must be", lambda: dict(k=z(8, 2, 128))),
    (ValueError, "v must have shape", lambda: dict(v=z(8, 4, 64))), (ValueError, "must be contiguous", lambda: dict(q=z(8, 64, 4).transpose(1, 2))),
    (ValueError, "without k_starts", lambda: dict(k=z(9, 2, 64), v=z(9, 2, 64))), (TypeError, "starts must be", lambda: dict(starts=i32(0, 8).long())),
    (ValueError, "starts must be", lambda: dict(starts=i32(0))), (ValueError, "starts must be", lambda: dict(starts=i32(0, 8)[None])),
    (ValueError, "k_starts must have", lambda: dict(k_starts=i32(0, 4, 8))), (ValueError, "out must have", lambda: dict(out=z(8, 64, 4))),
    (TypeError, "lse must be", lambda: dict(lse=z(8, 4))), (TypeError, "workspace must be", lambda: dict(workspace=z(64))),
    (jq.JQError, None, lambda: dict(q=z(8, 3, 64))), (jq.JQError, None, lambda: dict(q=z(8, 4, 32), k=z(8, 2, 32), v=z(8, 2, 32))),
    (jq.JQError, None, lambda: dict(q=z(8, 4 * 64 + 4)[:, :256].view(8, 4, 64)))], ids=lambda v: "x")
def test_prompt_attention(error, match, kw):
    kw = kw()
    args = {**dict(q=z(8, 4, 64), k=z(8, 2, 64), v=z(8, 2, 64), starts=i32(0, 8)), **kw}
    out = None if "out" in kw or args["q"].shape != (8, 4, 64) else z(8, 4, 64)
    refused(error, lambda: jb.jq_prompt_attention(**{"out": out, **args}), out, match)


@pytest.mark.parametrize("error,match,kw", [
    (TypeError, "k_cache must be", lambda: dict(k_cache=z(5, 2, 16, 64, dtype=torch.float32))),
    (ValueError, "no scales", lambda: dict(k_scale=z(5, 2, 16, dtype=torch.float32))),
    (ValueError, "needs k_scale", lambda: dict(k_cache=z(5, 2, 16, 64).to(E4M3), v_cache=z(5, 2, 16, 64).to(E4M3))),
    (ValueError, "v_cache must have", lambda: dict(v_cache=z(4, 2, 16, 64))), (ValueError, "heads of", lambda: dict(q=z(8, 4, 128))),
    (ValueError, "page_table must be", lambda: dict(page_table=i32(0, 1))), (ValueError, "page_table must be", lambda: dict(page_table=z(2, 4, dtype=torch.int32))),
    (ValueError, "lens must have", lambda: dict(lens=i32(8, 8))), (TypeError, "lens must be", lambda: dict(lens=i32(8).float())),
    (jq.JQError, None, lambda: dict(max_len=49)), (jq.JQError, None, lambda: dict(max_len=0)), (jq.JQError, None, lambda: dict(q=z(8, 3, 64))),
    (jq.JQError, None, lambda: dict(k_cache=z(5, 2, 24, 64), v_cache=z(5, 2, 24, 64)))], ids=lambda v: "x")
def test_chunk_attention(error, match, kw):
    kw = kw()
    args = {**dict(q=z(8, 4, 64), k_cache=z(5, 2, 16, 64), v_cache=z(5, 2, 16, 64), page_table=i32(0, 1, 2)[None],
                   starts=i32(0, 8), lens=i32(40)), **kw}
    out = None if args["q"].shape != (8, 4, 64) else z(8, 4, 64)
    refused(error, lambda: jb.jq_chunk_attention(**{"out": out, **args}), out, match)


@pytest.mark.parametrize("error,match,kw", [
    (ValueError, "k must be", lambda: dict(k=z(8, 128))), (ValueError, "q must have", lambda: dict(q=z(7, 4, 64))),
    (ValueError, "q_weight must have", lambda: dict(q_weight=z(32))), (TypeError, "k_weight must be", lambda: dict(k_weight=z(64, dtype=torch.float32))),
    (TypeError, "positions must be", lambda: dict(positions=torch.zeros((8,), dtype=torch.int64, device=DEV))),
    (ValueError, "sin without cos", lambda: dict(cos=None)), (ValueError, "sin must have", lambda: dict(sin=z(20, 16, dtype=torch.float32))),
    (ValueError, "without a k_cache", lambda: dict(slots=torch.zeros((8,), dtype=torch.int64, device=DEV))),
    (ValueError, "without a k_cache", lambda: dict(k_scale=z(1, dtype=torch.float32))),
    (ValueError, "the cache", lambda: dict(k_cache=z(5, 4, 16, 64), v_cache=z(5, 4, 16, 64))),
    (ValueError, "slots must have", lambda: dict(k_cache=z(5, 2, 16, 64), v_cache=z(5, 2, 16, 64), slots=torch.zeros((7,), dtype=torch.int64, device=DEV))),
    (ValueError, "q_out without q", lambda: dict(q=None, q_weight=None, q_out=z(8, 4, 64))), (jq.JQError, None, lambda: dict(eps=-1.0)),
    (ValueError, "k_out must have", lambda: dict(k_out=z(8, 2, 32))),
    (jq.JQError, None, lambda: dict(cos=z(20, 20, dtype=torch.float32), sin=z(20, 20, dtype=torch.float32)))], ids=lambda v: "x")
def test_norm_rope_append(error, match, kw):
    kw = kw()
    t = torch.zeros((20, 32), dtype=torch.float32, device=DEV)
    args = {**dict(q=z(8, 4, 64), k=z(8, 2, 64), v=z(8, 2, 64), q_weight=z(64), k_weight=z(64), positions=i32(*range(8)),
                   cos=t, sin=t), **kw}
    out = z(8, 2, 64)
    refused(error, lambda: jb.jq_qk_norm_rope_append(**{"k_out": out, **args}), out, match)


@pytest.mark.parametrize("error,match,kw", [
    (TypeError, "gate must be", lambda: dict(gate=z(4, 64, dtype=torch.float32))), (ValueError, "a matrix", lambda: dict(gate=z(4, 8, 8))),
    (ValueError, "up must have", lambda: dict(up=z(4, 32))), (ValueError, "has no scale", lambda: dict(scale=z(4, 1, dtype=torch.float32))),
    (ValueError, "contiguous", lambda: dict(gate=z(64, 4).t())), (jq.JQError, None, lambda: dict(gate=z(4, 60), up=z(4, 60), y=None)),
    (jq.JQError, None, lambda: dict(gate=z(4, 72), up=z(4, 72), y=None, out="int4")),
    (jq.JQError, None, lambda: dict(gate=z(0, 64), up=z(0, 64), y=None)),
    (TypeError, "y must be", lambda: dict(out="fp8")), (ValueError, "out must be", lambda: dict(out="int8"))], ids=lambda v: "x")
def test_gated_act(error, match, kw):
    out = z(4, 64)
    refused(error, lambda: jb.jq_gated_act(**{**dict(gate=z(4, 64), up=z(4, 64), y=out), **kw()}), out, match)
