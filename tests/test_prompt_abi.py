"""Checks without a GPU of the operators that take whole prompts through a block: bad arguments are rejected before
anything is launched (fake addresses are never dereferenced: every call below fails validation), workspaces have the
size that their layout asks for, and the binding refuses what it can see."""

import os

import pytest

from paper_2609_33601_amd import jq, jq_block as jb

pytestmark = pytest.mark.skipif(not os.path.exists(jq.LIB_PATH),
                                reason="libjq.so not built (run __graft_entry__.build())")

A = 0x10000  # a fake, 256-byte-aligned address
ARG, SHAPE, ALIGN, SMALL = (jq.JQ_ERR_INVALID_ARG, jq.JQ_ERR_UNSUPPORTED_SHAPE, jq.JQ_ERR_MISALIGNED,
                            jq.JQ_ERR_WORKSPACE_TOO_SMALL)


def _call(name, ok, **kw):
    unknown = set(kw) - set(ok)
    assert not unknown, unknown
    return getattr(jb.lib(), name)(*{**ok, **kw}.values())


APPEND = dict(q=A, qs=512, k=A, ks=128, v=A, vs=128, T=4, Hq=8, Hk=2, D=64, qw=A, kw=A, eps=1e-6, pos=A, cos=A, sin=A,
              P=100, R=64, inter=0, slots=A, qo=A, qos=512, ko=None, kos=0, kc=A, vc=A, ksc=None, vsc=None, pages=4,
              page=16, type=0, stream=None)
NO_CACHE = dict(v=None, slots=None, kc=None, vc=None, ko=A, kos=128)


@pytest.mark.parametrize("want,kw", [
    (ARG, dict(k=None)), (ARG, dict(v=None)), (ARG, dict(pos=None)), (ARG, dict(slots=None)), (ARG, dict(q=None)),
    (ARG, dict(qo=None)), (ARG, dict(qw=None)), (ARG, dict(kw=None)), (ARG, dict(Hq=0)), (ARG, dict(Hq=-1)),
    (ARG, dict(Hk=0)), (ARG, dict(T=0)), (ARG, dict(D=0)), (ARG, dict(cos=None)), (ARG, dict(sin=None)), (ARG, dict(P=0)),
    (ARG, dict(R=-16)), (ARG, dict(vc=None)), (ARG, dict(kc=None)), (ARG, dict(pages=0)), (ARG, dict(type=2)),
    (ARG, dict(type=1)), (ARG, dict(ksc=A)), (ARG, dict(eps=-1.0)), (ARG, dict(eps=float("nan"))), (ARG, dict(qs=504)),
    (ARG, dict(ks=120)), (ARG, dict(vs=64)), (ARG, dict(qos=8)), (ARG, dict(ko=A, kos=64)),
    (ARG, {**NO_CACHE, "ko": None}), (ARG, {**NO_CACHE, "v": A}), (ARG, {**NO_CACHE, "slots": A}),
    (ARG, {**NO_CACHE, "vc": A}), (ARG, {**NO_CACHE, "ksc": A}), (ARG, {**NO_CACHE, "vsc": A}),
    (ARG, {**NO_CACHE, "Hk": 0}), (ARG, {**NO_CACHE, "kos": 120}),
    (SHAPE, dict(D=40)), (SHAPE, dict(D=272, qs=4096, ks=1024, vs=1024, qos=4096)), (SHAPE, dict(R=24)), (SHAPE, dict(R=80)),
    (SHAPE, dict(page=8)), (SHAPE, dict(page=48)), (SHAPE, dict(pages=1 << 31)), (SHAPE, dict(T=1 << 28)),
    (SHAPE, dict(T=1 << 31)), (SHAPE, {**NO_CACHE, "Hk": 1 << 17, "ks": 1 << 24, "kos": 1 << 24}),
    (ALIGN, dict(q=A + 8)), (ALIGN, dict(k=A + 8)), (ALIGN, dict(v=A + 2)), (ALIGN, dict(qo=A + 8)), (ALIGN, dict(qw=A + 8)),
    (ALIGN, dict(kw=A + 2)), (ALIGN, dict(ko=A + 8, kos=128)), (ALIGN, dict(cos=A + 4)), (ALIGN, dict(pos=A + 2)),
    (ALIGN, dict(slots=A + 4)), (ALIGN, dict(kc=A + 8)), (ALIGN, dict(ks=132)), (ALIGN, {**NO_CACHE, "kos": 132}),
    (ALIGN, dict(type=1, ksc=A + 4, vsc=A))], ids=str)
def test_norm_rotate_append_refuses(want, kw):
    assert _call("jq_qk_norm_rope_append", APPEND, **kw) == want


ACT = dict(gate=A, gs=128, up=A, us=128, M=4, N=128, act=0, out=0, y=A, s=None, stream=None)


@pytest.mark.parametrize("want,kw", [
    (ARG, dict(gate=None)), (ARG, dict(y=None)), (ARG, dict(M=0)), (ARG, dict(N=0)), (ARG, dict(N=-8)), (ARG, dict(act=3)),
    (ARG, dict(act=-1)), (ARG, dict(out=3)), (ARG, dict(out=1)), (ARG, dict(out=2)), (ARG, dict(s=A)), (ARG, dict(gs=120)),
    (ARG, dict(us=64)), (ARG, dict(gs=1 << 33)), (SHAPE, dict(N=60)), (SHAPE, dict(N=65544, gs=1 << 17, us=1 << 17)),
    (SHAPE, dict(N=72, out=2, s=A)), (SHAPE, dict(M=(1 << 30) + 1)), (SHAPE, dict(M=1 << 30, N=1024, gs=1024, us=1024)),
    (ALIGN, dict(gs=132)), (ALIGN, dict(us=130)), (ALIGN, dict(gate=A + 8)), (ALIGN, dict(up=A + 2)), (ALIGN, dict(y=A + 8)),
    (ALIGN, dict(out=1, s=A + 2))], ids=str)
def test_gated_act_refuses(want, kw):
    assert _call("jq_gated_act", ACT, **kw) == want


PROMPT = dict(q=A, qs=512, k=A, ks=128, v=A, vs=128, starts=A, kstarts=None, T=100, Tk=100, B=2, Hq=8, Hk=2, D=64,
              scale=0.125, causal=1, out=A, lse=None, ws=None, n=0, stream=None)
LONG = dict(kstarts=A, Tk=5000)  # cut into parts: needs a workspace


@pytest.mark.parametrize("want,kw", [
    (ARG, dict(q=None)), (ARG, dict(k=None)), (ARG, dict(v=None)), (ARG, dict(starts=None)), (ARG, dict(out=None)),
    (ARG, dict(T=0)), (ARG, dict(Tk=0)), (ARG, dict(B=0)), (ARG, dict(Hq=0)), (ARG, dict(Hk=-2)), (ARG, dict(qs=504)),
    (ARG, dict(ks=120)), (ARG, dict(vs=64)), (ARG, dict(ks=(1 << 25) + 8)), (ARG, dict(vs=1 << 26)), (ARG, LONG),
    (SHAPE, dict(D=32)), (SHAPE, dict(D=96)), (SHAPE, dict(Hq=9, qs=576)), (SHAPE, dict(B=(1 << 20) + 1)),
    (SHAPE, dict(T=1 << 28)), (SHAPE, dict(T=(1 << 30) + 1)), (SHAPE, dict(Tk=(1 << 30) + 1)),
    (SHAPE, dict(B=1 << 20, T=1 << 20, Hq=16, Hk=16, qs=1024, ks=1024, vs=1024)), (ALIGN, dict(qs=516)), (ALIGN, dict(ks=132)),
    (ALIGN, dict(q=A + 8)), (ALIGN, dict(k=A + 8)), (ALIGN, dict(v=A + 2)), (ALIGN, dict(out=A + 8)),
    (ALIGN, dict(starts=A + 2)), (ALIGN, dict(kstarts=A + 2)), (ALIGN, dict(lse=A + 1)),
    (ALIGN, {**LONG, "ws": A + 16, "n": 1 << 30}), (SMALL, {**LONG, "ws": A, "n": 256})], ids=str)
def test_prompt_attention_refuses(want, kw):
    assert _call("jq_prompt_attention", PROMPT, **kw) == want


CHUNK = dict(q=A, qs=512, kc=A, vc=A, ksc=None, vsc=None, table=A, cols=8, starts=A, lens=A, T=100, B=2, Hq=8, Hk=2, D=64,
             pages=100, page=16, max_len=128, scale=0.125, causal=1, type=0, out=A, lse=None, ws=None, n=0, stream=None)


@pytest.mark.parametrize("want,kw", [
    (ARG, dict(q=None)), (ARG, dict(kc=None)), (ARG, dict(vc=None)), (ARG, dict(table=None)), (ARG, dict(starts=None)),
    (ARG, dict(lens=None)), (ARG, dict(out=None)), (ARG, dict(cols=0)), (ARG, dict(T=0)), (ARG, dict(B=0)),
    (ARG, dict(max_len=0)), (ARG, dict(max_len=129)), (ARG, dict(pages=0)), (ARG, dict(type=3)), (ARG, dict(type=1)),
    (ARG, dict(ksc=A)), (ARG, dict(type=1, vsc=A)), (ARG, dict(qs=8)), (ARG, dict(max_len=5000, cols=400)),
    (SHAPE, dict(D=80)), (SHAPE, dict(Hq=7)), (SHAPE, dict(page=24)), (SHAPE, dict(page=1 << 17)),
    (SHAPE, dict(cols=1 << 31, max_len=128)), (SHAPE, dict(T=1 << 28)), (ALIGN, dict(kc=A + 8)), (ALIGN, dict(q=A + 2)),
    (ALIGN, dict(table=A + 2)), (ALIGN, dict(lens=A + 1)), (ALIGN, dict(type=1, ksc=A, vsc=A + 8)),
    (SMALL, dict(max_len=5000, cols=400, ws=A, n=1024))], ids=str)
def test_chunk_attention_refuses(want, kw):
    assert _call("jq_chunk_attention", CHUNK, **kw) == want


def test_workspaces():
    """Nothing for one part or invalid sizes; else 4 (D + 2) bytes for each query row and part, rounded up to 256."""
    for f, args in ((jb.jq_prompt_attention_workspace_bytes, (100, 100, 2, 8, 2, 64)),
                    (jb.jq_chunk_attention_workspace_bytes, (100, 2, 8, 2, 64, 128))):
        assert f(*args) == 0 and f(*args[:-2], 2, 63) == 0 and f(-1, *args[1:]) == 0
    for T, B, Hq, Hk, D, n in ((16, 1, 32, 8, 128, 2080), (1, 1, 8, 1, 64, 100000), (100, 3, 12, 2, 256, 9000)):
        got = jb.jq_chunk_attention_workspace_bytes(T, B, Hq, Hk, D, n)
        row = 4 * (D + 2) * T * Hq
        for got in (got, jb.jq_prompt_attention_workspace_bytes(T, n, B, Hq, Hk, D)):
            assert got % 256 == 0 and any(0 <= got - parts * row < 256 for parts in range(2, 1025))


def test_binding_refuses_names_and_tensors():
    torch = pytest.importorskip("torch")
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="act must be one of"):
        jb.jq_gated_act(x, x, act="relu")
    with pytest.raises(ValueError, match="out must be one of"):
        jb.jq_gated_act(x, x, out="fp4")
    if not os.path.exists(jb.NATIVE_PATH):
        pytest.skip("_jq_block.so not built")
    with pytest.raises(ValueError, match="must be on the GPU"):
        jb.jq_gated_act(x, x)
    with pytest.raises(TypeError, match="must be a torch.Tensor"):
        jb.jq_gated_act(None)
    q = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="must be on the GPU"):
        jb.jq_prompt_attention(q, q, q, None)
    with pytest.raises(TypeError, match="k_cache must be"):
        jb.jq_chunk_attention(q, q.float(), q, None, None, None)
    with pytest.raises(ValueError, match="must be on the GPU"):
        jb.jq_qk_norm_rope_append(q, q, q, None, None, None, None, None)
