"""C-ABI checks of the decoder block's other operators that need no GPU: the library exports every symbol that
include/jq_block.h declares, and rejects bad arguments before launching anything (fake addresses are never
dereferenced: every call below fails validation)."""

import ctypes
import os
import re

import pytest

from paper_2609_33601_amd import jq, jq_block as jb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "jq_block.h")

pytestmark = pytest.mark.skipif(not os.path.exists(jq.LIB_PATH),
                                reason="libjq.so not built (run __graft_entry__.build())")

A = 0x10000  # a fake, 256-byte-aligned address
ARG, SHAPE, ALIGN, SMALL = (jq.JQ_ERR_INVALID_ARG, jq.JQ_ERR_UNSUPPORTED_SHAPE, jq.JQ_ERR_MISALIGNED,
                            jq.JQ_ERR_WORKSPACE_TOO_SMALL)


def _call(name, ok, **kw):
    unknown = set(kw) - set(ok)
    assert not unknown, unknown
    return getattr(jb.lib(), name)(*{**ok, **kw}.values())


def test_exports_every_declared_symbol():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(jq_[a-z0-9_]+)\s*\(", text))
    assert names == set(jb.SIGNATURES), names ^ set(jb.SIGNATURES)
    lib = ctypes.CDLL(jq.LIB_PATH)
    for n in names:
        assert hasattr(lib, n), n


NORM = dict(x=A, xs=64, r=None, rs=0, w=A, M=4, D=64, eps=1e-6, out=0, y=A, s=None, ro=None, ros=0, stream=None)


@pytest.mark.parametrize("want,kw", [
    (ARG, dict(x=None)), (ARG, dict(w=None)), (ARG, dict(y=None)), (ARG, dict(M=0)), (ARG, dict(M=-1)), (ARG, dict(D=0)),
    (ARG, dict(out=3)), (ARG, dict(out=-1)), (ARG, dict(r=A, rs=64)), (ARG, dict(ro=A, ros=64)), (ARG, dict(out=1)),
    (ARG, dict(s=A)), (ARG, dict(eps=-1.0)), (ARG, dict(eps=float("nan"))), (ARG, dict(xs=56)), (ARG, dict(xs=1 << 33)),
    (ARG, dict(r=A, rs=8, ro=A, ros=64)), (ARG, dict(r=A, rs=64, ro=A, ros=8)),
    (SHAPE, dict(D=60, xs=64)), (SHAPE, dict(D=65536 + 8, xs=65536 + 8)), (SHAPE, dict(M=(1 << 30) + 1)),
    (SHAPE, dict(D=72, xs=72, out=2, s=A)), (ALIGN, dict(xs=68)), (ALIGN, dict(x=A + 8)), (ALIGN, dict(w=A + 2)),
    (ALIGN, dict(y=A + 8)), (ALIGN, dict(out=1, s=A + 2)), (ALIGN, dict(r=A + 2, rs=64, ro=A, ros=64)),
    (ALIGN, dict(r=A, rs=64, ro=A + 4, ros=64)), (ALIGN, dict(r=A, rs=68, ro=A, ros=64))], ids=str)
def test_norm_refuses(want, kw):
    assert _call("jq_rmsnorm", NORM, **kw) == want


QUANT = dict(x=A, xs=64, M=4, K=64, q=A, s=A, stream=None)


@pytest.mark.parametrize("want,kw", [
    (ARG, dict(x=None)), (ARG, dict(q=None)), (ARG, dict(s=None)), (ARG, dict(M=0)), (ARG, dict(K=-16)),
    (ARG, dict(xs=48)), (SHAPE, dict(K=24, xs=24)), (SHAPE, dict(K=65552, xs=65552)), (SHAPE, dict(M=1 << 31)),
    (SHAPE, dict(M=1 << 30, K=1024, xs=1024)), (ALIGN, dict(xs=66)), (ALIGN, dict(x=A + 8)), (ALIGN, dict(q=A + 8)),
    (ALIGN, dict(s=A + 2))], ids=str)
def test_quantize_fp8_refuses(want, kw):
    assert _call("jq_quantize_act_fp8", QUANT, **kw) == want


PACK = dict(w=A, N=4, K=64, q=A, s=A, stream=None)


@pytest.mark.parametrize("want,kw", [
    (ARG, dict(w=None)), (ARG, dict(q=None)), (ARG, dict(s=None)), (ARG, dict(N=0)), (SHAPE, dict(K=8)),
    (SHAPE, dict(K=40)), (SHAPE, dict(N=1 << 30, K=1024)), (ALIGN, dict(w=A + 8)), (ALIGN, dict(q=A + 4)),
    (ALIGN, dict(s=A + 1))], ids=str)
def test_pack_fp8_refuses(want, kw):
    assert _call("jq_pack_weight_fp8", PACK, **kw) == want


GEMM = dict(q=A, s=A, M=4, K=64, wq=A, ws=A, N=32, b=None, y=A, stream=None)


@pytest.mark.parametrize("want,kw", [
    (ARG, dict(q=None)), (ARG, dict(s=None)), (ARG, dict(wq=None)), (ARG, dict(ws=None)), (ARG, dict(y=None)),
    (ARG, dict(M=0)), (ARG, dict(N=-4)), (ARG, dict(K=0)), (SHAPE, dict(K=8)), (SHAPE, dict(K=72)),
    (SHAPE, dict(K=65536 + 16)), (SHAPE, dict(M=1 << 31)), (SHAPE, dict(N=(1 << 22) + 1)),
    (SHAPE, dict(M=1 << 20, N=1 << 18)), (ALIGN, dict(q=A + 8)), (ALIGN, dict(wq=A + 4)), (ALIGN, dict(y=A + 2)),
    (ALIGN, dict(s=A + 2)), (ALIGN, dict(ws=A + 2)), (ALIGN, dict(b=A + 1))], ids=str)
def test_fp8_gemm_refuses(want, kw):
    assert _call("jq_fp8_gemm", GEMM, **kw) == want


def test_fp8_linear_refuses():
    need = jb.jq_fp8_workspace_bytes(4, 64)
    assert need == 256 + 256 and jb.jq_fp8_workspace_bytes(300, 1040) == 300 * 1040 + 192 + 300 * 9 * 4 + 80
    assert jb.jq_fp8_workspace_bytes(0, 64) == 0 and jb.jq_fp8_workspace_bytes(4, 65) == 0
    ok = dict(x=A, xs=64, M=4, K=64, wq=A, ws=A, N=32, b=None, y=A, wsp=A, n=need, stream=None)
    for want, kw in [(ARG, dict(x=None)), (ARG, dict(wq=None)), (ARG, dict(ws=None)), (ARG, dict(y=None)),
                     (ARG, dict(wsp=None)), (ARG, dict(M=0)), (ARG, dict(xs=32)), (SHAPE, dict(K=24)),
                     (ALIGN, dict(wsp=A + 16)), (ALIGN, dict(x=A + 8)), (ALIGN, dict(b=A + 1)), (SMALL, dict(n=need - 1)),
                     (SMALL, dict(n=0))]:
        assert _call("jq_fp8_linear", ok, **kw) == want, kw


APPEND = dict(q=A, qs=512, k=A, ks=128, v=A, vs=128, T=4, Hq=8, Hk=2, D=64, pos=A, cos=A, sin=A, P=100, R=64, inter=0,
              slots=A, qo=A, qos=512, kc=A, vc=A, ksc=None, vsc=None, pages=4, page=16, type=0, stream=None)


@pytest.mark.parametrize("want,kw", [
    (ARG, dict(k=None)), (ARG, dict(v=None)), (ARG, dict(pos=None)), (ARG, dict(slots=None)), (ARG, dict(q=None)),
    (ARG, dict(qo=None)), (ARG, dict(Hq=0)), (ARG, dict(Hq=-1)), (ARG, dict(Hk=0)), (ARG, dict(T=0)), (ARG, dict(D=0)),
    (ARG, dict(cos=None)), (ARG, dict(sin=None)), (ARG, dict(P=0)), (ARG, dict(R=-16)), (ARG, dict(kc=None)),
    (ARG, dict(vc=None)), (ARG, dict(pages=0)), (ARG, dict(type=2)), (ARG, dict(type=1)), (ARG, dict(ksc=A)),
    (ARG, dict(type=1, ksc=A)), (ARG, dict(qs=504)), (ARG, dict(ks=120)), (ARG, dict(vs=64)), (ARG, dict(qos=8)),
    (SHAPE, dict(D=40)), (SHAPE, dict(D=272, qs=4096, ks=1024, vs=1024, qos=4096)), (SHAPE, dict(R=24)), (SHAPE, dict(R=80)),
    (SHAPE, dict(page=8)), (SHAPE, dict(page=48)), (SHAPE, dict(page=1 << 17)), (SHAPE, dict(pages=1 << 31)),
    (SHAPE, dict(T=1 << 28)), (SHAPE, dict(T=1 << 31)), (ALIGN, dict(q=A + 8)), (ALIGN, dict(k=A + 8)),
    (ALIGN, dict(v=A + 2)), (ALIGN, dict(qo=A + 8)), (ALIGN, dict(cos=A + 4)), (ALIGN, dict(sin=A + 8)),
    (ALIGN, dict(pos=A + 2)), (ALIGN, dict(slots=A + 4)), (ALIGN, dict(kc=A + 8)), (ALIGN, dict(ks=132)),
    (ALIGN, dict(type=1, ksc=A + 4, vsc=A))], ids=str)
def test_rope_append_refuses(want, kw):
    assert _call("jq_rope_append", APPEND, **kw) == want


ATTEND = dict(q=A, kc=A, vc=A, ksc=None, vsc=None, table=A, cols=8, lens=A, B=2, Tq=1, Hq=8, Hk=2, D=64, pages=20, page=16,
              max_len=128, scale=0.125, causal=1, type=0, out=A, lse=None, ws=None, n=0, stream=None)


@pytest.mark.parametrize("want,kw", [
    (ARG, dict(q=None)), (ARG, dict(kc=None)), (ARG, dict(vc=None)), (ARG, dict(table=None)), (ARG, dict(lens=None)),
    (ARG, dict(out=None)), (ARG, dict(cols=0)), (ARG, dict(B=0)), (ARG, dict(Tq=0)), (ARG, dict(Hq=0)), (ARG, dict(Hk=0)),
    (ARG, dict(max_len=0)), (ARG, dict(max_len=129)), (ARG, dict(pages=0)), (ARG, dict(type=5)), (ARG, dict(type=1)),
    (ARG, dict(ksc=A, vsc=A)), (SHAPE, dict(Hq=7)), (SHAPE, dict(D=96)), (SHAPE, dict(D=32)), (SHAPE, dict(page=8)),
    (SHAPE, dict(page=20)), (SHAPE, dict(B=1 << 21)), (SHAPE, dict(B=1 << 20, Tq=4)), (SHAPE, dict(Tq=1 << 21)),
    (SHAPE, dict(Hq=1 << 17)), (SHAPE, dict(max_len=1 << 31)), (ALIGN, dict(q=A + 8)), (ALIGN, dict(out=A + 8)),
    (ALIGN, dict(table=A + 2)), (ALIGN, dict(lens=A + 2)), (ALIGN, dict(lse=A + 2)), (ALIGN, dict(kc=A + 8)),
    (ALIGN, dict(type=1, ksc=A, vsc=A + 8))], ids=str)
def test_attention_refuses(want, kw):
    assert _call("jq_paged_attention", ATTEND, **kw) == want


def test_attention_workspace():
    assert jb.jq_paged_attention_workspace_bytes(2, 1, 8, 2, 64, 16) == 0
    assert jb.jq_paged_attention_workspace_bytes(2, 1, 8, 3, 64, 4096) == 0
    assert jb.jq_paged_attention_workspace_bytes(0, 1, 8, 2, 64, 4096) == 0
    need = jb.jq_paged_attention_workspace_bytes(2, 1, 8, 2, 64, 65536)
    assert need > 0 and need % 256 == 0
    long = dict(cols=4096, max_len=65536)
    assert _call("jq_paged_attention", ATTEND, **long) == ARG
    assert _call("jq_paged_attention", ATTEND, ws=A, n=need - 1, **long) == SMALL
    assert _call("jq_paged_attention", ATTEND, ws=A + 64, n=need, **long) == ALIGN


def test_gemm_routes():
    """The GPU tests' products run on every kernel, and every size has one."""
    from tests.routes import fp8_route
    from tests.test_gpu_block import GEMM_SHAPES

    assert {fp8_route(*s) for s in GEMM_SHAPES} == set(range(10))
    # many small blocks would not fit a grid: the tiled kernels take those
    for M, K, N in ((1 << 30, 16, 1), (1 << 25, 16, 1 << 12), (1 << 16, 65536, 1 << 22)):
        assert fp8_route(M, K, N) in (8, 9)
    assert fp8_route(1, 65536, 1 << 22) in range(10)


def test_binding_refuses():
    torch = pytest.importorskip("torch")
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="on the GPU"):
        jb.jq_rmsnorm(x, x[0])
    with pytest.raises(ValueError, match="out must be"):
        jb.jq_rmsnorm(x, x[0], out="int8")
    with pytest.raises(ValueError, match="without a residual"):
        jb.jq_rmsnorm(x, x[0], residual_out=x)
    with pytest.raises(ValueError, match="on the GPU"):
        jb.jq_quantize_act_fp8(x)
    cache = torch.zeros((2, 1, 16, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="has no scales"):
        jb.jq_paged_attention(x.view(4, 1, 1, 64), cache, cache, None, None, k_scale=cache)
    with pytest.raises(ValueError, match="needs k_scale"):
        jb.jq_paged_attention(x.view(4, 1, 1, 64), cache.to(torch.float8_e4m3fn), cache, None, None)
