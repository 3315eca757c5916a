"""Python binding of the decoder block's other operators (include/jq_block.h).

What a served block runs around its W4A4 linears (jq.py): the RMS norm that
feeds a quantised linear, the 8-bit linear, the rotation of new queries and
keys with their append to a paged cache, and attention over that cache.  As in
jq.py, a call only turns GPU torch tensors into pointers and the current HIP
stream (of the device that its tensors are on) and raises on a non-OK status;
there is no other path.  The checks themselves are compiled (_jq_block.so,
csrc/jq_block_py.cpp): TypeError for a wrong type, ValueError for a wrong shape
or place, JQError for what the library refuses.  A call given a stream runs as
under torch.cuda.stream(stream): what it allocates belongs to that stream.

    cache    k_cache, v_cache  [pages, Hk, page_size, D]  bf16, or float8_e4m3fn with
             k_scale, v_scale  [pages, Hk, page_size]     fp32 for each token and head
"""

import ctypes
import importlib.util
import os

from . import jq
from .jq import JQError

_vp, _i64, _sz, _int, _f = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t, ctypes.c_int, ctypes.c_float

# Symbols of include/jq_block.h, with (restype, argtypes).
SIGNATURES = {
    "jq_rmsnorm": (_int, [_vp, _i64, _vp, _i64, _vp, _i64, _i64, _f, _int, _vp, _vp, _vp, _i64, _vp]),
    "jq_quantize_act_fp8": (_int, [_vp, _i64, _i64, _i64, _vp, _vp, _vp]),
    "jq_pack_weight_fp8": (_int, [_vp, _i64, _i64, _vp, _vp, _vp]),
    "jq_fp8_workspace_bytes": (_sz, [_i64, _i64]),
    "jq_fp8_gemm": (_int, [_vp, _vp, _i64, _i64, _vp, _vp, _i64, _vp, _vp, _vp]),
    "jq_fp8_linear": (_int, [_vp, _i64, _i64, _i64, _vp, _vp, _i64, _vp, _vp, _vp, _sz, _vp]),
    "jq_rope_append": (_int, [_vp, _i64, _vp, _i64, _vp, _i64, _i64, _i64, _i64, _i64, _vp, _vp, _vp, _i64, _i64, _int,
                              _vp, _vp, _i64, _vp, _vp, _vp, _vp, _i64, _i64, _int, _vp]),
    "jq_paged_attention_workspace_bytes": (_sz, [_i64] * 6),
    "jq_paged_attention": (_int, [_vp, _vp, _vp, _vp, _vp, _vp, _i64, _vp, _i64, _i64, _i64, _i64, _i64, _i64, _i64,
                                  _i64, _f, _int, _int, _vp, _vp, _vp, _sz, _vp]),
}

NORM_OUT = {"bf16": 0, "fp8": 1, "int4": 2}

NATIVE_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_jq_block.so")

_lib = None


def lib():
    """The loaded libjq.so with this header's symbols (raises if it has not been built)."""
    global _lib
    if _lib is None:
        loaded = jq.lib()
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(loaded, name)
            fn.restype = res
            fn.argtypes = args
        _lib = loaded
    return _lib


class _Native:
    """The compiled half, loaded at the first call (torch must be loaded before it)."""

    def __getattr__(self, name):
        import torch  # noqa: F401

        if not os.path.exists(NATIVE_PATH):
            raise RuntimeError(f"{NATIVE_PATH} is missing: build the HIP library first, with torch for ROCm installed "
                               "(python -c 'import __graft_entry__ as g; g.build()')")
        lib()
        spec = importlib.util.spec_from_file_location("_jq_block", NATIVE_PATH)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        global _native
        _native = module
        return getattr(module, name)


_native = _Native()


def _stream(stream):
    return None if stream is None else stream.cuda_stream


def _done(result, where):
    if result.__class__ is int:
        raise JQError(result, where)
    return result


def jq_rmsnorm(x, weight, eps=1e-6, residual=None, out="bf16", y=None, scale=None, residual_out=None, stream=None):
    """RMS norm of x (+ residual), bf16 [M,D]; rows of x and of the residual may be apart.

    Returns a tuple.  out = "bf16": (y bf16 [M,D],); "fp8": (y float8_e4m3fn [M,D], scale fp32 [M, ceil(D/128)]), the
    operand of jq_fp8_gemm; "int4": (y uint8 [M,D/2], scale fp32 [M]), the operand of jq_w4a4_gemm.  With a residual
    bf16(x + residual) follows; residual_out=residual updates it in place.
    """
    kind = NORM_OUT.get(out)
    if kind is None:
        raise ValueError(f"out must be one of {sorted(NORM_OUT)}, got {out!r}")
    return _done(_native.rmsnorm(x, weight, eps, residual, kind, y, scale, residual_out, _stream(stream)), "jq_rmsnorm")


def jq_quantize_act_fp8(x, q=None, scale=None, stream=None):
    """x bf16 [M,K] (rows may be apart) -> (q float8_e4m3fn [M,K], scale fp32 [M, ceil(K/128)])."""
    return _done(_native.quantize_act_fp8(x, q, scale, _stream(stream)), "jq_quantize_act_fp8")


def jq_pack_weight_fp8(w, wq=None, w_scale=None, stream=None):
    """w bf16 [N,K] -> (wq float8_e4m3fn [N,K], w_scale fp32 [ceil(N/128), ceil(K/128)])."""
    return _done(_native.pack_weight_fp8(w, wq, w_scale, _stream(stream)), "jq_pack_weight_fp8")


def jq_fp8_workspace_bytes(M, K):
    return int(lib().jq_fp8_workspace_bytes(int(M), int(K)))


def jq_fp8_gemm(q, scale, wq, w_scale, bias=None, y=None, stream=None):
    """The 8-bit product of quantised activations (jq_quantize_act_fp8, or jq_rmsnorm's "fp8"); returns bf16 [M,N]."""
    return _done(_native.fp8_gemm(q, scale, wq, w_scale, bias, y, _stream(stream)), "jq_fp8_gemm")


def jq_fp8_linear(x, wq, w_scale, bias=None, y=None, workspace=None, stream=None):
    """y = 8-bit linear of x (bf16 [M,K], rows may be apart) with a packed weight; returns bf16 [M,N]."""
    return _done(_native.fp8_linear(x, wq, w_scale, bias, y, workspace, _stream(stream)), "jq_fp8_linear")


def jq_rope_append(q, k, v, positions, cos, sin, slots, k_cache, v_cache, k_scale=None, v_scale=None,
                   interleaved=False, q_out=None, stream=None):
    """Rotate q [T,Hq,D] and k [T,Hk,D] (bf16, tokens may be apart) by positions int32 [T] on the first R elements of
    a head (cos, sin fp32 [P,R/2]; None for R = 0), write k and v into the cache at slots int64 [T] (negative: not
    appended; the slots of a call differ), and return the rotated q (q_out=q: in place).  q = None only appends, and
    returns None."""
    return _done(_native.rope_append(q, k, v, positions, cos, sin, slots, k_cache, v_cache, k_scale, v_scale,
                                     interleaved, q_out, _stream(stream)), "jq_rope_append")


def jq_paged_attention_workspace_bytes(B, Tq, Hq, Hk, D, max_len):
    return int(lib().jq_paged_attention_workspace_bytes(int(B), int(Tq), int(Hq), int(Hk), int(D), int(max_len)))


def jq_paged_attention(q, k_cache, v_cache, page_table, lens, k_scale=None, v_scale=None, max_len=None, sm_scale=None,
                       causal=True, out=None, lse=None, workspace=None, stream=None):
    """Attention of the newest tokens q [B,Tq,Hq,D] (bf16) over the cached tokens of each sequence, the new ones among
    them; returns bf16 [B,Tq,Hq,D].

    page_table int32 [B,columns], lens int32 [B]; max_len bounds the lengths (the table's capacity by default) and
    decides how the cache is split; sm_scale is D**-0.5 by default; lse fp32 [B,Tq,Hq], if given, gets the logarithms
    of the softmax denominators.
    """
    return _done(_native.paged_attention(q, k_cache, v_cache, page_table, lens, k_scale, v_scale, max_len, sm_scale,
                                         causal, out, lse, workspace, _stream(stream)), "jq_paged_attention")
