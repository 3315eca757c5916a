"""Python binding of the decoder block's other operators (include/jq_block.h).

What a served block runs around its W4A4 linears (jq.py): the RMS norm that
feeds a quantised linear, the 8-bit linear, the rotation of new queries and
keys with their append to a paged cache, and attention over that cache.  As in
jq.py, every function only marshals GPU torch tensors into pointers and the
current HIP stream and raises on a non-OK status; there is no other path.

    cache    k_cache, v_cache  [pages, Hk, page_size, D]  bf16, or float8_e4m3fn with
             k_scale, v_scale  [pages, Hk, page_size]     fp32 for each token and head
"""

import ctypes

from . import jq
from .jq import _check, _dev, _stream_ptr, _torch

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


def _rows(t, dtype, shape, name):
    """(device pointer, elements between rows) of `t`, a GPU tensor of this dtype and shape whose rows (all but the
    first dimension) are contiguous."""
    torch = _torch()
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be on the GPU, got {t.device}")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.is_contiguous():
        return t.data_ptr(), t[0].numel() if t.shape[0] else 0
    need = 1
    for size, stride in zip(reversed(t.shape[1:]), reversed(t.stride()[1:])):
        if size != 1 and stride != need:
            raise ValueError(f"{name}: the elements of a row must be contiguous")
        need *= size
    return t.data_ptr(), t.stride(0) if t.shape[0] > 1 else need


def _one_device(first, *others):
    for t in others:
        if t is not None and t.device != first.device:
            raise ValueError(f"all tensors must be on one device, got {first.device} and {t.device}")


def jq_rmsnorm(x, weight, eps=1e-6, residual=None, out="bf16", y=None, scale=None, residual_out=None, stream=None):
    """RMS norm of x (+ residual), bf16 [M,D]; rows of x and of the residual may be apart.

    Returns a tuple.  out = "bf16": (y bf16 [M,D],); "fp8": (y float8_e4m3fn [M,D], scale fp32 [M, ceil(D/128)]), the
    operand of jq_fp8_gemm; "int4": (y uint8 [M,D/2], scale fp32 [M]), the operand of jq_w4a4_gemm.  With a residual
    bf16(x + residual) follows; residual_out=residual updates it in place.
    """
    torch = _torch()
    M, D = x.shape
    if out not in NORM_OUT:
        raise ValueError(f"out must be one of {sorted(NORM_OUT)}, got {out!r}")
    if residual is None and residual_out is not None:
        raise ValueError("residual_out without a residual")
    xp, xs = _rows(x, torch.bfloat16, None, "x")
    _one_device(x, weight, residual, y, scale, residual_out)
    dtype, shape = torch.bfloat16, (M, D)
    sshape = None
    if out == "fp8":
        dtype, sshape = torch.float8_e4m3fn, (M, (D + 127) // 128)
    elif out == "int4":
        dtype, shape, sshape = torch.uint8, (M, D // 2), (M,)
    if y is None:
        y = torch.empty(shape, dtype=dtype, device=x.device)
    sp = None
    if sshape is not None:
        if scale is None:
            scale = torch.empty(sshape, dtype=torch.float32, device=x.device)
        sp = _dev(scale, torch.float32, sshape, "scale")
    elif scale is not None:
        raise ValueError("a bf16 output has no scale")
    rp = ro = None
    rs = ros = 0
    if residual is not None:
        rp, rs = _rows(residual, torch.bfloat16, x.shape, "residual")
        if residual_out is None:
            residual_out = torch.empty((M, D), dtype=torch.bfloat16, device=x.device)
        ro, ros = _rows(residual_out, torch.bfloat16, x.shape, "residual_out")
    st = lib().jq_rmsnorm(xp, xs, rp, rs, _dev(weight, torch.bfloat16, (D,), "weight"), M, D, eps, NORM_OUT[out],
                          _dev(y, dtype, shape, "y"), sp, ro, ros, _stream_ptr(stream))
    _check(st, "jq_rmsnorm")
    res = (y,) if sshape is None else (y, scale)
    return res if residual is None else res + (residual_out,)


def jq_quantize_act_fp8(x, q=None, scale=None, stream=None):
    """x bf16 [M,K] (rows may be apart) -> (q float8_e4m3fn [M,K], scale fp32 [M, ceil(K/128)])."""
    torch = _torch()
    M, K = x.shape
    xp, xs = _rows(x, torch.bfloat16, None, "x")
    _one_device(x, q, scale)
    sshape = (M, (K + 127) // 128)
    if q is None:
        q = torch.empty((M, K), dtype=torch.float8_e4m3fn, device=x.device)
    if scale is None:
        scale = torch.empty(sshape, dtype=torch.float32, device=x.device)
    st = lib().jq_quantize_act_fp8(xp, xs, M, K, _dev(q, torch.float8_e4m3fn, (M, K), "q"),
                                   _dev(scale, torch.float32, sshape, "scale"), _stream_ptr(stream))
    _check(st, "jq_quantize_act_fp8")
    return q, scale


def jq_pack_weight_fp8(w, wq=None, w_scale=None, stream=None):
    """w bf16 [N,K] -> (wq float8_e4m3fn [N,K], w_scale fp32 [ceil(N/128), ceil(K/128)])."""
    torch = _torch()
    N, K = w.shape
    _one_device(w, wq, w_scale)
    sshape = ((N + 127) // 128, (K + 127) // 128)
    if wq is None:
        wq = torch.empty((N, K), dtype=torch.float8_e4m3fn, device=w.device)
    if w_scale is None:
        w_scale = torch.empty(sshape, dtype=torch.float32, device=w.device)
    st = lib().jq_pack_weight_fp8(_dev(w, torch.bfloat16, None, "w"), N, K,
                                  _dev(wq, torch.float8_e4m3fn, (N, K), "wq"),
                                  _dev(w_scale, torch.float32, sshape, "w_scale"), _stream_ptr(stream))
    _check(st, "jq_pack_weight_fp8")
    return wq, w_scale


def jq_fp8_workspace_bytes(M, K):
    return int(lib().jq_fp8_workspace_bytes(int(M), int(K)))


def _weight_fp8(wq, w_scale, K):
    torch = _torch()
    N = wq.shape[0]
    return N, _dev(wq, torch.float8_e4m3fn, (N, K), "wq"), _dev(w_scale, torch.float32,
                                                               ((N + 127) // 128, (K + 127) // 128), "w_scale")


def jq_fp8_gemm(q, scale, wq, w_scale, bias=None, y=None, stream=None):
    """The 8-bit product of quantised activations (jq_quantize_act_fp8, or jq_rmsnorm's "fp8"); returns bf16 [M,N]."""
    torch = _torch()
    M, K = q.shape
    N, wp, wsp = _weight_fp8(wq, w_scale, K)
    _one_device(q, scale, wq, w_scale, bias, y)
    if y is None:
        y = torch.empty((M, N), dtype=torch.bfloat16, device=q.device)
    bp = None if bias is None else _dev(bias, torch.bfloat16, (N,), "bias")
    st = lib().jq_fp8_gemm(_dev(q, torch.float8_e4m3fn, None, "q"),
                           _dev(scale, torch.float32, (M, (K + 127) // 128), "scale"), M, K, wp, wsp, N, bp,
                           _dev(y, torch.bfloat16, (M, N), "y"), _stream_ptr(stream))
    _check(st, "jq_fp8_gemm")
    return y


def jq_fp8_linear(x, wq, w_scale, bias=None, y=None, workspace=None, stream=None):
    """y = 8-bit linear of x (bf16 [M,K], rows may be apart) with a packed weight; returns bf16 [M,N]."""
    torch = _torch()
    M, K = x.shape
    xp, xs = _rows(x, torch.bfloat16, None, "x")
    N, wp, wsp = _weight_fp8(wq, w_scale, K)
    _one_device(x, wq, w_scale, bias, y, workspace)
    if y is None:
        y = torch.empty((M, N), dtype=torch.bfloat16, device=x.device)
    if workspace is None:
        workspace = torch.empty((jq_fp8_workspace_bytes(M, K),), dtype=torch.uint8, device=x.device)
    bp = None if bias is None else _dev(bias, torch.bfloat16, (N,), "bias")
    st = lib().jq_fp8_linear(xp, xs, M, K, wp, wsp, N, bp, _dev(y, torch.bfloat16, (M, N), "y"),
                             _dev(workspace, torch.uint8, None, "workspace"), workspace.numel(), _stream_ptr(stream))
    _check(st, "jq_fp8_linear")
    return y


def _cache(k_cache, v_cache, k_scale, v_scale):
    """(pages, Hk, page_size, D, type, the four pointers) of a paged cache."""
    torch = _torch()
    if k_cache.dim() != 4:
        raise ValueError("a cache is [pages, Hk, page_size, D]")
    pages, Hk, page, D = k_cache.shape
    if k_cache.dtype is torch.bfloat16:
        if k_scale is not None or v_scale is not None:
            raise ValueError("a bf16 cache has no scales")
        return (pages, Hk, page, D, 0, _dev(k_cache, torch.bfloat16, None, "k_cache"),
                _dev(v_cache, torch.bfloat16, k_cache.shape, "v_cache"), None, None)
    if k_scale is None or v_scale is None:
        raise ValueError("an 8-bit cache needs k_scale and v_scale")
    return (pages, Hk, page, D, 1, _dev(k_cache, torch.float8_e4m3fn, None, "k_cache"),
            _dev(v_cache, torch.float8_e4m3fn, k_cache.shape, "v_cache"),
            _dev(k_scale, torch.float32, k_cache.shape[:3], "k_scale"),
            _dev(v_scale, torch.float32, k_cache.shape[:3], "v_scale"))


def jq_rope_append(q, k, v, positions, cos, sin, slots, k_cache, v_cache, k_scale=None, v_scale=None,
                   interleaved=False, q_out=None, stream=None):
    """Rotate q [T,Hq,D] and k [T,Hk,D] (bf16, tokens may be apart) by positions int32 [T] on the first R elements of
    a head (cos, sin fp32 [P,R/2]; None for R = 0), write k and v into the cache at slots int64 [T] (negative: not
    appended), and return the rotated q (q_out=q: in place).  q = None only appends."""
    torch = _torch()
    pages, Hk, page, D, kind, kcp, vcp, ksp, vsp = _cache(k_cache, v_cache, k_scale, v_scale)
    T = k.shape[0]
    kp, ks = _rows(k, torch.bfloat16, (T, Hk, D), "k")
    vp, vs = _rows(v, torch.bfloat16, (T, Hk, D), "v")
    _one_device(k, q, v, positions, cos, sin, slots, k_cache, v_cache, k_scale, v_scale, q_out)
    qp = qop = None
    Hq = qs = qos = 0
    if q is not None:
        Hq = q.shape[1]
        qp, qs = _rows(q, torch.bfloat16, (T, Hq, D), "q")
        if q_out is None:
            q_out = torch.empty((T, Hq, D), dtype=torch.bfloat16, device=q.device)
        qop, qos = _rows(q_out, torch.bfloat16, (T, Hq, D), "q_out")
    elif q_out is not None:
        raise ValueError("q_out without q")
    P = R = 0
    cp = sp = None
    if cos is not None:
        P, R = cos.shape[0], 2 * cos.shape[1]
        cp = _dev(cos, torch.float32, None, "cos")
        sp = _dev(sin, torch.float32, cos.shape, "sin")
    st = lib().jq_rope_append(qp, qs, kp, ks, vp, vs, T, Hq, Hk, D, _dev(positions, torch.int32, (T,), "positions"),
                              cp, sp, P, R, int(interleaved), _dev(slots, torch.int64, (T,), "slots"), qop, qos, kcp,
                              vcp, ksp, vsp, pages, page, kind, _stream_ptr(stream))
    _check(st, "jq_rope_append")
    return q_out


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
    torch = _torch()
    B, Tq, Hq, D = q.shape
    pages, Hk, page, Dc, kind, kcp, vcp, ksp, vsp = _cache(k_cache, v_cache, k_scale, v_scale)
    if Dc != D:
        raise ValueError(f"q has heads of {D}, the cache of {Dc}")
    _one_device(q, k_cache, v_cache, k_scale, v_scale, page_table, lens, out, lse, workspace)
    if page_table.dim() != 2 or page_table.shape[0] != B:
        raise ValueError(f"page_table must be [{B}, columns], got {tuple(page_table.shape)}")
    columns = page_table.shape[1]
    if max_len is None:
        max_len = columns * page
    if sm_scale is None:
        sm_scale = D ** -0.5
    if out is None:
        out = torch.empty(q.shape, dtype=torch.bfloat16, device=q.device)
    if workspace is None:
        need = jq_paged_attention_workspace_bytes(B, Tq, Hq, Hk, D, max_len)
        workspace = torch.empty((need,), dtype=torch.uint8, device=q.device) if need else None
    wp, wn = (None, 0) if workspace is None else (_dev(workspace, torch.uint8, None, "workspace"), workspace.numel())
    st = lib().jq_paged_attention(_dev(q, torch.bfloat16, None, "q"), kcp, vcp, ksp, vsp,
                                  _dev(page_table, torch.int32, None, "page_table"), columns,
                                  _dev(lens, torch.int32, (B,), "lens"), B, Tq, Hq, Hk, D, pages, page, max_len,
                                  sm_scale, int(causal), kind, _dev(out, torch.bfloat16, q.shape, "out"),
                                  None if lse is None else _dev(lse, torch.float32, (B, Tq, Hq), "lse"), wp, wn,
                                  _stream_ptr(stream))
    _check(st, "jq_paged_attention")
    return out
