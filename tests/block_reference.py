"""Plain implementations, in 64 bits, of the decoder block's other operators, for the tests.

Written from the formulas that include/jq_block.h states; nothing of the
package is used.  A function that bounds an error returns the bound beside the
value; the bounds follow from the formats (half a unit in the last place of
bf16 is at most 2^-8 of a value, of e4m3 2^-4 or 2^-10 of the scale) and from
the lengths of the fp32 sums.
"""

import math

import torch

BF16 = 2.0 ** -8 * 1.02     # one rounding to bf16, and what fp32 steps before it may move
E4M3_MAX = 448.0


def blocks(n):
    return -(-n // 128)


def fp8_scale(a):
    """Scale of values whose largest magnitude is a (64 bits)."""
    return torch.where(a > 0, (a / E4M3_MAX).clamp_min(2.0 ** -126), torch.zeros_like(a))


def fp8_blocks(y):
    """y [M,D] -> the scale of each 128 columns [M, ceil(D/128)] and of each element [M,D]."""
    pad = torch.nn.functional.pad(y, (0, -y.shape[1] % 128)).view(y.shape[0], -1, 128)
    s = fp8_scale(pad.abs().amax(2))
    return s, s.repeat_interleave(128, 1)[:, : y.shape[1]]


def check_fp8(codes, scale, y):
    """Codes (float8) and scales stand for y (64 bits) within one rounding."""
    s, per = fp8_blocks(y)
    assert torch.all((scale.double() - s).abs() <= 1e-5 * s), "scales"
    check_fp8_values(codes, scale.double().repeat_interleave(128, 1)[:, : y.shape[1]], y)


def check_fp8_values(codes, scale, y):
    v = codes.double() * scale
    tol = torch.maximum(y.abs() * 2.0 ** -4, scale * 2.0 ** -10) * 1.001
    bad = (v - y).abs() > tol
    assert not bad.any(), f"{int(bad.sum())} codes beyond half a step"
    # the nearest code itself, except beside a tie
    q = torch.where(scale > 0, y / scale.clamp_min(1e-300), torch.zeros_like(y))
    lo, hi = (q * (1 - 1e-4)).float().to(torch.float8_e4m3fn), (q * (1 + 1e-4)).float().clamp(-448, 448).to(torch.float8_e4m3fn)
    sure = lo.view(torch.uint8) == hi.view(torch.uint8)
    assert torch.equal(codes.float()[sure], lo.float()[sure]), "not the nearest codes"  # by value: zero has two signs


def norm(x, weight, eps, residual=None):
    """(y, h) in 64 bits."""
    h = x.double() + (0 if residual is None else residual.double())
    return h / torch.sqrt((h * h).mean(1, keepdim=True) + eps) * weight.double(), h


def fp8_linear(q, s, wq, ws, bias):
    """(y, bound of its error) of quantised operands."""
    K, N = q.shape[1], wq.shape[0]
    kb = torch.arange(K, device=q.device) // 128
    nb = torch.arange(N, device=q.device) // 128
    x = q.double() * s.double()[:, kb]
    w = wq.double() * ws.double()[nb[:, None], kb[None, :]]
    y = x @ w.t()
    size = x.abs() @ w.abs().t()
    if bias is not None:
        y = y + bias.double()
        size = size + bias.double().abs()
    # The matrix core cuts the products of eight neighbouring k at 2^-14 of the largest of them, so each of the seven
    # others loses less than that; the sums above them are fp32.
    return y, BF16 * y.abs() + (7 * 2.0 ** -14 + (16 + blocks(K) + 20) * 2.0 ** -24) * size


def rotate(x, positions, cos, sin, interleaved):
    """(x rotated, bound) of x [T,H,D]."""
    x = x.double()
    out, size = x.clone(), x.abs()
    half = cos.shape[1]
    ok = (positions >= 0) & (positions < cos.shape[0])
    p = torch.where(ok, positions, 0).long()
    c = torch.where(ok[:, None], cos.double()[p], math.nan)[:, None]
    s = torch.where(ok[:, None], sin.double()[p], math.nan)[:, None]
    i = torch.arange(half, device=x.device)
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    a, b = x[..., ia], x[..., ib]
    out[..., ia], out[..., ib] = a * c - b * s, a * s + b * c
    size[..., ia] = size[..., ib] = a.abs() + b.abs()
    return out, BF16 * out.abs() + 2.0 ** -22 * size


def cached(cache, scale, table, n):
    """The first n cached rows of a sequence, 64 bits [Hk, n, D], and of the table's pages only."""
    page = cache.shape[2]
    pages = table.long()[: -(-n // page)]
    x = cache.view(torch.uint8)[pages].view(cache.dtype).double()
    if scale is not None:
        x = x * scale[pages].double()[..., None]
    return x.transpose(0, 1).reshape(cache.shape[1], -1, cache.shape[3])[:, :n]


def attention(q, k_cache, v_cache, table, lens, k_scale=None, v_scale=None, sm_scale=None, causal=True):
    """(out, lse, bound of out) in 64 bits."""
    B, Tq, Hq, D = q.shape
    Hk = k_cache.shape[1]
    G = Hq // Hk
    sm_scale = D ** -0.5 if sm_scale is None else sm_scale
    out = torch.zeros((B, Tq, Hq, D), dtype=torch.float64, device=q.device)
    bound = torch.zeros_like(out)
    lse = torch.full((B, Tq, Hq), -math.inf, dtype=torch.float64, device=q.device)
    for b in range(B):
        n = int(lens[b])
        if n <= 0:
            continue
        k, v = cached(k_cache, k_scale, table[b], n), cached(v_cache, v_scale, table[b], n)
        for i in range(Tq):
            m = min(n, n - Tq + 1 + i) if causal else n
            if m <= 0:
                continue
            x = q[b, i].double().view(Hk, G, D)
            z = (x[:, :, None] * k[:, None, :m]).sum(-1) * sm_scale
            size = ((x.abs()[:, :, None] * k.abs()[:, None, :m]).sum(-1) * abs(sm_scale)).amax(-1, keepdim=True)
            p = torch.softmax(z, -1)
            o = (p[..., None] * v[:, None, :m]).sum(2)
            a = (p[..., None] * v.abs()[:, None, :m]).sum(2)
            out[b, i] = o.reshape(Hq, D)
            lse[b, i] = torch.logsumexp(z, -1).reshape(Hq)
            # P's rounding to bf16; the scores' error, which moves every weight; the sums'; the output's rounding
            e = 2.0 ** -8 + 2 * (D + 16) * 2.0 ** -24 * size + (m + 64) * 2.0 ** -24
            bound[b, i] = (1.02 * (e * a) + BF16 * o.abs()).reshape(Hq, D)
    return out, lse, bound
