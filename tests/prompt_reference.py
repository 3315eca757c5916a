"""Plain implementations, in 64 bits, of the operators that take whole prompts through a block, for the tests.

Written from the formulas that include/jq_block.h states; nothing of the package is used.  A function that bounds an
error returns the bound beside the value, from the formats and the lengths of the fp32 sums.
"""

import math

import torch

from tests import block_reference as ref

BF16 = ref.BF16


def attention(q, k, v, causal=True, sm_scale=None):
    """(out, lse, bound of out, bound of lse) of one sequence: q [n,Hq,D] over k, v [m,Hk,D], 64 bits."""
    n, Hq, D = q.shape
    m, Hk = k.shape[0], k.shape[1]
    sm_scale = D ** -0.5 if sm_scale is None else sm_scale
    out = torch.zeros((n, Hq, D), dtype=torch.float64, device=q.device)
    bound, lse = torch.zeros_like(out), torch.full((n, Hq), -math.inf, dtype=torch.float64, device=q.device)
    lse_bound = torch.zeros_like(lse)
    if m == 0:
        return out, lse, bound, lse_bound
    t, i = torch.arange(m, device=q.device)[None], torch.arange(n, device=q.device)[:, None]
    seen = t <= m - n + i if causal else torch.ones((n, m), dtype=torch.bool, device=q.device)
    some = seen.any(1)
    for h in range(Hq):
        x, kh, vh = q[:, h].double(), k[:, h * Hk // Hq].double(), v[:, h * Hk // Hq].double()
        z = (x @ kh.t() * sm_scale).masked_fill(~seen, -math.inf)
        size = (x.abs() @ kh.abs().t() * abs(sm_scale)).nan_to_num(nan=0.0, posinf=0.0).masked_fill(~seen, 0.0).amax(1, keepdim=True)
        top = z.amax(1, keepdim=True)
        w = torch.exp(z - torch.where(top > -math.inf, top, 0.0))
        total = w.sum(1, keepdim=True)
        p = torch.where(total > 0, w / total, 0.0)
        # a token counts for the queries that see it alone, whatever its values are
        bad = ~vh.isfinite().all(1)
        o = p @ torch.where(bad[:, None], 0.0, vh)
        a = p @ torch.where(bad[:, None], 0.0, vh.abs())
        for j in bad.nonzero().flatten().tolist():
            o = o + torch.where(seen[:, j, None], p[:, j, None] * vh[j], 0.0)
            # its weight is rounded too, which moves what its finite values add
            a = a + p[:, j, None] * torch.where(vh[j].isfinite(), vh[j].abs(), 0.0)
        out[:, h] = torch.where(some[:, None], o, 0.0)
        lse[:, h] = torch.where(some, (top + torch.log(total))[:, 0], -math.inf)
        # a score's error moves every weight, the denominator's too; weights are rounded to bf16 once; the sums'
        # errors; the output's rounding
        score = (D + 16) * 2.0 ** -24 * size
        e = 2.0 ** -8 + 2 * score + (m + 64) * 2.0 ** -24
        bound[:, h] = 1.02 * e * a + BF16 * o.abs() + 2.0 ** -126
        lse_bound[:, h] = (score + (m + 64) * 2.0 ** -24)[:, 0] + 2.0 ** -22 * lse[:, h].abs().nan_to_num(posinf=0.0) + 2.0 ** -22
    return out, lse, bound, lse_bound


def check_attention(got, got_lse, q, k, v, causal=True, sm_scale=None):
    """One sequence's rows against 64 bits."""
    out, lse, bound, lse_bound = attention(q, k, v, causal, sm_scale)
    got = got.double()
    fine = out.isfinite()
    assert torch.equal(fine, got.isfinite()), "infinities or NaN elsewhere"
    inf = out.isinf()
    assert torch.equal(got[inf], out[inf]) and torch.equal(out.isnan(), got.isnan()), "other infinities"
    off = (got - out).abs()[fine] - bound[fine]
    assert not (off > 0).any(), f"{int((off > 0).sum())} outputs beyond their bound, worst by {float(off.max())}"
    if got_lse is not None:
        g = got_lse.double()
        known = lse.isfinite()
        assert torch.equal(g[~known].nan_to_num(nan=7.0), lse[~known].nan_to_num(nan=7.0)), "lse of empty rows"
        assert torch.all((g - lse).abs()[known] <= lse_bound[known]), "lse"


def head_norm(x, weight, eps):
    """(x normalised over its last axis, how far fp32 may be off) in 64 bits."""
    x = x.double()
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
    return y, (x.shape[-1] + 8) * 2.0 ** -24 * y.abs()


def rotate(y, err, positions, cos, sin, interleaved):
    """(y [T,H,D] rotated, how far fp32 may be off, given err of y) in 64 bits."""
    out, e = y.clone(), err.clone()
    half = 0 if cos is None else cos.shape[1]
    if half == 0:
        return out, e
    ok = (positions >= 0) & (positions < cos.shape[0])
    p = torch.where(ok, positions, 0).long()
    c = torch.where(ok[:, None], cos.double()[p], math.nan)[:, None]
    s = torch.where(ok[:, None], sin.double()[p], math.nan)[:, None]
    i = torch.arange(half, device=y.device)
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    a, b = y[..., ia], y[..., ib]
    out[..., ia], out[..., ib] = a * c - b * s, a * s + b * c
    e[..., ia] = e[..., ib] = err[..., ia] + err[..., ib] + 2.0 ** -22 * (a.abs() + b.abs())
    return out, e


def activation(gate, up, act):
    """act(gate) * up in 64 bits, without cancellation in the left tail."""
    x = gate.double()
    if act == "silu":
        y = x * torch.sigmoid(x)
    elif act == "gelu":
        y = x * 0.5 * torch.special.erfc(-x / math.sqrt(2.0))
    else:
        y = x * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3))
    return y if up is None else y * up.double()
