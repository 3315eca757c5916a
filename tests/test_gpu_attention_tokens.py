"""Paged attention takes every token that a query sees exactly once: at the seams of tiles, waves, blocks and parts, of
every kernel and join.

With queries of zero all weights are 1, a sum of whole numbers is exact in any order, and a missing or doubled token
changes a count.  Value d of token t is 1 where t % D == d (or where t / D == d, which catches whole stretches), so
output d is the number of such tokens over the number seen.  A second pattern has weights 1 and 2 by position.  The
random ones bound the error with what the kernels do round: weights to 16 bits, outputs to 8.
"""

import math

import pytest

from paper_2609_33601_amd import jq_block as jb
from tests import block_reference as ref
from tests.test_gpu_block import _filled, _randn

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# (Tq, Hq, Hk, D, page, lens): 16-column and 64-column calls of one part, of few, of 8 and of 32 or more
CASES = [
    (1, 8, 2, 64, 16, [1, 15, 16, 17, 31, 32, 33, 127, 128, 129, 383, 384]),
    (1, 4, 1, 128, 32, [385, 511, 512, 513, 1000, 0, 641]),
    (1, 32, 8, 256, 64, [1537, 700, 385]),
    (1, 4, 2, 64, 16, [14001]),
    (1, 7, 1, 128, 64, [32700]),
    (1, 2, 2, 256, 128, [32768]),
    (1, 8, 8, 64, 16, [5121, 4000, 33]),
    (3, 4, 1, 128, 16, [9000, 8193, 2]),
    (16, 1, 1, 64, 16, [4113, 16, 7, 130]),
    (16, 2, 2, 256, 32, [2049, 1025]),
    (20, 2, 2, 64, 16, [64, 65, 130, 383, 0, 19]),
    (64, 3, 1, 128, 32, [2081, 64, 1300, 700]),
    (65, 4, 4, 256, 16, [1000, 449]),
    (33, 2, 1, 64, 16, [8199]),
    (24, 4, 1, 128, 64, [15000]),
    (17, 1, 1, 256, 64, [20011]),
    (300, 2, 1, 64, 16, [301, 500, 260]),
    (130, 4, 2, 128, 16, [130, 700]),
]


def parts_of(Tq, Hq, Hk, D, B, max_len):
    """The parts of the key axis, from what the workspace holds: D sums, a maximum and a sum of each part's rows."""
    n = jb.jq_paged_attention_workspace_bytes(B, Tq, Hq, Hk, D, max_len)
    return max(1, n // (B * Tq * Hq * (D + 2) * 4))


def test_cases_take_every_path():
    """One part; some; those that several groups of lanes join, and 32 or more; with 16 and with 64 columns."""
    seen = set()
    for Tq, Hq, Hk, D, page, lens in CASES:
        p = parts_of(Tq, Hq, Hk, D, len(lens), -(-max(lens) // page) * page)
        seen.add((Tq * (Hq // Hk) > 16, D, "one" if p == 1 else "few" if p < 8 else "some" if p < 32 else "many"))
    for wide in (False, True):
        assert {s[2] for s in seen if s[0] == wide} >= {"one", "some", "many"}, seen
        assert {s[1] for s in seen if s[0] == wide and s[2] == "many"} == {64, 128, 256}, seen


def rounded(want):
    """What an output may be: bf16 of the result, or of one that the weights (as two bf16 each, 2^-16 off at most), the
    powers of two and the division have moved by up to 2^-14."""
    return [(want * (1 + d)).bfloat16().double() for d in (-2.0 ** -14, 2.0 ** -14)]


def _visible(lens, Tq, causal):
    """The number of tokens that each query sees, int64 [B,Tq]."""
    n = torch.tensor(lens, device="cuda")[:, None]
    i = torch.arange(Tq, device="cuda")[None]
    return (n - Tq + 1 + i if causal else n + 0 * i).clamp_min(0)


def _set(cache, scale, table, lens, rows):
    """rows [tokens, D] as the cached rows of every sequence and head, exactly."""
    page = cache.shape[2]
    for b, n in enumerate(lens):
        if n == 0:
            continue
        t = torch.arange(n, device="cuda")
        at = (table[b, t // page].long(), slice(None), t % page)
        x = rows[:n, None].expand(n, cache.shape[1], -1)
        if scale is None:
            cache[at] = x.to(cache.dtype)
        else:  # codes of half the values, scales of two
            cache.view(torch.uint8)[at] = (x / 2).to(cache.dtype).view(torch.uint8)
            scale[at] = 2.0


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("Tq,Hq,Hk,D,page,lens", CASES)
def test_every_token_once(Tq, Hq, Hk, D, page, lens, weighted, causal, kind):
    print("[gpu-attention] once", Tq, Hq, Hk, D, page, lens, weighted, causal, kind, flush=True)
    kc, vc, ks, vs, table, ln, g = _filled(lens, Hk, D, page, kind, Tq + D + len(lens))
    most = max(lens)
    t = torch.arange(most, device="cuda")
    keys = torch.zeros((most, D), device="cuda")
    keys[:, 3] = ((t * 2654435761) >> 7) % 2  # 0 or 1
    _set(kc, ks, table, lens, keys)
    q = torch.zeros((len(lens), Tq, Hq, D), dtype=torch.bfloat16, device="cuda")
    if weighted:
        q[..., 3] = 1.0
    weight = (2.0 ** keys[:, 3]).double() if weighted else torch.ones((most,), dtype=torch.float64, device="cuda")
    seen = _visible(lens, Tq, causal)
    total = torch.cat((weight.new_zeros(1), weight.cumsum(0)))[seen]
    stretch = max(D, -(-most // D))
    for cls in (t % D, t // stretch):
        values = (cls[:, None] == torch.arange(D, device="cuda")).float()
        _set(vc, vs, table, lens, values)
        lse = torch.zeros((len(lens), Tq, Hq), device="cuda")
        out = jb.jq_paged_attention(q, kc, vc, table, ln, ks, vs, sm_scale=math.log(2), causal=causal, lse=lse).double()
        sums = torch.cat((weight.new_zeros((1, D)), (weight[:, None] * values).cumsum(0)))[seen]  # [B,Tq,D]
        want = sums / total.clamp_min(1)[..., None]
        lo, hi = rounded(want[:, :, None])
        assert bool(((lo <= out) & (out <= hi)).all()), "out"
        empty = (seen == 0)[..., None].expand(lse.shape)
        assert torch.equal(lse == -math.inf, empty)
        off = (lse.double() - total.clamp_min(1).log()[..., None]).abs()[~empty]
        assert bool((off <= 2.0 ** -20 * (1 + total.clamp_min(1).log()[..., None].expand(lse.shape)[~empty])).all()), "lse"


def attention64(q, kc, vc, ks, vs, table, lens, causal):
    """(out, lse, bound of out, bound of lse) in 64 bits."""
    B, Tq, Hq, D = q.shape
    Hk = kc.shape[1]
    G = Hq // Hk
    out = torch.zeros((B, Hk, Tq, G, D), dtype=torch.float64, device=q.device)
    bound = torch.zeros_like(out)
    lse = torch.full((B, Hk, Tq, G), -math.inf, dtype=torch.float64, device=q.device)
    lbound = torch.zeros_like(lse)
    for b, n in enumerate(lens):
        if n == 0:
            continue
        k, v = ref.cached(kc, ks, table[b], n), ref.cached(vc, vs, table[b], n)
        for h in range(Hk):
            x = q[b].double().view(Tq, Hk, G, D)[:, h].reshape(Tq * G, D)
            z = torch.mm(x, k[h].t().contiguous()) * D ** -0.5
            size = torch.mm(x.abs(), k[h].abs().t().contiguous()).amax(1, keepdim=True) * D ** -0.5
            m = _visible([n], Tq, causal)[0].repeat_interleave(G)[:, None]
            z = z.masked_fill(torch.arange(n, device=q.device) >= m, -math.inf)
            some = m[:, 0] > 0
            p = torch.where(some[:, None], torch.softmax(z, 1), 0.0)
            o, a = torch.mm(p, v[h].contiguous()), torch.mm(p, v[h].abs().contiguous())
            # the scores' and their sums' error in fp32, which moves every weight; then what a weight as two bf16 loses
            # (the second rounds 2^-7 of it to 2^-8 of that), and the output's own rounding
            s = 2 * (D + 16) * 2.0 ** -24 * size + (n + 64) * 2.0 ** -24
            out[b, h], bound[b, h] = o.view(Tq, G, D), ((2.0 ** -15 + s) * a + ref.BF16 * o.abs()).view(Tq, G, D)
            l = torch.logsumexp(z, 1)
            lse[b, h] = l.view(Tq, G)
            lbound[b, h] = torch.where(some, s[:, 0] + 2.0 ** -20 * (1 + l.abs()), 0.0).view(Tq, G)
    turn = lambda x: x.transpose(1, 2).reshape(B, Tq, Hq, *x.shape[4:])  # noqa: E731
    return turn(out), turn(lse), turn(bound), turn(lbound)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("Tq,Hq,Hk,D,page,lens", CASES)
def test_error(Tq, Hq, Hk, D, page, lens, causal, kind):
    """Within the bound, and in rms no more than a tenth above the outputs' own rounding."""
    print("[gpu-attention] error", Tq, Hq, Hk, D, page, lens, causal, kind, flush=True)
    kc, vc, ks, vs, table, ln, g = _filled(lens, Hk, D, page, kind, 7 * Tq + D + len(lens))
    q = _randn((len(lens), Tq, Hq, D), g, 1.5)
    lse = torch.zeros((len(lens), Tq, Hq), device="cuda")
    out = jb.jq_paged_attention(q, kc, vc, table, ln, ks, vs, causal=causal, lse=lse).double()
    want, wlse, bound, lbound = attention64(q, kc, vc, ks, vs, table, lens, causal)
    assert bool(((out - want).abs() <= bound).all()), "out"
    empty = wlse == -math.inf
    assert torch.equal(lse == -math.inf, empty) and not bool(out[empty].any())
    assert bool(((lse.double() - wlse).abs() <= lbound)[~empty].all()), "lse"
    assert float((out - want).norm()) <= 1.1 * float((want.bfloat16().double() - want).norm())


def test_a_missing_token_shows():
    """The bounds above, held against results that lack one token or have it twice."""
    D, n = 64, 4097
    cls = torch.arange(n) % D
    lo, hi = rounded(torch.bincount(cls, minlength=D).double() / n)
    for lost in (0, 31, 32, 127, 128, 640, 4095, 4096):
        for times in (0, 2):
            count = torch.ones((n,), dtype=torch.float64)
            count[lost] = times
            got = (torch.bincount(cls, weights=count, minlength=D) / count.sum()).bfloat16().double()
            assert not bool(((lo <= got) & (got <= hi)).all())
            assert abs(math.log(float(count.sum())) - math.log(n)) > 2.0 ** -20 * (1 + math.log(n))
