"""e4m3 codes beside an infinity or NaN: the scale shows it, and a finite value's code is that of fl32(v / s)."""

import math

import pytest

from paper_2609_33601_amd import jq_block as jb

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

E4M3 = torch.float8_e4m3fn
ROWS = [math.inf, -math.inf, math.nan, None]  # what stands among a row's values


def _rows(D, seed):
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((len(ROWS), D), generator=g, device="cuda").bfloat16()
    for i, v in enumerate(ROWS):
        if v is not None:
            x[i, 5 + 11 * i] = v
    return x


def _check(codes, scale, y):
    """Codes and the scale that each element has, of values y (64 bits) among which an infinity or NaN stands.

    v / inf is 0 and inf / inf is NaN; with a NaN among them the scale is NaN, and so is every quotient."""
    codes = codes.float()
    nan_block = scale.isnan()
    inf_block = scale.isinf()
    assert torch.equal(codes.isnan(), nan_block | (inf_block & y.isinf()))
    assert not bool(codes[inf_block & y.isfinite()].any())
    fine = ~nan_block & ~inf_block
    assert bool(codes[fine].isfinite().all()) and (not bool(fine.any()) or bool(codes[fine].any()))


@pytest.mark.parametrize("D", [64, 128, 400, 1040, 4096])
def test_quantize(D):
    print("[gpu-block] quantize infinite", D, flush=True)
    x = _rows(D, D)
    q, s = jb.jq_quantize_act_fp8(x)
    per = s.repeat_interleave(128, 1)[:, :D]
    assert s[0, 0] == math.inf and s[1, 0] == math.inf and bool(s[2, 0].isnan()) and bool(s[3].isfinite().all())
    assert bool(s[:, 1:].isfinite().all())
    _check(q, per, x.double())


@pytest.mark.parametrize("D", [128, 272])
def test_pack(D):
    print("[gpu-block] pack infinite", D, flush=True)
    for v in ROWS:
        w = torch.ones((130, D), dtype=torch.bfloat16, device="cuda")
        if v is not None:
            w[3, 100] = v
        q, s = jb.jq_pack_weight_fp8(w)
        per = s.repeat_interleave(128, 0)[:130].repeat_interleave(128, 1)[:, :D]
        _check(q, per, w.double())


@pytest.mark.parametrize("D", [64, 128, 256, 512, 1040, 4096])
def test_norm(D):
    """A row with an infinity has r = 0: its finite values become 0, the infinity NaN, and the scale of its block NaN."""
    print("[gpu-block] norm infinite", D, flush=True)
    x = _rows(D, D + 1)
    w = torch.ones((D,), dtype=torch.bfloat16, device="cuda")
    q, s = jb.jq_rmsnorm(x, w, out="fp8")
    per = s.repeat_interleave(128, 1)[:, :D]
    h = x.double()
    y = h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6)
    _check(q, per, y)
    # an infinite weight: the scale is one, and the other values' codes are 0
    w[7] = math.inf
    q, s = jb.jq_rmsnorm(x[3:], w, out="fp8")
    assert s[0, 0] == math.inf
    y = h[3:] / torch.sqrt((h[3:] ** 2).mean(1, keepdim=True) + 1e-6) * w.double()
    _check(q, s.repeat_interleave(128, 1)[:, :D], y)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,R", [(16, 0), (64, 0), (96, 32), (128, 64), (256, 0)])
def test_append(D, R, interleaved):
    print("[gpu-block] append infinite", D, R, interleaved, flush=True)
    T = len(ROWS)
    kv = []
    for seed in (1, 2):
        x = torch.ones((T, 2, D), dtype=torch.bfloat16, device="cuda") * seed
        for i, v in enumerate(ROWS):
            if v is not None:
                x[i, 1, D - 1 - i] = v  # past the rotated elements, in the second head alone
        kv.append(x)
    cos, sin = (torch.ones((8, R // 2), device="cuda") * c for c in (0.6, 0.8)) if R else (None, None)
    kc, vc = (torch.zeros((1, 2, 16, D), device="cuda").to(E4M3) for _ in range(2))
    ks, vs = (torch.zeros((1, 2, 16), device="cuda") for _ in range(2))
    at = torch.arange(T, device="cuda")
    jb.jq_rope_append(None, *kv, at.int(), cos, sin, at, kc, vc, ks, vs, interleaved=interleaved)
    for cache, scale, x in ((kc, ks, kv[0]), (vc, vs, kv[1])):
        got = cache.view(torch.uint8)[0, :, :T].transpose(0, 1).contiguous().view(E4M3)
        _check(got, scale[0, :, :T].t()[..., None].expand(x.shape), x.double())
        assert bool(scale[0, 0, :T].isfinite().all())
