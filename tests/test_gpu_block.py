"""The decoder block's other operators on the GPU, against plain implementations in 64 bits
(tests/block_reference.py), at the sizes, masks and layouts where they can go wrong."""

import math

import pytest

from paper_2609_33601_amd import jq, jq_block as jb
from tests import block_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

E4M3 = torch.float8_e4m3fn


def _gen(seed):
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(shape, g, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).bfloat16()


def _say(*a):
    print("[gpu-block]", *a, flush=True)


def _within(got, want, bound, what):
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in other places"
    d = torch.nan_to_num((got - want).abs() - bound)
    assert bool((d <= 0).all()), f"{what}: off by up to {float(d.max())} beyond the bound"


# ---------------------------------------------------------------------------
# RMS norm

NORM_SHAPES = [(1, 8), (3, 64), (70, 72), (33, 128), (5, 136), (130, 256), (9, 264), (7, 512), (4, 1000), (2, 1032),
               (6, 4096), (3, 4104), (2, 8200), (1, 16384), (2, 32768), (1, 65536), (1200, 192), (700, 3072)]


@pytest.mark.parametrize("out", ["bf16", "fp8", "int4"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("M,D", NORM_SHAPES)
def test_norm(M, D, residual, out):
    if out == "int4" and D % 64:
        pytest.skip("int4 rows are whole 64s")
    _say("norm", M, D, residual, out)
    g = _gen(M * 131 + D)
    x = _randn((M, D), g, 2.0)
    x[:, :: max(1, D // 3)] *= 30
    x[0] = 0                                     # a row of zeros
    if M > 2:
        x[1] *= 2.0 ** -60                       # eps decides
        x[2] = _randn((D,), g, 1e4)
    r = _randn((M, D), g, 3.0) if residual else None
    if residual:
        r[0] = 0
    w = _randn((D,), g, 0.5) + 1
    got = jb.jq_rmsnorm(x, w, 1e-5, residual=r, out=out)
    y, h = ref.norm(x, w, 1e-5, r)
    if residual:
        _within(got[-1], h, ref.BF16 * h.abs(), "residual")
        got = got[:-1]
    if out == "bf16":
        assert len(got) == 1
        _within(got[0], y, ref.BF16 * y.abs(), "y")
    elif out == "fp8":
        ref.check_fp8(got[0], got[1], y)
    else:
        s = y.abs().amax(1) / 7
        assert bool(((got[1].double() - s).abs() <= 1e-5 * s).all())
        lo, hi = (got[0] & 15).to(torch.int8), (got[0] >> 4).to(torch.int8)
        q = torch.stack((lo, hi), 2).view(M, D)
        q = torch.where(q > 7, q - 16, q).double()
        t = torch.where(s[:, None] > 0, y / s.clamp_min(1e-300)[:, None], torch.zeros_like(y))
        assert bool(((q - t).abs() <= 0.5 + 1e-4).all())
        sure = ((t - t.floor()) - 0.5).abs() > 1e-4
        assert torch.equal(q[sure], t.round()[sure])


def test_norm_strides_and_in_place():
    g = _gen(3)
    M, D = 37, 520
    _say("norm strides")
    big, rbig = _randn((M, 3 * D), g), _randn((M, 2 * D), g)
    x, r = big[:, D:2 * D], rbig[:, D:]
    w = _randn((D,), g)
    y0, h0 = jb.jq_rmsnorm(x.contiguous(), w, residual=r.contiguous())
    keep, rkeep = big.clone(), rbig.clone()
    y1, h1 = jb.jq_rmsnorm(x, w, residual=r, residual_out=r)
    assert h1.data_ptr() == r.data_ptr()
    assert torch.equal(y0, y1) and torch.equal(h0, h1)
    assert torch.equal(big, keep) and torch.equal(rbig[:, :D], rkeep[:, :D])
    # the norm may overwrite its input
    x2 = x.contiguous()
    assert torch.equal(jb.jq_rmsnorm(x2, w, y=x2)[0], jb.jq_rmsnorm(x, w)[0])


@pytest.mark.parametrize("out", ["bf16", "fp8"])
@pytest.mark.parametrize("D", [128, 4096])
def test_norm_not_finite(D, out):
    """An infinity or NaN stays in its row."""
    _say("norm not finite", D, out)
    g = _gen(4)
    x, w = _randn((9, D), g), _randn((D,), g) + 2
    good = jb.jq_rmsnorm(x, w, out=out)
    x[3, 5], x[6, D - 1] = math.inf, math.nan
    got = jb.jq_rmsnorm(x, w, out=out)
    rows = [0, 1, 2, 4, 5, 7, 8]
    if out == "bf16":
        assert torch.equal(got[0][rows], good[0][rows])
        assert bool(got[0][6].isnan().all()) and bool(got[0][3, 5].isnan())
    else:
        assert torch.equal(got[0].view(torch.uint8)[rows], good[0].view(torch.uint8)[rows])
        assert torch.equal(got[1][rows], good[1][rows])
        assert not bool(torch.isfinite(got[1][6]).any())
        assert not bool(torch.isfinite(got[1][3, 0]))


def test_norm_int4_feeds_the_linear():
    """The int4 form is the operand of jq_w4a4_gemm."""
    _say("norm int4 -> W4A4")
    g = _gen(5)
    M, K, N = 19, 256, 96
    x, w = _randn((M, K), g), _randn((K,), g) + 1
    wq, ws = jq.jq_pack_weight_int4(_randn((N, K), g, 0.05))
    q, s = jb.jq_rmsnorm(x, w, out="int4")
    y = jq.jq_w4a4_gemm(q, s, wq, ws)
    acc = jq.jq_w4a4_gemm_i32(q, wq).double()
    want = acc * s.double()[:, None] * ws.double()
    _within(y, want, ref.BF16 * want.abs(), "y")


# ---------------------------------------------------------------------------
# 8-bit linear


@pytest.mark.parametrize("M,K", [(1, 16), (3, 128), (5, 144), (65, 640), (2, 4096), (7, 12288), (1, 65536), (300, 1040)])
def test_quantize_fp8(M, K):
    _say("quantize", M, K)
    g = _gen(M + K)
    x = _randn((M, 2 * K), g, 5.0)[:, K:]
    x[0, : min(K, 128)] = 0
    if M > 2:
        x[1] *= 2.0 ** -120
        x[2] = x[2].sign() * 3e38
    q, s = jb.jq_quantize_act_fp8(x)
    ref.check_fp8(q, s, x.double())
    assert bool((s[0, 0] == 0)) and not bool(q.view(torch.uint8)[0, : min(K, 128)].any())
    x = x.contiguous()
    x[0, 3] = math.nan
    q, s = jb.jq_quantize_act_fp8(x)
    assert bool(s[0, 0].isnan()) and bool(torch.isfinite(s.flatten()[1:]).all())


@pytest.mark.parametrize("N,K", [(1, 16), (128, 128), (129, 272), (300, 1040), (77, 4096)])
def test_pack_fp8(N, K):
    _say("pack", N, K)
    g = _gen(N + K)
    w = _randn((N, K), g, 0.02)
    q, s = jb.jq_pack_weight_fp8(w)
    pad = torch.nn.functional.pad(w.double(), (0, -K % 128, 0, -N % 128)).view(ref.blocks(N), 128, -1, 128)
    want = ref.fp8_scale(pad.abs().amax((1, 3)))
    assert bool(((s.double() - want).abs() <= 1e-5 * want).all())
    per = s.double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
    ref.check_fp8_values(q, per, w.double())


def _fp8_operands(M, K, N, seed):
    g = _gen(seed)
    x = _randn((M, K), g)
    x[:, :: max(1, K // 5)] *= 20
    x[M // 2] = 0
    q, s = jb.jq_quantize_act_fp8(x)
    wq, ws = jb.jq_pack_weight_fp8(_randn((N, K), g, 0.02))
    # scales that differ from block to block, so that one taken from the wrong place shows
    ws *= torch.rand(ws.shape, generator=g, device="cuda") * 4 + 0.25
    s *= torch.rand(s.shape, generator=g, device="cuda") * 4 + 0.25
    return x, q, s, wq, ws, _randn((N,), g)


GEMM_SHAPES = [(1, 16, 1), (1, 128, 16), (1, 4096, 4096), (2, 144, 33), (16, 256, 64), (17, 1040, 129), (33, 4112, 257),
               (77, 640, 1000), (100, 2048, 96), (128, 128, 128), (129, 400, 130), (200, 1024, 4096), (257, 272, 513),
               (300, 4096, 255), (1000, 528, 1030), (1111, 1152, 2222), (4100, 384, 4200), (5, 65536, 20), (2, 16, 5000),
               (200, 4096, 2100), (130, 1040, 2500), (700, 2064, 1203), (1030, 16, 2100), (513, 144, 2056),
               (2500, 2192, 2600), (3000, 16, 4104), (37, 624, 2737), (24, 4112, 4100),
               (4096, 400, 4096), (4352, 656, 8201)]


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("M,K,N", GEMM_SHAPES)
def test_fp8_gemm(M, K, N, bias):
    _say("gemm", M, K, N, bias)
    _, q, s, wq, ws, b = _fp8_operands(M, K, N, M + K + N)
    guard = torch.full((M * N + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
    y = jb.jq_fp8_gemm(q, s, wq, ws, bias=b if bias else None, y=guard[: M * N].view(M, N))
    want, bound = ref.fp8_linear(q, s, wq, ws, b if bias else None)
    _within(y, want, bound, "y")
    assert bool((guard[M * N:] == 7.0).all()), "written past the output"
    again = jb.jq_fp8_gemm(q, s, wq, ws, bias=b if bias else None)
    assert torch.equal(again, y), "two calls differ"


@pytest.mark.parametrize("M,K,N", GEMM_SHAPES)
def test_fp8_gemm_exact(M, K, N):
    """Whole-number codes and scales that are powers of two: every product and sum is exact, and so is the output."""
    _say("gemm exact", M, K, N)
    g = _gen(M * 7 + K + N)
    pick = torch.tensor([-4, -3, -2, -1.5, -1, -0.5, 0, 0.5, 1, 1.5, 2, 3, 4], device="cuda")
    q, wq = (pick[torch.randint(0, 13, shape, generator=g, device="cuda")].to(E4M3) for shape in ((M, K), (N, K)))
    s, ws = (2.0 ** torch.randint(-2, 2, shape, generator=g, device="cuda").float()
             for shape in ((M, ref.blocks(K)), (ref.blocks(N), ref.blocks(K))))
    want = ref.fp8_linear(q, s, wq, ws, None)[0]     # a multiple of 2^-6 below 2^18 * 16: 24 bits hold it up to K = 4096
    if K > 4096:
        pytest.skip("sums may need more than 24 bits")
    assert torch.equal(jb.jq_fp8_gemm(q, s, wq, ws), want.float().bfloat16())


@pytest.mark.parametrize("M,K,N", [(1, 256, 48), (40, 1040, 200), (300, 640, 520)])
def test_fp8_linear_is_its_parts(M, K, N):
    _say("linear", M, K, N)
    x, _, _, wq, ws, b = _fp8_operands(M, K, N, 9)
    wide = torch.zeros((M, K + 24), dtype=torch.bfloat16, device="cuda")
    wide[:, 8:8 + K] = x
    q, s = jb.jq_quantize_act_fp8(x)
    assert torch.equal(jb.jq_fp8_linear(wide[:, 8:8 + K], wq, ws, bias=b), jb.jq_fp8_gemm(q, s, wq, ws, bias=b))


@pytest.mark.parametrize("M", [4, 200, 4300])
def test_fp8_gemm_not_finite(M):
    """A NaN scale or code shows in its row (of activations) or column (of weights) alone."""
    _say("gemm not finite", M)
    K, N = 384, 4200 if M > 4000 else 300
    _, q, s, wq, ws, _ = _fp8_operands(M, K, N, 10)
    good = jb.jq_fp8_gemm(q, s, wq, ws)
    s[1, 2] = math.nan
    wq.view(torch.uint8)[N - 1, 7] = 0x7F
    y = jb.jq_fp8_gemm(q, s, wq, ws)
    nan = torch.zeros_like(y, dtype=torch.bool)
    nan[1], nan[:, N - 1] = True, True
    assert torch.equal(y.isnan(), nan)
    assert torch.equal(y[~nan], good[~nan])


# ---------------------------------------------------------------------------
# rotation and append


def _tables(P, R):
    f = 10000.0 ** (-torch.arange(0, R, 2, device="cuda", dtype=torch.float64) / R)
    a = torch.arange(P, device="cuda", dtype=torch.float64)[:, None] * f
    return a.cos().float(), a.sin().float()


def _cache(pages, Hk, page, D, kind):
    """Caches filled with a pattern, and their scales or None."""
    if kind == "bf16":
        return [torch.full((pages, Hk, page, D), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)] + [None] * 2
    c = [torch.full((pages, Hk, page, D), 3.0, device="cuda").to(E4M3) for _ in range(2)]
    return c + [torch.full((pages, Hk, page), 5.0, device="cuda") for _ in range(2)]


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,Hq,Hk,D,R,page", [(1, 1, 1, 64, 64, 16), (5, 8, 2, 128, 128, 16), (67, 32, 8, 128, 64, 32),
                                               (9, 3, 3, 256, 256, 64), (130, 4, 1, 64, 16, 128), (4, 2, 2, 96, 32, 16),
                                               (3, 2, 1, 16, 16, 16), (7, 0, 2, 128, 0, 16), (6, 5, 1, 240, 80, 32),
                                               (2000, 2, 1, 128, 128, 16)])
def test_rope_append(T, Hq, Hk, D, R, page, interleaved, kind):
    _say("append", T, Hq, Hk, D, R, page, interleaved, kind)
    g = _gen(T + Hq + D)
    rows = _randn((T, (Hq + 2 * Hk) * D + 8), g, 2.0)
    q = rows[:, : Hq * D].view(T, Hq, D) if Hq else None
    k = rows[:, Hq * D:(Hq + Hk) * D].view(T, Hk, D)
    v = rows[:, (Hq + Hk) * D:(Hq + 2 * Hk) * D].view(T, Hk, D)
    P = 500
    cos, sin = _tables(P, R) if R else (None, None)
    pos = torch.randint(0, P, (T,), generator=g, device="cuda", dtype=torch.int32)
    pages = -(-T // page) + 2
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:T]
    kc, vc, ks, vs = _cache(pages, Hk, page, D, kind)
    if T > 3:
        slots[1], slots[2] = -1, pages * page          # padding, and past the cache
        k[3, 0] = 0                                     # a head of zeros
    got = jb.jq_rope_append(q, k, v, pos, cos, sin, slots, kc, vc, ks, vs, interleaved=interleaved)
    turn = (lambda x: ref.rotate(x, pos, cos, sin, interleaved)) if R else (lambda x: (x.double(), 0 * x.double()))
    if Hq:
        _within(got, *turn(q), "q")
    live = (slots >= 0) & (slots < pages * page)
    at = (slots[live] // page, slice(None), slots[live] % page)
    untouched = torch.ones((pages, page), dtype=torch.bool, device="cuda")
    untouched[at[0], at[2]] = False
    for name, cache, scale, (want, bound) in (("k", kc, ks, turn(k)), ("v", vc, vs, (v.double(), 0 * v.double()))):
        want, bound = want[live], bound[live]
        bytes_at = cache.view(torch.uint8 if kind == "fp8" else torch.int16)
        if kind == "bf16":
            _within(cache[at], want, bound, name)
        else:
            s = ref.fp8_scale(want.abs().amax(2))
            assert bool(((scale[at].double() - s).abs() <= 1e-5 * s).all()), name
            ref.check_fp8_values(bytes_at[at].view(E4M3), scale[at].double()[..., None].expand(want.shape), want)
            assert bool((scale.transpose(1, 2)[untouched] == 5.0).all())
        first = _cache(1, 1, 16, D, kind)[0].view(bytes_at.dtype).flatten()[0]
        assert bool((bytes_at.transpose(1, 2)[untouched] == first).all()), f"{name}: written outside the slots"


def test_rope_append_in_place_and_bad_positions():
    _say("append in place")
    g = _gen(8)
    T, Hq, Hk, D = 6, 4, 2, 64
    q, k, v = _randn((T, Hq, D), g), _randn((T, Hk, D), g), _randn((T, Hk, D), g)
    cos, sin = _tables(10, 32)
    pos = torch.tensor([0, 9, 10, -1, 2 ** 31 - 1, 3], dtype=torch.int32, device="cuda")
    slots = torch.arange(T, device="cuda")
    kc, vc, _, _ = _cache(2, Hk, 16, D, "bf16")
    out = jb.jq_rope_append(q, k, v, pos, cos, sin, slots, kc, vc)
    want, bound = ref.rotate(q, pos, cos, sin, False)
    _within(out, want, bound, "q")
    bad = [2, 3, 4]
    assert bool(out[bad, :, :32].isnan().all()) and not bool(out[bad, :, 32:].isnan().any())
    assert torch.equal(vc[0, :, :T].transpose(0, 1), v)
    again = jb.jq_rope_append(q, k, v, pos, cos, sin, slots, kc, vc, q_out=q)
    assert again.data_ptr() == q.data_ptr()
    assert torch.equal(q.view(torch.int16), out.view(torch.int16))


# ---------------------------------------------------------------------------
# paged attention


def _filled(lens, Hk, D, page, kind, seed, spare=3):
    """Caches with NaN wherever no sequence has a token, a shuffled page table, and the scales."""
    g = _gen(seed)
    need = [max(0, -(-n // page)) for n in lens]
    pages = sum(need) + spare
    cols = max(max(need), 1)
    order = torch.randperm(pages, generator=g, device="cuda")
    table = torch.full((len(lens), cols), -7, dtype=torch.int32, device="cuda")  # entries past a sequence are not read
    used = torch.zeros((pages, page), dtype=torch.bool, device="cuda")
    at = 0
    for b, n in enumerate(lens):
        mine = order[at: at + need[b]]
        at += need[b]
        table[b, : need[b]] = mine.int()
        for i, p in enumerate(mine.tolist()):
            used[p, : min(page, n - i * page)] = True
    out = []
    for _ in range(2):
        x = _randn((pages, Hk, page, D), g)
        if kind == "fp8":
            s = x.abs().amax(-1).float() / 448
            x = (x.float() / s[..., None]).to(E4M3)
            bits = x.view(torch.uint8)
            bits.transpose(1, 2)[~used] = 0x7F
            s.transpose(1, 2)[~used] = math.nan
            out.append((x, s))
        else:
            x.transpose(1, 2)[~used] = math.nan
            out.append((x, None))
    (kc, ks), (vc, vs) = out
    return kc, vc, ks, vs, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), g


def _attend_and_check(q, kc, vc, ks, vs, table, lens, **kw):
    causal = kw.get("causal", True)
    lse = torch.full(q.shape[:3], 9.0, device="cuda")
    out = jb.jq_paged_attention(q, kc, vc, table, lens, k_scale=ks, v_scale=vs, lse=lse, **kw)
    want, wlse, bound = ref.attention(q, kc, vc, table, lens.clamp(0, kw.get("max_len") or 1 << 30), ks, vs,
                                      kw.get("sm_scale"), causal)
    _within(out, want, bound, "out")
    empty = torch.isinf(wlse)
    assert torch.equal(torch.isinf(lse), empty)
    assert bool(((lse.double() - wlse)[~empty].abs() <= 1e-4 * (1 + wlse[~empty].abs())).all()), "lse"
    assert not bool(out[empty].any()), "a query that sees nothing gives zeros"
    return out


LENS = {"one": [1], "few": [0, 1, 2, 15, 16, 17, 31, 32, 33, 0, 63, 64, 65, 127, 128, 129, 200], "long": [3001, 5, 0, 4097]}


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("lens", list(LENS))
@pytest.mark.parametrize("Hq,Hk,D,page", [(1, 1, 64, 16), (8, 8, 128, 16), (32, 8, 128, 64), (7, 1, 256, 32), (28, 4, 64, 128),
                                          (20, 1, 128, 16), (40, 1, 256, 16), (70, 2, 64, 256)])
def test_attention_one_token(Hq, Hk, D, page, lens, kind):
    _say("attend", Hq, Hk, D, page, lens, kind)
    kc, vc, ks, vs, table, ln, g = _filled(LENS[lens], Hk, D, page, kind, Hq + D)
    q = _randn((len(LENS[lens]), 1, Hq, D), g, 1.5)
    out = _attend_and_check(q, kc, vc, ks, vs, table, ln)
    assert torch.equal(out, jb.jq_paged_attention(q, kc, vc, table, ln, k_scale=ks, v_scale=vs)), "two calls differ"


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("Tq,Hq,Hk,D", [(2, 4, 4, 128), (5, 6, 2, 64), (33, 2, 1, 128), (64, 4, 4, 128), (7, 8, 1, 256),
                                         (65, 1, 1, 64), (40, 3, 1, 256)])
def test_attention_several_tokens(Tq, Hq, Hk, D, causal, kind):
    """Several new tokens; sequences shorter than them leave causal queries with nothing to see."""
    lens = [Tq, Tq + 1, 0, 1, Tq // 2, Tq + 100, 700]
    _say("attend", Tq, Hq, Hk, D, causal, kind)
    kc, vc, ks, vs, table, ln, g = _filled(lens, Hk, D, 16, kind, Tq + D)
    q = _randn((len(lens), Tq, Hq, D), g, 1.5)
    _attend_and_check(q, kc, vc, ks, vs, table, ln, causal=causal)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("Tq,Hq,Hk,D,lens", [(20, 2, 2, 128, [5000, 1, 2600]), (17, 2, 1, 64, [4099, 0, 130, 3000]),
                                             (9, 4, 2, 256, [2500, 1300])])
def test_attention_several_tokens_of_long_caches(Tq, Hq, Hk, D, lens, kind):
    """Many columns over key axes that are cut into parts, most of which a short sequence does not have."""
    _say("attend long", Tq, Hq, Hk, D, kind)
    kc, vc, ks, vs, table, ln, g = _filled(lens, Hk, D, 32, kind, Tq + D)
    q = _randn((len(lens), Tq, Hq, D), g, 1.5)
    out = _attend_and_check(q, kc, vc, ks, vs, table, ln)
    assert torch.equal(out, jb.jq_paged_attention(q, kc, vc, table, ln, k_scale=ks, v_scale=vs)), "two calls differ"


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("Tq", [1, 24])
@pytest.mark.parametrize("rate", [0.02, 0.3, -0.3])
def test_attention_scores_that_climb(Tq, rate, kind):
    """Scores that rise (or fall) along the keys, a little or much within a step: the running maximum keeps up."""
    _say("attend climb", Tq, rate, kind)
    lens = [700, 333]
    kc, vc, ks, vs, table, ln, g = _filled(lens, 2, 64, 16, kind, 17)
    q = 1 + _randn((2, Tq, 4, 64), g, 0.1)
    for b, n in enumerate(lens):
        for t in range(n):
            row = kc[table[b, t // 16], :, t % 16]
            row[:] = (rate * t + row.float() * 0.01).to(row.dtype) if kind == "bf16" else torch.ones_like(row.float()).to(row.dtype)
            if kind == "fp8":
                ks[table[b, t // 16], :, t % 16] = rate * t
    _attend_and_check(q, kc, vc, ks, vs, table, ln, causal=False)


def test_attention_scale_peaks_and_bounds():
    _say("attend scale")
    lens = [500, 70, 1]
    kc, vc, ks, vs, table, ln, g = _filled(lens, 2, 128, 16, "bf16", 11)
    q = _randn((3, 1, 4, 128), g, 20.0)                    # scores of hundreds: one token takes all
    _attend_and_check(q, kc, vc, ks, vs, table, ln)
    _attend_and_check(q, kc, vc, ks, vs, table, ln, sm_scale=0.0)
    _attend_and_check(q, kc, vc, ks, vs, table, ln, sm_scale=-0.3)
    # lengths beyond max_len count as max_len, negative ones as 0
    _attend_and_check(q, kc, vc, ks, vs, table, ln, max_len=64)
    ln2 = torch.tensor([500, -5, 1], dtype=torch.int32, device="cuda")
    _attend_and_check(q, kc, vc, ks, vs, table, ln2)
    ln3 = torch.tensor([2 ** 31 - 1, 70, -2 ** 31], dtype=torch.int32, device="cuda")
    a = jb.jq_paged_attention(q, kc, vc, table, ln3, max_len=500)
    assert torch.equal(a[:2], jb.jq_paged_attention(q, kc, vc, table, ln, max_len=500)[:2]) and not bool(a[2].any())


@pytest.mark.parametrize("max_len", [None, 2000])
def test_attention_pages_outside_the_cache(max_len):
    """A page number that is none makes its own sequence NaN, and no other."""
    _say("attend bad pages", max_len)
    lens = [100, 2000, 90]
    kc, vc, ks, vs, table, ln, g = _filled(lens, 2, 128, 16, "bf16", 12)
    q = _randn((3, 1, 4, 128), g)
    good = jb.jq_paged_attention(q, kc, vc, table, ln, max_len=max_len)
    for bad in (-1, kc.shape[0], 2 ** 31 - 1, -2 ** 31):
        t = table.clone()
        t[1, 77] = bad
        lse = torch.zeros((3, 1, 4), device="cuda")
        out = jb.jq_paged_attention(q, kc, vc, t, ln, max_len=max_len, lse=lse)
        assert bool(out[1].isnan().all()) and bool(lse[1].isnan().all())
        assert torch.equal(out[[0, 2]], good[[0, 2]])


def test_attention_not_finite():
    """A NaN among the cached rows or queries shows in the heads and sequences that see it alone."""
    _say("attend not finite")
    lens = [300, 40, 60]
    kc, vc, ks, vs, table, ln, g = _filled(lens, 2, 64, 16, "bf16", 13)
    q = _randn((3, 1, 8, 64), g)
    good = jb.jq_paged_attention(q, kc, vc, table, ln)
    kc[table[0, 3], 1, 4, 9] = math.nan
    vc[table[1, 0], 0, 2, 5] = math.inf
    out = jb.jq_paged_attention(q, kc, vc, table, ln)
    assert bool(out[0, 0, 4:].isnan().all()) and torch.equal(out[0, 0, :4], good[0, 0, :4])
    assert bool((out[1, 0, :4, 5] == math.inf).all()) and torch.equal(out[1, 0, 4:], good[1, 0, 4:])
    assert torch.equal(out[2], good[2])


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_cache_beyond_32_bits(kind):
    """Offsets in the cache that pass 32 bits, in append and attention."""
    _say("large cache", kind)
    Hk, page, D = 8, 64, 128
    pages = (1 << 33) // (Hk * page * D * (2 if kind == "bf16" else 1)) + 9      # over 8 GiB
    g = _gen(14)
    dt = torch.bfloat16 if kind == "bf16" else E4M3
    kc, vc = (torch.empty((pages, Hk, page, D), dtype=dt, device="cuda") for _ in range(2))
    ks, vs = ((torch.empty((pages, Hk, page), device="cuda") if kind == "fp8" else None) for _ in range(2))
    n = 200
    table = torch.tensor([[pages - 1, 2, pages // 2 + 5, pages - 7]], dtype=torch.int32, device="cuda")
    t = torch.arange(n, device="cuda")
    slots = table[0].long()[t // page] * page + t % page
    k, v, q = _randn((n, Hk, D), g), _randn((n, Hk, D), g), _randn((1, 1, 16, D), g)
    cos, sin = _tables(n, D)
    jb.jq_rope_append(None, k, v, t.int(), cos, sin, slots, kc, vc, ks, vs)
    want, bound = ref.rotate(k, t, cos, sin, False)
    if kind == "bf16":
        _within(kc[slots // page, :, slots % page], want, bound, "k")
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    small = [x[table[0].long()].contiguous() if x.dtype != E4M3 else x.view(torch.uint8)[table[0].long()].view(E4M3)
             for x in (kc, vc)]
    scales = [None if x is None else x[table[0].long()] for x in (ks, vs)]
    plain = torch.arange(4, dtype=torch.int32, device="cuda")[None]
    a = jb.jq_paged_attention(q, kc, vc, table, lens, k_scale=ks, v_scale=vs)
    b = _attend_and_check(q, *small, *scales, plain, lens)
    assert torch.equal(a, b)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("Tq,Hq,Hk,D", [(2, 2, 2, 64), (16, 1, 1, 128), (4, 8, 2, 256), (4, 2, 1, 128), (17, 2, 2, 64),
                                         (40, 3, 1, 128), (64, 2, 2, 256), (33, 2, 1, 128)])
def test_attention_not_finite_where_some_see_it(Tq, Hq, Hk, D, kind):
    """Values that are infinite or NaN reach the causal queries that see their token, and no other."""
    lens = [Tq + 1, 130, 700, Tq, Tq // 2, 257 + Tq]
    _say("attend not finite, causal", Tq, Hq, Hk, D, kind)
    kc, vc, ks, vs, table, ln, g = _filled(lens, Hk, D, 16, kind, 3 * Tq + D)
    q = _randn((len(lens), Tq, Hq, D), g, 1.5)
    good = _attend_and_check(q, kc, vc, ks, vs, table, ln)
    reached = torch.zeros(good.shape, dtype=torch.bool, device="cuda")
    for b, n in enumerate(lens):
        for back, h, d in ((0, 0, 3), (Tq // 2, Hk - 1, D - 1)):
            t = n - 1 - back                                   # seen from query Tq - 1 - back on
            if t < 0:
                continue
            page, place = int(table[b, t // 16]), t % 16
            mine = reached[b, Tq - 1 - back:, h * (Hq // Hk):(h + 1) * (Hq // Hk)]
            if kind == "bf16":
                vc[page, h, place, d] = math.nan if back else math.inf
                mine[..., d] = True
            elif back:
                vc.view(torch.uint8)[page, h, place, d] = 0xFF  # the code of NaN
                mine[..., d] = True
            else:
                vs[page, h, place] = math.nan                  # of a whole row
                mine[:] = True
    out = jb.jq_paged_attention(q, kc, vc, table, ln, k_scale=ks, v_scale=vs)
    assert torch.equal(out[~reached], good[~reached])
    assert not bool(torch.isfinite(out[reached]).any())


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("Tq,Hq,Hk,D", [(1, 8, 2, 128), (1, 4, 4, 64), (2, 8, 1, 256), (64, 2, 2, 128)])
def test_attention_error_is_the_outputs_rounding(Tq, Hq, Hk, D, kind):
    """Weights have 16 bits in their product, so that the outputs' rounding to 8 is the only one that shows: the rms error
    is that of the rounded 64-bit result, within a tenth."""
    _say("attend error", Tq, Hq, Hk, D, kind)
    lens = [2000, 333]
    kc, vc, ks, vs, table, ln, g = _filled(lens, Hk, D, 16, kind, 23)
    q = _randn((2, Tq, Hq, D), g, 1.5)
    want = ref.attention(q, kc, vc, table, ln, ks, vs)[0]
    out = jb.jq_paged_attention(q, kc, vc, table, ln, k_scale=ks, v_scale=vs).double()
    assert float((out - want).norm()) <= 1.1 * float((want.bfloat16().double() - want).norm())


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n", [1, 16, 17, 33, 40, 63, 65, 300])
def test_attention_infinite_values(n, D):
    """An infinity in the first or last cached value is an infinity of that output element, and of no other."""
    _say("attend infinite", n, D)
    kc, vc, ks, vs, table, ln, g = _filled([n], 1, D, 16, "bf16", n + D)
    q = _randn((1, 1, 3, D), g)
    good = jb.jq_paged_attention(q, kc, vc, table, ln)
    for t in {0, n - 1}:
        v = vc.clone()
        v[table[0, t // 16], 0, t % 16, 7] = -math.inf
        out = jb.jq_paged_attention(q, kc, v, table, ln)
        assert bool((out[..., 7] == -math.inf).all())
        keep = torch.arange(D, device="cuda") != 7
        assert torch.equal(out[..., keep], good[..., keep])


# ---------------------------------------------------------------------------
# streams and graphs


def test_given_stream_owns_what_a_call_allocates():
    """Outputs and workspaces of a call with a stream come from that stream's memory, so nobody else gets them early."""
    _say("given stream")
    g = _gen(18)
    x = _randn((333, 1024), g)
    wq, ws = jb.jq_pack_weight_fp8(_randn((96, 1024), g, 0.05))
    kc, vc, ks, vs, table, ln, _ = _filled([3000, 7], 2, 64, 16, "bf16", 19)
    q = _randn((2, 1, 4, 64), g)
    assert jb.jq_paged_attention_workspace_bytes(2, 1, 4, 2, 64, 3008) > 0
    want = jb.jq_fp8_linear(x, wq, ws), jb.jq_paged_attention(q, kc, vc, table, ln)
    y, out = torch.empty_like(want[0]), torch.empty_like(want[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    torch.cuda.empty_cache()

    def owned():
        return sum(s["total_size"] for s in torch.cuda.memory_snapshot() if s["stream"] == side.cuda_stream)

    assert owned() == 0
    jb.jq_fp8_linear(x, wq, ws, y=y, stream=side)
    assert owned() > 0
    side.synchronize()
    torch.cuda.empty_cache()
    jb.jq_paged_attention(q, kc, vc, table, ln, out=out, stream=side)
    assert owned() > 0
    side.synchronize()
    assert torch.cuda.current_stream() != side
    assert torch.equal(y, want[0]) and torch.equal(out, want[1])
    norm = jb.jq_rmsnorm(x, x[0].contiguous(), stream=side)[0]
    side.synchronize()
    assert torch.equal(norm, jb.jq_rmsnorm(x, x[0].contiguous())[0])


def test_other_stream_and_graph():
    """The whole chain on another stream, and captured: each replay equals the eager result."""
    _say("stream and graph")
    g = _gen(15)
    T, Hq, Hk, D = 4, 8, 2, 64
    dim, F = Hq * D, 768
    x, r = _randn((T, dim), g), _randn((T, dim), g)
    w1, w2 = _randn((dim,), g) + 1, _randn((dim,), g) + 1
    wq, wqs = jb.jq_pack_weight_fp8(_randn(((Hq + 2 * Hk) * D, dim), g, 0.05))
    wf, wfs = jb.jq_pack_weight_fp8(_randn((F, dim), g, 0.05))
    cos, sin = _tables(600, D)
    lens = [500, 33, 64, 1]
    kc, vc, ks, vs, table, ln, _ = _filled(lens, Hk, D, 16, "fp8", 16)
    pos = (ln - 1).clone()
    slots = table.long().gather(1, (pos.long() // 16)[:, None])[:, 0] * 16 + pos.long() % 16

    def chain():
        q8, s8, h = jb.jq_rmsnorm(x, w1, residual=r, out="fp8")
        qkv = jb.jq_fp8_gemm(q8, s8, wq, wqs)
        q, k, v = qkv.split((Hq * D, Hk * D, Hk * D), 1)
        q = jb.jq_rope_append(q.view(T, Hq, D), k.view(T, Hk, D), v.view(T, Hk, D), pos, cos, sin, slots, kc, vc, ks, vs)
        o = jb.jq_paged_attention(q.view(T, 1, Hq, D), kc, vc, table, ln, k_scale=ks, v_scale=vs, max_len=512)
        n, s = jb.jq_rmsnorm(o.view(T, dim), w2, residual=h, out="fp8")[:2]
        return jb.jq_fp8_gemm(n, s, wf, wfs)

    want = chain()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = chain()
    side.synchronize()
    assert torch.equal(want, other)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = chain()
    for i in range(4):
        x.copy_(_randn((T, dim), g))
        eager = chain().clone()
        torch.cuda.synchronize()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager), i
