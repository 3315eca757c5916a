"""Attention of packed prompts and of chunks over the paged cache (include/jq_block.h), against 64 bits."""

import itertools

import pytest
import torch

from paper_2609_33601_amd import jq, jq_block as jb
from tests import block_reference as block
from tests import prompt_reference as ref

pytestmark = pytest.mark.gpu

DEV = "cuda"


def starts(lens, first=0):
    return torch.tensor([first] + [first + n for n in itertools.accumulate(lens)], dtype=torch.int32, device=DEV)


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def heads(tokens, counts, D, g):
    """Views of one fused projection's rows."""
    x = torch.randn((tokens, sum(counts) * D), generator=g, device=DEV).bfloat16()
    return [p.view(tokens, -1, D) for p in x.split([c * D for c in counts], dim=1)]


def check_all(out, lse, q, k, v, lens, klens, causal, sm_scale=None, first=0):
    a, b = first, 0 if klens is not lens else first
    for n, m in zip(lens, klens):
        ref.check_attention(out[a:a + n], None if lse is None else lse[a:a + n], q[a:a + n], k[b:b + m], v[b:b + m],
                            causal, sm_scale)
        a, b = a + n, b + m


LENS = [[1], [2, 1], [3], [64], [65, 63], [127, 128, 129], [300, 0, 17], [0, 0, 1, 0], [31, 33, 1, 256, 2]]


@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
@pytest.mark.parametrize("Hq,Hk", [(4, 4), (8, 2), (7, 1)], ids=str)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("lens", LENS, ids=str)
def test_packed(lens, D, Hq, Hk, causal):
    q, k, v = heads(sum(lens), (Hq, Hk, Hk), D, gen(sum(lens) + D + Hq))
    lse = torch.empty((sum(lens), Hq), device=DEV)
    out = jb.jq_prompt_attention(q, k, v, starts(lens), causal=causal, lse=lse)
    check_all(out, lse, q, k, v, lens, lens, causal)


@pytest.mark.parametrize("lens,klens", [([5, 40, 3], [70, 3, 0]), ([1, 1, 1], [1000, 1, 64]), ([130], [2500]),
                                        ([200, 9], [199, 700])], ids=str)
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_keys_apart(lens, klens, D, causal):
    """Other numbers of keys than queries: parts of a long key axis, queries that see nothing."""
    Hq, Hk, g = 6, 2, gen(D + sum(klens))
    q, = heads(sum(lens), (Hq,), D, g)
    k, v = heads(sum(klens), (Hk, Hk), D, g)
    lse = torch.empty((sum(lens), Hq), device=DEV)
    out = jb.jq_prompt_attention(q, k, v, starts(lens), starts(klens), causal=causal, lse=lse)
    check_all(out, lse, q, k, v, lens, klens, causal)


@pytest.mark.parametrize("lens,klens", [([16, 16, 3, 16], [4100, 3000, 0, 2900]), ([1] * 6, [2000, 1, 6500, 63, 64, 1025]),
                                        ([40, 0, 2], [3001, 500, 1501])], ids=str)
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_keys_apart_in_parts(lens, klens, D, causal):
    """Several sequences, whose key axes are cut, shorter ones into fewer parts than the longest could have."""
    Hq, Hk, g = 6, 2, gen(2 * D + sum(klens))
    assert jb.jq_prompt_attention_workspace_bytes(sum(lens), sum(klens), len(lens), Hq, Hk, D) > 0
    q, = heads(sum(lens), (Hq,), D, g)
    k, v = heads(sum(klens), (Hk, Hk), D, g)
    lse = torch.empty((sum(lens), Hq), device=DEV)
    out = jb.jq_prompt_attention(q, k, v, starts(lens), starts(klens), causal=causal, lse=lse)
    check_all(out, lse, q, k, v, lens, klens, causal)


@pytest.mark.parametrize("D,Hq,Hk,lens", [(128, 32, 32, [1500, 600]), (128, 32, 8, [2000, 1, 70]), (64, 40, 8, [1700, 130]),
                                          (256, 16, 16, [900, 77])], ids=str)
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
def test_many_columns(D, Hq, Hk, lens, causal):
    """Enough tiles for the widest blocks."""
    q, k, v = heads(sum(lens), (Hq, Hk, Hk), D, gen(D + Hq))
    out = jb.jq_prompt_attention(q, k, v, starts(lens), causal=causal)
    check_all(out, None, q, k, v, lens, lens, causal)


@pytest.mark.parametrize("n", [64, 65, 200, 257, 700])
def test_many_sequences(n):
    lens = [(7 * i) % 23 for i in range(n)]
    q, k, v = heads(sum(lens), (4, 2, 2), 64, gen(n))
    out = jb.jq_prompt_attention(q, k, v, starts(lens))
    check_all(out, None, q, k, v, lens, lens, True)


@pytest.mark.parametrize("paged", [False, True], ids=["own", "cache"])
@pytest.mark.parametrize("n,first", [(65, 0), (129, 5), (4096, 0), (4097, 40), (9000, 1)], ids=str)
def test_every_sequence_is_found(n, first, paged):
    """Empty ones, full tiles, more than a tile, and rows before and behind; a sample against 64 bits."""
    lens = [(0, 1, 3, 0, 64, 1, 0, 2, 33)[(i + i // 9) % 9] if i % 500 != 77 else 300 for i in range(n)]
    T, g = sum(lens) + first + 9, gen(n)
    out = torch.full((T, 6, 64), float("nan"), device=DEV).bfloat16()
    q, k, v = heads(T, (6, 2, 2), 64, g)
    s = starts(lens, first)
    if paged:
        kv, scales, table = cache_of([m + i % 70 for i, m in enumerate(lens)], 2, 64, 16, "bf16", g)
        klens = torch.tensor([m + i % 70 for i, m in enumerate(lens)], dtype=torch.int32, device=DEV)
        jb.jq_chunk_attention(q, *kv, table, s, klens, out=out)
    else:
        jb.jq_prompt_attention(q, k, v, s, out=out)
    assert out[:first].isnan().all() and out[T - 9:].isnan().all() and not out[first:T - 9].isnan().any()
    at = s.tolist()
    for b in {*range(0, n, max(1, n // 60)), *range(n - 5, n)} | {b for b in range(n) if lens[b] == 300}:
        i, j = at[b], at[b + 1]
        if j > i:
            kb, vb = rows_of(kv, scales, table, b, lens[b] + b % 70) if paged else (k[i:j], v[i:j])
            ref.check_attention(out[i:j], None, q[i:j], kb, vb, True, None)


@pytest.mark.parametrize("at", ["first", "last", "apart"])
@pytest.mark.parametrize("n", [100, 5000, 65536])
def test_few_tokens_of_many_sequences(n, at):
    """A padded batch: most sequences are empty, there are more of them than tokens."""
    g, some = gen(n), [5, 1, 40, 2, 1]
    where = {"first": range(5), "last": range(n - 5, n), "apart": [0, 7, n // 2, n // 2 + 1, n - 2]}[at]
    lens = [0] * n
    for b, m in zip(where, some):
        lens[b] = m
    q, k, v = heads(50, (6, 2, 2), 64, g)
    out = torch.full((50, 6, 64), float("nan"), device=DEV).bfloat16()
    jb.jq_prompt_attention(q, k, v, starts(lens), out=out)
    check_all(out[:49], None, q, k, v, some, some, True)
    assert out[49:].isnan().all()


@pytest.mark.parametrize("klen", [0, 3000], ids=["own", "long"])
def test_rows_of_no_sequence_stay(klen):
    """Rows before the first and behind the last sequence, with one part and with several."""
    lens, g = [20, 40], gen(3)
    q, = heads(90, (4,), 64, g)
    k, v = heads(klen or 90, (2, 2), 64, g)
    out, lse = torch.full((90, 4, 64), 7.0, device=DEV).bfloat16(), torch.full((90, 4), 7.0, device=DEV)
    ks = starts([klen // 3, klen - klen // 3]) if klen else None
    r = jb.jq_prompt_attention(q, k, v, starts(lens, 11), ks, out=out, lse=lse)
    assert r.data_ptr() == out.data_ptr()
    for t in (out[:11], out[71:], lse[:11], lse[71:]):
        assert torch.all(t == 7)
    check_all(out, lse, q, k, v, lens, [klen // 3, klen - klen // 3] if klen else lens, True, first=11)


@pytest.mark.parametrize("bad", [[0, 50, 20, 90], [-5, 30, 1000, 2000], [90, 0, 0, 0], [50, 40, 30, 20]], ids=str)
def test_bad_starts_touch_nothing_else(bad):
    q, k, v = heads(90, (4, 2, 2), 64, gen(4))
    whole = torch.full((90 + 64, 4, 64), 7.0, device=DEV).bfloat16()
    s = torch.tensor(bad, dtype=torch.int32, device=DEV)
    jb.jq_prompt_attention(q, k, v, s, out=whole[:90])
    torch.cuda.synchronize()
    assert torch.all(whole[90:] == 7)


@pytest.mark.parametrize("sm_scale", [-0.3, 0.0, 1.5])
@pytest.mark.parametrize("D", [64, 128])
def test_scales(D, sm_scale):
    lens = [100, 3]
    q, k, v = heads(103, (4, 2, 2), D, gen(5))
    lse = torch.empty((103, 4), device=DEV)
    out = jb.jq_prompt_attention(q, k, v, starts(lens), sm_scale=sm_scale, lse=lse)
    check_all(out, lse, q, k, v, lens, lens, True, sm_scale)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_climbing_scores(D):
    """The running maximum moves at every step."""
    n, g = 400, gen(6)
    q, k, v = (t.clone() for t in heads(n, (2, 2, 2), D, g))
    k *= torch.linspace(0.0, 12.0, n, device=DEV)[:, None, None]
    lse = torch.empty((n, 2), device=DEV)
    for causal in (True, False):
        out = jb.jq_prompt_attention(q, k, v, starts([n]), causal=causal, lse=lse)
        check_all(out, lse, q, k, v, [n], [n], causal)


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")], ids=str)
@pytest.mark.parametrize("token", [0, 37, 64, 130, 255])
@pytest.mark.parametrize("D,Hq,Hk", [(64, 4, 4), (128, 8, 2), (256, 2, 1)], ids=str)
def test_values_reach_only_queries_that_see_them(D, Hq, Hk, token, value):
    n = 256
    q, k, v = heads(n, (Hq, Hk, Hk), D, gen(7))
    v = v.clone()
    v[token, Hk - 1, 5] = value
    out = jb.jq_prompt_attention(q, k, v, starts([n]))
    check_all(out, None, q, k, v, [n], [n], True)


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")], ids=str)
def test_keys_reach_only_queries_that_see_them(value):
    n, D = 200, 128
    q, k, v = heads(n, (4, 2, 2), D, gen(8))
    k = k.clone()
    k[77, 1, 3] = value
    out = jb.jq_prompt_attention(q, k, v, starts([n]))
    clean = jb.jq_prompt_attention(q, heads(n, (4, 2, 2), D, gen(8))[1], v, starts([n]))
    assert torch.equal(out[:77], clean[:77]) and torch.equal(out[:, :2], clean[:, :2])
    z = q[77:, 2:].float()[..., 3] * value  # the score's sign decides between no weight and NaN
    nan = out[77:, 2:].isnan()
    assert torch.equal(nan.all(-1), ~(z == -float("inf"))) and torch.equal(nan.any(-1), nan.all(-1))


def test_other_sequences_values_do_not_reach():
    """What follows a sequence in memory counts for nothing, whatever it is."""
    lens = [37, 50, 21]
    q, k, v = heads(108, (4, 2, 2), 128, gen(9))
    k, v = k.clone(), v.clone()
    k[37:87] = float("nan")
    v[37:87] = float("inf")
    for causal in (True, False):
        out = jb.jq_prompt_attention(q, k, v, starts(lens), causal=causal)
        for a, b in ((0, 37), (87, 108)):
            ref.check_attention(out[a:b], None, q[a:b], k[a:b], v[a:b], causal)


def test_every_key_counts_once():
    """Equal scores and one-hot values: each key's weight is 1 / (keys seen), exactly up to the roundings."""
    D = 128
    for n in (128, 200):
        q = torch.zeros((n, 1, D), device=DEV).bfloat16()
        k = torch.zeros_like(q)
        for base in range(0, n, D):
            v = torch.zeros((n, 1, D), device=DEV)
            i = torch.arange(base, min(n, base + D), device=DEV)
            v[i, 0, i - base] = 1.0
            out = jb.jq_prompt_attention(q, k, v.bfloat16(), starts([n]))[:, 0].double()
            want = torch.zeros((n, D), dtype=torch.float64, device=DEV)
            t = torch.arange(n, device=DEV)
            want[:, : len(i)] = torch.where(t[:, None] >= i[None], 1.0 / (t[:, None] + 1), 0.0)
            assert torch.all((out - want).abs() <= 2.0 ** -8 * 1.01 * want)


# ---------------------------------------------------------------------------
# chunks over the cache


def cache_of(lens, Hk, D, page, kind, g, spare=3):
    need = [-(-max(n, 0) // page) for n in lens]
    pages = sum(need) + spare
    cols = max(max(need), 1) + 1
    table = torch.full((len(lens), cols), 1 << 30, dtype=torch.int32, device=DEV)  # entries past a length are not read
    order = torch.randperm(pages, generator=g, device=DEV).int()
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    x = [torch.randn((pages, Hk, page, D), generator=g, device=DEV) for _ in range(2)]
    if kind == "bf16":
        return [t.bfloat16() for t in x], [None, None], table
    s = [torch.rand((pages, Hk, page), generator=g, device=DEV) * 0.01 + 0.001 for _ in x]
    return [(t * 60).clamp(-448, 448).to(torch.float8_e4m3fn) for t in x], s, table


def rows_of(kv, scales, table, b, n):
    return [block.cached(c, s, table[b], n).transpose(0, 1) for c, s in zip(kv, scales)]


def check_chunk(out, lse, q, kv, scales, table, new, lens, causal, sm_scale=None):
    at = 0
    for b, (a, n) in enumerate(zip(new, lens)):
        n = max(n, 0)
        k, v = rows_of(kv, scales, table, b, n) if n else (q.new_zeros((0, kv[0].shape[1], q.shape[2])),) * 2
        ref.check_attention(out[at:at + a], None if lse is None else lse[at:at + a], q[at:at + a], k, v, causal, sm_scale)
        at += a


CHUNKS = [([1], [1]), ([1, 1, 1], [5, 700, 64]), ([16], [2080]), ([40, 1, 3], [40, 1, 900]), ([0, 7, 0], [33, 20, 0]),
          ([130, 1], [131, 4097]), ([9], [3]), ([5, 6], [-1, 6])]


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
@pytest.mark.parametrize("D,Hq,Hk,page", [(64, 8, 2, 16), (128, 8, 8, 16), (128, 12, 2, 64), (256, 4, 1, 32)], ids=str)
@pytest.mark.parametrize("new,lens", CHUNKS, ids=str)
def test_chunk(new, lens, D, Hq, Hk, page, causal, kind):
    g = gen(D + sum(lens) + page)
    kv, scales, table = cache_of(lens, Hk, D, page, kind, g)
    q = torch.randn((sum(new), Hq, D), generator=g, device=DEV).bfloat16()
    lse = torch.empty((sum(new), Hq), device=DEV)
    out = jb.jq_chunk_attention(q, *kv, table, starts(new), torch.tensor(lens, dtype=torch.int32, device=DEV), *scales,
                                max_len=max(max(lens), 1), causal=causal, lse=lse)
    check_chunk(out, lse, q, kv, scales, table, new, lens, causal)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("D,Hq,Hk", [(64, 32, 8), (128, 32, 8), (256, 16, 4)], ids=str)
def test_chunk_many_columns(D, Hq, Hk, kind):
    new, lens, g = [1200, 1, 900], [2000, 333, 900], gen(D)
    kv, scales, table = cache_of(lens, Hk, D, 32, kind, g)
    q, = heads(sum(new), (Hq,), D, g)
    out = jb.jq_chunk_attention(q, *kv, table, starts(new), torch.tensor(lens, dtype=torch.int32, device=DEV), *scales)
    check_chunk(out, None, q, kv, scales, table, new, lens, True)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("limit", [2100, 9000, 1 << 20])
def test_chunk_under_a_long_limit(limit, D, kind):
    """Each sequence is cut by its own length: ends of parts, and a last part of one key."""
    new, lens, g = [40, 1, 3, 64, 1, 20], [513, 1025, 5, 2049, 0, 1537], gen(limit + D)
    kv, scales, table = cache_of(lens, 2, D, 16, kind, g)
    wide = torch.full((6, -(-limit // 16)), 1 << 30, dtype=torch.int32, device=DEV)
    wide[:, : table.shape[1]] = table[:, : wide.shape[1]]
    q = torch.randn((sum(new), 8, D), generator=g, device=DEV).bfloat16()
    lse = torch.empty((sum(new), 8), device=DEV)
    out = jb.jq_chunk_attention(q, *kv, wide, starts(new), torch.tensor(lens, dtype=torch.int32, device=DEV), *scales,
                                max_len=limit, lse=lse)
    check_chunk(out, lse, q, kv, scales, table, new, lens, True)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_chunk_max_len_bounds_lengths(kind):
    g = gen(11)
    kv, scales, table = cache_of([500, 40], 2, 128, 16, kind, g)
    q = torch.randn((8, 4, 128), generator=g, device=DEV).bfloat16()
    lens = torch.tensor([500, 40], dtype=torch.int32, device=DEV)
    out = jb.jq_chunk_attention(q, *kv, table, starts([5, 3]), lens, *scales, max_len=300)
    check_chunk(out, None, q, kv, scales, table, [5, 3], [300, 40], True)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("length,place", [(60, 1), (2000, 100)], ids=["short", "parts"])
def test_chunk_bad_page_is_nan(length, place, kind):
    """A page outside the cache: NaN for its own sequence, nothing for the others."""
    g, lens, new = gen(12), [length, 50], [4, 6]
    kv, scales, table = cache_of(lens, 2, 64, 16, kind, g)
    q = torch.randn((10, 4, 64), generator=g, device=DEV).bfloat16()
    lens_t = torch.tensor(lens, dtype=torch.int32, device=DEV)
    for bad in (-1, kv[0].shape[0], 1 << 30):
        wrong = table.clone()
        wrong[0, place] = bad
        out = jb.jq_chunk_attention(q, *kv, wrong, starts(new), lens_t, *scales)
        assert out[:4].isnan().all()
        check_chunk(out[4:], None, q[4:], kv, scales, table[1:], new[1:], lens[1:], True)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("token", [3, 90, 127])
def test_chunk_values_reach_only_queries_that_see_them(token, kind):
    g, lens, new = gen(13), [128], [100]
    for what in ("value", "scale") if kind == "fp8" else ("value",):
        kv, scales, table = cache_of(lens, 2, 128, 16, kind, g)
        page, place = int(table[0, token // 16]), token % 16
        if what == "scale":
            scales[1][page, 1, place] = float("inf")
            kv[1].view(torch.uint8)[page, 1, place] = 0x38  # ones, so that no product is 0 times infinity
        elif kind == "fp8":
            kv[1].view(torch.uint8)[page, 1, place, 9] = 0x7F
        else:
            kv[1][page, 1, place, 9] = float("nan")
        q = torch.randn((100, 4, 128), generator=g, device=DEV).bfloat16()
        out = jb.jq_chunk_attention(q, *kv, table, starts(new), torch.tensor(lens, dtype=torch.int32, device=DEV), *scales)
        check_chunk(out, None, q, kv, scales, table, new, lens, True)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_chunk_places_past_the_end_count_for_nothing(kind):
    g, lens, new = gen(14), [35, 70], [20, 70]
    kv, scales, table = cache_of(lens, 2, 128, 16, kind, g)
    for b, n in enumerate(lens):
        page = int(table[b, n // 16])
        for c, s in zip(kv, scales):
            if kind == "fp8":
                c.view(torch.uint8)[page, :, n % 16:] = 0x7F
                s[page, :, n % 16:] = float("nan")
            else:
                c[page, :, n % 16:] = float("nan")
    q = torch.randn((90, 4, 128), generator=g, device=DEV).bfloat16()
    for causal in (True, False):
        out = jb.jq_chunk_attention(q, *kv, table, starts(new), torch.tensor(lens, dtype=torch.int32, device=DEV), *scales,
                                    causal=causal)
        check_chunk(out, None, q, kv, scales, table, new, lens, causal)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_chunk_agrees_with_paged_attention(kind):
    """Equal blocks, which jq_paged_attention takes too: both within their bounds of the same result."""
    B, n, lens, g = 3, 8, [300, 8, 77], gen(15)
    kv, scales, table = cache_of(lens, 2, 128, 16, kind, g)
    table = torch.where(table >= kv[0].shape[0], 0, table)
    q = torch.randn((B * n, 8, 128), generator=g, device=DEV).bfloat16()
    lens_t = torch.tensor(lens, dtype=torch.int32, device=DEV)
    a = jb.jq_chunk_attention(q, *kv, table, starts([n] * B), lens_t, *scales)
    b = jb.jq_paged_attention(q.view(B, n, 8, 128), *kv, table, lens_t, *scales).view(B * n, 8, 128)
    check_chunk(a, None, q, kv, scales, table, [n] * B, lens, True)
    check_chunk(b, None, q, kv, scales, table, [n] * B, lens, True)


# ---------------------------------------------------------------------------
# streams, graphs, buffers


def test_streams_graphs_and_buffers():
    g, lens, new = gen(16), [3000, 64], [30, 64]
    kv, scales, table = cache_of(lens, 2, 128, 16, "bf16", g)
    q, k, v = heads(94, (8, 2, 2), 128, g)
    s, lens_t = starts(new), torch.tensor(lens, dtype=torch.int32, device=DEV)
    ks = starts([60, 34])
    calls = {
        "chunk": lambda **kw: jb.jq_chunk_attention(q, *kv, table, s, lens_t, max_len=3000, **kw),
        "prompt": lambda **kw: jb.jq_prompt_attention(q, k, v, s, ks, **kw),
    }
    need = {"chunk": jb.jq_chunk_attention_workspace_bytes(94, 2, 8, 2, 128, 3000),
            "prompt": jb.jq_prompt_attention_workspace_bytes(94, 94, 2, 8, 2, 128)}
    assert need["chunk"] > 0
    for name, call in calls.items():
        want = call()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = call(stream=side)
        side.synchronize()
        assert torch.equal(got, want)
        out = torch.empty_like(want)
        ws = torch.empty((max(need[name], 1),), dtype=torch.uint8, device=DEV)
        assert torch.equal(call(out=out, workspace=ws), want) and torch.equal(out, want)
        if need[name]:
            with pytest.raises(jq.JQError):
                call(workspace=ws[: need[name] - 256])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = call()
        for _ in range(3):
            y.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, want)
            assert torch.equal(call(), want)


def test_the_same_call_gives_the_same_bits():
    q, k, v = heads(2000, (32, 8, 8), 128, gen(17))
    s = starts([1500, 500])
    a = jb.jq_prompt_attention(q, k, v, s)
    for _ in range(3):
        assert torch.equal(jb.jq_prompt_attention(q, k, v, s), a)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_chunk_pages_that_sequences_share(kind):
    """A common beginning, held once."""
    g, new, lens = gen(18), [40, 1, 7], [300, 290, 64]
    kv, scales, table = cache_of(lens, 2, 64, 16, kind, g)
    table[1, :16] = table[0, :16]
    table[2, :4] = table[0, 4]
    q = torch.randn((sum(new), 6, 64), generator=g, device=DEV).bfloat16()
    out = jb.jq_chunk_attention(q, *kv, table, starts(new), torch.tensor(lens, dtype=torch.int32, device=DEV), *scales)
    check_chunk(out, None, q, kv, scales, table, new, lens, True)


def test_a_graph_follows_its_starts_and_lengths():
    g, T, cap = gen(19), 96, 2048
    kv, scales, table = cache_of([cap] * 3, 2, 128, 16, "fp8", g)
    q = torch.randn((T, 8, 128), generator=g, device=DEV).bfloat16()
    s, lens = starts([1, 1, 1]), torch.tensor([1, 1, 1], dtype=torch.int32, device=DEV)
    out = torch.zeros_like(q)
    call = lambda: jb.jq_chunk_attention(q, *kv, table, s, lens, *scales, max_len=cap, out=out)
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for new, n in (([90, 1, 5], [90, 2048, 700]), ([0, 0, 3], [0, 5, 1999]), ([32, 32, 32], [1000, 31, 64])):
        s.copy_(starts(new))
        lens.copy_(torch.tensor(n, dtype=torch.int32))
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        check_chunk(out, None, q, kv, scales, table, new, n, True)
        assert (out[sum(new):] == 7).all()
        replayed = out.clone()
        call()
        assert torch.equal(out, replayed)
