"""The kernels that long prompts and long caches take, against 64 bits: tiles whose four waves have columns of their own
over many whole steps, tiles of 256 columns, key axes in parts; each with an infinity or NaN among the values of tokens
that only some of a tile's columns see.  Every test asserts the plan that its shape is meant to meet."""

import itertools
import math

import pytest
import torch

from paper_2609_33601_amd import jq_block as jb
from tests import block_reference as block
from tests import prompt_reference as ref
from tests.prompt_routes import Plan, plan

pytestmark = pytest.mark.gpu

DEV = "cuda"
INF, NAN = math.inf, math.nan


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def starts(lens):
    return i32([0, *itertools.accumulate(lens)])


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def heads(tokens, counts, D, g):
    """Views of one fused projection's rows."""
    x = torch.randn((tokens, sum(counts) * D), generator=g, device=DEV).bfloat16()
    return [p.view(tokens, -1, D) for p in x.split([c * D for c in counts], dim=1)]


def cache_of(lens, Hk, D, page, kind, g):
    """[k, v], [their scales], page table."""
    need = [-(-n // page) for n in lens]
    order = torch.randperm(sum(need) + 3, generator=g, device=DEV).int()
    table = torch.full((len(lens), max(need)), 1 << 30, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    x = [torch.randn((len(order), Hk, page, D), generator=g, device=DEV) for _ in range(2)]
    if kind == "bf16":
        return [t.bfloat16() for t in x], [None, None], table
    s = [torch.rand(t.shape[:3], generator=g, device=DEV) * 0.01 + 0.001 for t in x]
    return [(t * 60).clamp(-448, 448).to(torch.float8_e4m3fn) for t in x], s, table


def rows_of(kv, scales, table, b, n):
    return [block.cached(c, s, table[b], n).transpose(0, 1) for c, s in zip(kv, scales)]


class Case:
    """A call over own keys or a cache, and the 64-bit keys and values of each sequence."""

    def __init__(self, kind, new, total, Hq, Hk, D, seed, page=16):
        self.kind, self.new, self.total = kind, new, total
        self.shape, g = (Hq, Hk, D), gen(seed)
        self.q, = heads(sum(new), (Hq,), D, g)
        if kind == "own":
            self.k, self.v = (t.clone() for t in heads(sum(total), (Hk, Hk), D, g))
        else:
            self.kv, self.scales, self.table = cache_of(total, Hk, D, page, kind, g)

    def plan(self):
        return plan(sum(self.new), len(self.new), *self.shape, sum(self.total) if self.kind == "own" else max(self.total),
                    self.kind)

    def put(self, b, token, head, at, value):
        """A value of one of sequence b's tokens (for an 8-bit cache NaN, whatever is asked for)."""
        if self.kind == "own":
            self.v[sum(self.total[:b]) + token, head, at] = value
            return
        page = self.kv[1].shape[2]
        where = (int(self.table[b, token // page]), head, token % page, at)
        if self.kind == "fp8":
            self.kv[1].view(torch.uint8)[where] = 0x7F
        else:
            self.kv[1][where] = value

    def run(self, causal, table=None):
        out = torch.full((sum(self.new), self.shape[0], self.shape[2]), 7.0, device=DEV).bfloat16()
        lse = torch.full(out.shape[:2], 7.0, device=DEV)
        if self.kind == "own":
            jb.jq_prompt_attention(self.q, self.k, self.v, starts(self.new), starts(self.total), causal=causal, out=out, lse=lse)
        else:
            jb.jq_chunk_attention(self.q, *self.kv, self.table if table is None else table, starts(self.new),
                                  i32(self.total), *self.scales, max_len=max(self.total), causal=causal, out=out, lse=lse)
        return out, lse

    def check(self, out, lse, causal, sequences=None):
        a = k0 = 0
        for b, (n, m) in enumerate(zip(self.new, self.total)):
            if sequences is None or b in sequences:
                k, v = (self.k[k0:k0 + m], self.v[k0:k0 + m]) if self.kind == "own" else rows_of(self.kv, self.scales, self.table, b, m)
                ref.check_attention(out[a:a + n], lse[a:a + n], self.q[a:a + n], k, v, causal)
            a, k0 = a + n, k0 + m


FOUR_WAVES = [([1400], [1400], 32, 8, 128), ([1000, 400], [1290, 403], 28, 4, 128), ([1500, 100], [1500, 150], 12, 4, 256)]
WIDEST = ([2000, 130], [2070, 131], 64, 8, 64)


@pytest.mark.parametrize("kind", ["own", "bf16", "fp8"])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
@pytest.mark.parametrize("new,total,Hq,Hk,D", FOUR_WAVES, ids=str)
def test_four_waves_of_columns(new, total, Hq, Hk, D, causal, kind):
    c = Case(kind, new, total, Hq, Hk, D, 1)
    assert c.plan() == Plan(128, 1)
    c.check(*c.run(causal), causal)


@pytest.mark.parametrize("kind", ["own", "bf16", "fp8"])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
def test_tiles_of_256_columns(causal, kind):
    """An 8-bit cache has 128 instead."""
    c = Case(kind, *WIDEST, 2)
    assert c.plan() == Plan(128 if kind == "fp8" else 256, 1)
    c.check(*c.run(causal), causal)


@pytest.mark.parametrize("kind", ["own", "bf16", "fp8"])
@pytest.mark.parametrize("new,total,Hq,Hk,D", [*FOUR_WAVES, WIDEST], ids=str)
def test_odd_values_in_wide_tiles(new, total, Hq, Hk, D, kind):
    c = Case(kind, new, total, Hq, Hk, D, 3)
    assert c.plan().cols == (256 if D == 64 and kind != "fp8" else 128)
    n, m = new[0], total[0]
    for token, head, at, value in ((m - n + 3, 0, 1, INF), (m - n + 401, Hk - 1, D - 1, NAN), (m - n // 2, 0, 40, -INF),
                                   (m - 2, Hk - 1, 7, INF), (m - 1, 1, 33, NAN), (5, Hk - 1, 2, NAN)):
        c.put(0, token, head, at, value)
    c.check(*c.run(True), True)
    c.check(*c.run(False), False)


@pytest.mark.parametrize("kind", ["own", "bf16", "fp8"])
@pytest.mark.parametrize("new,total,Hq,Hk,D", [([40], [3000], 8, 2, 64), ([800, 9], [4000, 2777], 16, 2, 64), ([300, 9], [3000, 700], 8, 2, 128),
                                               ([800, 9], [4000, 4000], 16, 2, 128), ([64], [3000], 8, 2, 256),
                                               ([400, 9], [4000, 4000], 16, 2, 256)], ids=str)
def test_odd_values_in_parts(new, total, Hq, Hk, D, kind):
    """The key axis in parts: columns that see nothing of a part with such a value, and tokens of an earlier part."""
    c = Case(kind, new, total, Hq, Hk, D, 4)
    assert c.plan().parts > 1
    n, m = new[0], total[0]
    for token, head, at, value in ((m - n + 3, 0, 1, INF), (m - 2, Hk - 1, 7, -INF), (m - 1, 0, D - 1, NAN),
                                   (m - n // 2, 0, 5, INF), (100, Hk - 1, 2, INF)):
        c.put(0, token, head, at, value)
    c.check(*c.run(True), True)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_odd_values_beside_a_bad_page(D, kind):
    """Queries that see the page are NaN, another sequence is as it was."""
    new, total = [40, 30], [3000, 2000]
    c = Case(kind, new, total, 8, 2, D, 5)
    assert c.plan().parts > 1
    for b, m in enumerate(total):
        c.put(b, m - 2, 1, 7, NAN)
    wrong = c.table.clone()
    wrong[0, 60] = 1 << 30
    out, lse = c.run(True, wrong)
    assert out[:40].isnan().all() and lse[:40].isnan().all()
    c.check(out, lse, True, [1])


@pytest.mark.parametrize("D", [64, 128, 256])
def test_odd_scales_in_parts(D):
    """An infinite scale of a value reaches the queries that see its token."""
    new, total = [300], [3000]
    c = Case("fp8", new, total, 8, 2, D, 6)
    assert c.plan().parts > 1
    for token in (2800, 2998):
        page, place = int(c.table[0, token // 16]), token % 16
        c.scales[1][page, 1, place] = INF
        c.kv[1].view(torch.uint8)[page, 1, place] = 0x38  # ones, so that no product is 0 times infinity
    c.put(0, 2900, 0, 3, NAN)
    c.check(*c.run(True), True)


@pytest.mark.parametrize("sm_scale", [-0.2, 0.0])
def test_odd_values_under_other_scales(sm_scale):
    c = Case("own", [1400], [1400], 32, 8, 128, 7)
    assert c.plan().cols == 128
    c.put(0, 700, 3, 9, INF)
    out = jb.jq_prompt_attention(c.q, c.k, c.v, starts([1400]), sm_scale=sm_scale)
    ref.check_attention(out, None, c.q, c.k, c.v, True, sm_scale)


@pytest.mark.parametrize("kind", ["own", "bf16", "fp8"])
def test_new_tokens_of_nan_values(kind):
    """What a request leaves whose numbers have run away: every new token's values NaN, another sequence beside it."""
    c = Case(kind, [200, 50], [600, 300], 8, 2, 128, 8)
    for token in range(400, 600):
        for head in range(2):
            c.put(0, token, head, slice(None), NAN)
    out, lse = c.run(True)
    assert out[:200].isnan().all() and lse.isfinite().all()
    c.check(out, lse, True, [1])


@pytest.mark.parametrize("kind", ["own", "bf16", "fp8"])
def test_odd_values_take_a_few_times_as_long(kind):
    """A request with such values may not hold up the others: both at most 20 times the finite call (4 was measured; one
    column after the other, as it was once, 160)."""

    def best(c):
        c.run(True)
        times = []
        for _ in range(5):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            c.run(True)
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)

    c = Case(kind, [512], [2048], 8, 2, 128, 9)
    finite = best(c)
    c.put(0, 2048 - 250, 1, 7, NAN)
    one = best(c)
    for token in range(2048 - 512, 2048):
        c.put(0, token, 0, slice(None), NAN)
    assert one <= 20 * finite and best(c) <= 20 * finite
