"""A cache of a type that no kernel reads is refused as that, whatever scales come with it (no GPU needed: checked first)."""

import os

import pytest

from paper_2609_33601_amd import jq, jq_block as jb

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.skipif(not os.path.exists(jq.LIB_PATH),
                                reason="libjq.so not built (run __graft_entry__.build())")


@pytest.mark.parametrize("scales", [False, True])
@pytest.mark.parametrize("kind", [torch.float16, torch.float32, torch.uint8, torch.int8, torch.float8_e5m2,
                                  torch.float8_e4m3fnuz])
def test_cache_of_a_wrong_type(kind, scales):
    cache = torch.zeros((2, 1, 16, 64), dtype=kind)
    s = torch.zeros((2, 1, 16)) if scales else None
    q = torch.zeros((1, 1, 1, 64), dtype=torch.bfloat16)
    with pytest.raises(TypeError, match="k_cache must be"):
        jb.jq_paged_attention(q, cache, cache, None, None, k_scale=s, v_scale=s)
    with pytest.raises(TypeError, match="k_cache must be"):
        jb.jq_rope_append(None, q[0], q[0], None, None, None, None, cache, cache, k_scale=s, v_scale=s)
