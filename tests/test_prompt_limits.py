"""Limits of the packed attention that need no GPU: the last number of sequences that is accepted, and the next one."""

import os

import pytest

from paper_2609_33601_amd import jq, jq_block as jb
from tests import test_prompt_abi as abi

pytestmark = pytest.mark.skipif(not os.path.exists(jq.LIB_PATH),
                                reason="libjq.so not built (run __graft_entry__.build())")

MOST = 65536
CALLS = {"jq_prompt_attention": abi.PROMPT, "jq_chunk_attention": abi.CHUNK}


@pytest.mark.parametrize("name", CALLS)
def test_sequences(name):
    """As many as a block's search can find.  A misaligned q keeps the accepted number from a launch."""
    q = abi.A + 8
    assert abi._call(name, CALLS[name], B=MOST, q=q) == abi.ALIGN
    assert abi._call(name, CALLS[name], B=MOST + 1, q=q) == abi.SHAPE
    assert abi._call(name, CALLS[name], B=1 << 18, q=q) == abi.SHAPE


def test_workspace_of_too_many_sequences_is_none():
    assert jb.jq_prompt_attention_workspace_bytes(100, 1 << 29, MOST, 8, 2, 64) > 0
    assert jb.jq_prompt_attention_workspace_bytes(100, 1 << 29, MOST + 1, 8, 2, 64) == 0
    assert jb.jq_chunk_attention_workspace_bytes(100, MOST, 8, 2, 64, 100000) > 0
    assert jb.jq_chunk_attention_workspace_bytes(100, MOST + 1, 8, 2, 64, 100000) == 0
