"""How a call of jq_prompt_attention or jq_chunk_attention is cut, as the library's own rules give it.

Bound to a function of the library that is no part of its C ABI: the calls and this query read the same rules, so a
test that asserts a plan here runs on the kernel that the plan names.
"""

import collections
import ctypes

from paper_2609_33601_amd import jq

Plan = collections.namedtuple("Plan", "cols parts")

KINDS = {"own": 0, "bf16": 1, "fp8": 2}


def plan(T, B, Hq, Hk, D, max_len, kind):
    """Columns of a tile and the most parts of a key axis; kind "own" (max_len: all keys), or the cache's type."""
    fn = jq.lib().jq_internal_prompt_plan
    fn.argtypes, fn.restype = [ctypes.c_int64] * 6 + [ctypes.c_int, ctypes.POINTER(ctypes.c_int * 2)], ctypes.c_int
    out = (ctypes.c_int * 2)()
    assert fn(T, B, Hq, Hk, D, max_len, KINDS[kind], ctypes.byref(out)) == 0
    return Plan(*out)
