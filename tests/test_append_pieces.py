"""Appending 16 tokens to a workgroup, where runs of tokens fill the 16-byte pieces of V, and those that do not (GPU)."""
import pytest
import torch

from paper_2502_17728_amd import ops
from test_cache_rules import rules
from test_kv_cache import append_case, check_append, ints, poisoned, table_rows

pytestmark = pytest.mark.gpu

# first slots of three stretches: on a piece, off it by one (and so in every workgroup after), backwards
SLOTS = {"aligned": lambda T: list(range(64, 64 + T)), "off_by_one": lambda T: list(range(65, 65 + T)),
         "gaps": lambda T: [64 + t + 16 * (t // 32) if t % 37 else -1 for t in range(T)],
         "pages_in_no_order": lambda T: [(T // 64 - t // 64) * 64 + t % 64 for t in range(T)]}


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("T,Hq,Hkv,d", [(83, 2, 2, 64), (83, 0, 2, 128), (771, 16, 16, 128)])
@pytest.mark.parametrize("which", sorted(SLOTS))
def test_sixteen_tokens_to_a_workgroup(which, T, Hq, Hkv, d, fmt):
    assert rules().append(T, Hkv, Hq // Hkv, d) == 16
    slots = SLOTS[which](T)
    qkv = append_case(T, Hq, Hkv, d, seed=T)
    cache = poisoned(max(slots) // 64 + 2, Hkv, d, fmt)
    before = cache.data.cpu()
    table = ops.rotary_table(ops.rotary_frequencies(32)[0], T)
    q = ops.kv_cache_append(cache, qkv.cuda(), ints(slots), ints(list(range(T))), table)
    assert (q is None) == (Hq == 0)
    check_append(cache, before, qkv, slots, q, table_rows(table, list(range(T))), False, Hq)
