"""How exact attention over the cache is, in the 2-norm, measured by what rounding the exact result costs (GPU).

In tiles of 16 rows the numerators are two bf16 parts (2^-16 of themselves at most is lost) and scores are fp32
sums (relative errors near 2^-20): beside the output's rounding, 2^-9 and less of each value, both are too small to
show, so the result is as exact as the 64-bit one rounded once.  2 % is left for values that round the other way.
Larger tiles round each numerator once, to the output's own precision: two independent errors of one size, sqrt(2)."""
import pytest
import torch

from test_attention_cache import KINDS, Batch
from test_cache_rules import plan

pytestmark = pytest.mark.gpu


def excess(b):
    want, _ = b.want()
    got = b.run().double().cpu()
    return float((got - want).norm() / (want.to(torch.bfloat16).double() - want).norm())


@pytest.mark.parametrize("fmt,d", KINDS)
@pytest.mark.parametrize("seqs,Hq,Hkv,prefix", [([(1, 300)], 8, 8, 0), ([(1, 3000), (1, 700), (1, 65)], 8, 2, 0), ([(4, 900)] * 3, 4, 1, 0),
                                                ([(1, 40), (1, 100)], 8, 2, 1500)])
def test_few_rows_are_as_exact_as_their_type(seqs, Hq, Hkv, prefix, fmt, d):
    b = Batch(seqs, Hq, Hkv, d, fmt, prefix=prefix, seed=11)
    own, shared, _ = plan(b.Q.shape[0], len(seqs), Hkv, Hq // Hkv, d, b.table.shape[1], -(-prefix // 64))
    assert own["rows"] == 16 and (not prefix or shared["rows"] == 16)
    assert excess(b) <= 1.02


@pytest.mark.parametrize("fmt,d", KINDS)
@pytest.mark.parametrize("seqs,rows", [([(12, 900)], 64), ([(50, 900)], 128), ([(90, 900)], 256)])
def test_many_rows_round_their_numerators_once(seqs, rows, fmt, d):
    b = Batch(seqs, 4, 1, d, fmt, seed=12)
    assert plan(b.Q.shape[0], len(seqs), 1, 4, d, b.table.shape[1])[0]["rows"] == rows
    assert excess(b) <= 2 ** 0.5 * 1.1
