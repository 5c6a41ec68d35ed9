"""Batches of dg_attention_paged whose spans and records are many: offsets that
start below the first row, contexts near the limit of keys, records taken in
turns, key heads that share an XCD, and values that are not finite in every
type and grouping.  Against 64 bits by the bound of test_gpu_attention_paged,
and against the same call in other launches, where the bits have to stay."""
import math

import pytest

from tests.test_gpu_attention_paged import LOG2E, Batch, captured, check, dg, same, scale  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,dim", [(4, 1, 64), (8, 2, 128)])
@pytest.mark.parametrize("split", [0, 64])
def test_offsets_below_the_first_row(dg, Hq, Hkv, dim, split):  # noqa: F811
    """An offset below 0 is brought to row 0 by the walk and by the join of its records."""
    b = Batch(dg, [20, 30], [200, 300], Hq, Hkv, dim, seed=31, behind=2)
    desc = dict(causal=1, split_keys=split, exp2="inst")
    want = b.run(dg, desc)
    check(b, want, desc)
    for first in (-1, -5, -(1 << 30), -(1 << 31)):
        b.cu[0] = first
        same(b.run(dg, desc), want)
        same(captured(b, dg, desc), want)
    # a sequence that ends below row 0 has no rows
    none = Batch(dg, [0, 20, 30], [200, 200, 300], Hq, Hkv, dim, seed=31,
                 dense=([b.dense[0]] + b.dense, b.q))
    clean = none.run(dg, desc)
    same(clean[:50], want[:50])
    none.cu[:2] = none.cu[:2] - 7
    none.cu[1] = -3
    same(none.run(dg, desc)[:50], clean[:50])
