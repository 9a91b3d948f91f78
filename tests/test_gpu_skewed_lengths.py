"""Decode attention over batches in which a few sets are far longer than the rest: most
states belong to few units, and there are more units than share their tiles."""
import numpy as np
import pytest

from gpu_util import say
from test_gpu_cache4 import Case

pytestmark = pytest.mark.gpu


def skewed(units, long, rows, pool, d=64, page=16):
    """`units` sets of up to 60 rows, of which those in `long` get `rows` rows: the pool's
    pages over and over, in another order each time (attention may read a page twice)."""
    r = np.random.default_rng(units + rows)
    lens = r.integers(0, 60, units // 2)
    c = Case(lens.tolist(), 4, 2, d, page, "bf16", pool, seed=units, extra_pages=0)
    per = -(-rows // page)
    pages = c.pool_rows // page
    c.table = np.pad(c.table, ((0, 0), (0, 0), (0, max(0, per - c.table.shape[2]))))
    for u in long:
        b, h = u // 2, u % 2
        c.table[b, h, :per] = np.concatenate([r.permutation(pages) for _ in range(-(-per // pages))])[:per] * page
        c.n[b, h] = rows
    return c


@pytest.mark.parametrize("pool", ["fp4", "bf16"])
@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("units,long,rows", [(64, [0], 32000), (512, [7, 300], 20000), (40, [39], 9000)])
def test_one_long_set(pool, weights, units, long, rows):
    say("one long set", pool, weights, units, rows)
    c = skewed(units, long, rows, pool)
    if pool != "fp4":
        weights = True
    a = c.check(None, 1.0, weights)
    b = c.run(None, 1.0, weights)
    assert np.array_equal(a[0], b[0])                   # fixed order of every sum


@pytest.mark.parametrize("pool", ["fp4", "bf16"])
@pytest.mark.parametrize("weights", [False, True])
def test_long_sets_among_many(pool, weights):
    say("long sets among many", pool, weights)
    c = skewed(4300, [0, 1, 2000, 4299], 3000, pool)
    c.check(None, 1.0, weights or pool != "fp4")
