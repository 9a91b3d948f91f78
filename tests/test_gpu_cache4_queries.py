"""Queries at the ends of their range, over 4-bit rows."""
import numpy as np
import pytest
import torch

import cache_ref as ref
from gpu_util import say
from test_gpu_cache4 import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sign", [-1, 1])
def test_infinite_query(dtype, d, sign):
    """A head all of whose logits are -inf gives zeros and no weight; where some are +inf, NaN."""
    say("infinite query", dtype, d, sign)
    c = Case([40, 70, 3], 3, 2, d, 16, dtype, "fp4", seed=d)
    inf = float("inf")
    code = 2 if sign < 0 else 10                        # channel 0 of every key: 1 or -1
    c.pools[0][:, 0] = (c.pools[0][:, 0] & 0xf0) | code
    c.q[0, 1, 0] = sign * inf                           # all logits -inf
    c.q[1, 4, 0] = -sign * inf                          # all logits +inf
    old = c.r.random((3, 2, c.table.shape[2] * 16))
    out, w = c.run(old, 0.5)
    q = c.q.double().cpu().numpy()
    q[0, 1], q[1, 4] = 0.0, 0.0
    want, tol, ww, wtol = ref.attention(q, *c.values(), c.table, c.n, 16, d ** -0.5, old, 0.5)
    want[0, 1] = 0.0
    ww[0, 0] = ww[0, 0] - 1.0 / 40                      # that head, of equal logits here, gives out nothing
    good = np.ones((3, 6), bool)
    good[1, 4] = False
    assert np.isnan(out[1, 4]).all() and np.isnan(w[1, 1, :70]).all()
    assert (np.abs(out - want) <= tol)[good].all() and (out[0, 1] == 0).all()
    for (b, h), x in ww.items():
        if (b, h) != (1, 1):
            assert (np.abs(w[b, h, :len(x)] - x) <= wtol[b, h] + 1e-37).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size,byte", [(2.0 ** -59, 186), (2.0 ** -61, 188), (1e-30, 220), (1e-36, 247), (3e-38, 251),
                                       (1e-38, 252), (1e-39, 252)])
def test_tiny_queries(d, size, byte):
    """Small fp32 queries (subnormal ones too) against large keys: logits of ordinary size, as
    exact as any; one head of another size beside them."""
    say("tiny queries", d, size, byte)
    c = Case([40, 70, 0, 33], 3, 2, d, 16, "f32", "fp4", seed=d)
    c.pools[2][:, 0] = byte
    c.q.mul_(size)
    c.q[1, 2] *= 2.0 ** -9
    c.check(c.r.random((4, 2, c.table.shape[2] * 16)), 0.5)
    c.check(None, 1.0, False)
