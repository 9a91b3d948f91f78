"""Rows that a decode attention leaves out (past a step's rows, or on pages outside the
pool) take part in nothing, whatever the pool's other rows hold: pool row 0, on which a
left-out row's loads may fall, is poisoned with NaN and infinities here."""
import numpy as np
import pytest
import torch

import cache_ref as ref
from gpu_util import cu, say
from paper_2607_28150_amd import smartgen as sg
from test_gpu_cache4 import Case

pytestmark = pytest.mark.gpu

# ragged lengths: parts of a step, splits and whole units that end inside a step
LENS = {"few": [1, 2, 33, 130, 0, 1000], "many": [1 + (37 * i) % 300 for i in range(140)],
        "most": [1 + (11 * i) % 50 for i in range(520)]}


def poison(c, kind):
    """Pool row 0, which belongs to nobody, and pages outside the pool; NaN or infinities
    in its keys, its values or both."""
    c.table[c.table == 0] = c.page
    for i, t in enumerate(c.pools):
        if kind.startswith("kv"[i]) or kind.startswith("both"):
            t[0] = float("nan") if kind.endswith("nan") else float("inf")
            if kind.endswith("inf"):
                t[0, ::3] = -float("inf")
    c.table[2, 0, 0], c.table[3, 1, -2] = -9 - c.page, c.pool_rows + 5


def plain(c, noalloc=False):
    """sg_decode_attn (or its form without a workspace) over the case."""
    B, Hq, d = c.q.shape
    Hkv, per = c.table.shape[1:]
    out = torch.full((B, Hq, d), 777.0, device="cuda")
    ws = None if noalloc else torch.full((max(16, sg.decode_workspace_size(B, Hq, Hkv, d, per, c.page)),), 0xff,
                                         dtype=torch.uint8, device="cuda")
    if noalloc:
        sg.sg_decode_attn_noalloc(c.q, *c.pools, cu(c.table), cu(c.n), c.page, out)
    else:
        sg.sg_decode_attn(c.q, *c.pools, cu(c.table), cu(c.n), c.page, out, ws=ws)
    return out.cpu().numpy()


@pytest.mark.parametrize("pool", ["bf16", "f32"])
@pytest.mark.parametrize("G,d,page", [(1, 128, 16), (2, 64, 7), (4, 128, 16), (4, 64, 1), (8, 128, 16), (8, 64, 24),
                                      (16, 128, 16)])
@pytest.mark.parametrize("kind", ["v nan", "v inf", "k nan", "both inf"])
def test_left_out_rows(pool, G, d, page, kind):
    say("left out", pool, G, d, page, kind)
    c = Case(LENS["few"], G, 2, d, page, pool, pool, seed=G + d)
    poison(c, kind)
    out, _ = c.check(None)                              # finite, and right
    want, tol, _, _ = ref.attention(c.q.double().cpu().numpy(), *c.values(), c.table, c.n, page, d ** -0.5)
    assert (np.abs(plain(c) - want) <= tol).all()
    assert (np.abs(plain(c, noalloc=True) - want) <= tol).all()


@pytest.mark.parametrize("lens", ["many", "most"])
@pytest.mark.parametrize("G", [4, 8])
def test_left_out_rows_of_every_plan(lens, G):
    """Units in equal parts and one workgroup per unit."""
    say("left out plans", lens, G)
    c = Case(LENS[lens], G, 2, 64, 16, "bf16", "bf16", seed=G)
    poison(c, "both nan")
    c.check(None)
    want, tol, _, _ = ref.attention(c.q.double().cpu().numpy(), *c.values(), c.table, c.n, 16, 64 ** -0.5)
    assert (np.abs(plain(c) - want) <= tol).all()


@pytest.mark.parametrize("pool", ["bf16", "f32"])
def test_nan_row_0_of_its_own_unit(pool):
    """A NaN value in pool row 0 reaches its channel of the unit that holds the row, no other."""
    say("nan row 0", pool)
    c = Case([33, 40], 4, 2, 64, 8, pool, pool, seed=4)
    b, h = (int(x[0]) for x in np.nonzero((c.table == 0).any(axis=-1)))
    c.table[b, h, np.nonzero(c.table[b, h] == 0)[0][0]], c.table[b, h, 0] = c.table[b, h, 0], 0
    c.pools[1][0, 5] = float("nan")
    out, w = c.run(None)
    nan = np.isnan(out).reshape(2, 2, 4, 64)
    assert nan[b, h, :, 5].all() and nan.sum() == 4 and not np.isnan(w).any()
    nan = np.isnan(plain(c)).reshape(2, 2, 4, 64)
    assert nan[b, h, :, 5].all() and nan.sum() == 4
