"""Which rows an eviction guards, where positions are negative or guards are off."""
import numpy as np
import pytest
import torch

from gpu_util import cu, say
from paper_2607_28150_amd import smartgen as sg

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("units", [3, 300])          # moves in a launch of their own, and by the unit itself
@pytest.mark.parametrize("sinks", [0, 2])
def test_negative_positions(units, sinks):
    """sinks = 0 guards nothing, rows of no token (position -1) included; a larger number
    guards every position below it."""
    say("negative positions", units, sinks)
    r = np.random.default_rng(units + sinks)
    n, k, page, d = 100, 40, 16, 64
    per = -(-n // page)
    w = r.permutation(units * per * page).reshape(units, -1).astype(np.float32)
    pos = r.integers(5, 1000, w.shape).astype(np.int32)
    pos[r.random(w.shape) < 0.3] = -1
    pos[:, 7] = 1
    pos[:, 11] = -2 ** 31
    pools = [torch.randn((units * per * page, d), device="cuda") for _ in range(2)]
    before = [t.clone() for t in pools]
    table = np.arange(units * per).reshape(units, per) * page
    kept = torch.empty(units, dtype=torch.int32, device="cuda")
    wout, pout = torch.zeros(w.shape, device="cuda"), torch.zeros(w.shape, dtype=torch.int32, device="cuda")
    ws = torch.empty(sg.evict_workspace_size(units, per, page), dtype=torch.uint8, device="cuda")
    sg.sg_evict(*pools, cu(table), cu([n] * units), page, cu([k] * units), torch.from_numpy(w).cuda(), kept, wout, ws,
                pos=torch.from_numpy(pos).cuda(), pos_out=pout, sinks=sinks)
    assert (kept == k).all()
    wout, pout = wout.cpu().numpy(), pout.cpu().numpy()
    for u in range(units):
        guarded = (pos[u, :n] < sinks) & (sinks > 0)
        order = sorted(range(n), key=lambda i: (not guarded[i], 0.0 if guarded[i] else -w[u, i], i))
        chosen = sorted(order[:k])
        stay = [i for i in chosen if i < k]
        src = np.arange(n)
        src[[i for i in range(k) if i not in stay]] = [i for i in chosen if i >= k]
        assert np.array_equal(wout[u, :k], w[u, src[:k]]) and np.array_equal(pout[u, :k], pos[u, src[:k]])
        assert (wout[u, k:n] == 0).all() and (pout[u, k:n] == -1).all()
        rows = u * per * page
        for a, b in zip(pools, before):
            assert torch.equal(a[rows:rows + k], b[rows + torch.from_numpy(src[:k])])
