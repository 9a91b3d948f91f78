"""Eviction by accumulated weight on the GPU, against the plain definition
(exact), and a decode loop of append, attention and eviction."""
import numpy as np
import pytest
import torch

import cache_ref as ref
from gpu_util import cu, say
from paper_2607_28150_amd import smartgen as sg

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


class Pool:
    """Rows of random bytes, so that a move is told apart from any other."""

    def __init__(self, dtype, rows, d, seed):
        g = torch.Generator().manual_seed(seed)
        u8 = lambda *s: torch.randint(0, 250, s, generator=g, dtype=torch.uint8)  # noqa: E731
        if dtype == "fp4":
            self.t = [u8(rows, d // 2).cuda(), u8(rows, d // 2).cuda(), u8(rows, 2, d // 32).cuda()]
        else:
            es = 4 if dtype == "f32" else 2
            view = torch.float32 if dtype == "f32" else torch.bfloat16
            self.t = [u8(rows, d * es).view(view).cuda() for _ in range(2)]
        self.s = self.t[2] if dtype == "fp4" else None

    def bytes(self):
        return [t.contiguous().view(torch.uint8).cpu().numpy().reshape(t.shape[0], -1).copy() for t in self.t]


def check(dtype, d, page, lens, budget, weight, pos=None, sinks=0, recent=None, in_place=False, table=None, seed=0,
          extra=1):
    r = np.random.default_rng(seed)
    units = len(lens)
    per = max(1, max(-(-max(n, 0) // page) for n in lens)) + extra if table is None else table.shape[1]
    if table is None:
        table = (r.permutation(units * per) * page).reshape(units, per)
    pool_rows = units * per * page
    pool = Pool(dtype, pool_rows, d, seed)
    before = pool.bytes()
    stride = weight.shape[1]
    w, n = torch.tensor(weight, dtype=torch.float32).cuda(), cu(lens)
    p = None if pos is None else cu(pos)
    kept = n if in_place else torch.full((units,), -7, **I32)
    wout = w if in_place else torch.full((units, stride), 777.0, device="cuda")
    pout = (None if pos is None else p if in_place else torch.full((units, stride), 777, **I32))
    ws = torch.full((sg.evict_workspace_size(units, per, page),), 0xff, dtype=torch.uint8, device="cuda")

    def call():
        sg.sg_evict(pool.t[0], pool.t[1], cu(table), n, page, cu(budget), w, kept, wout, ws, pos=p, pos_out=pout,
                    sinks=sinks, recent_from=None if recent is None else cu(recent), s_pool=pool.s)

    call()
    got = pool.bytes()
    for u in range(units):
        nn = min(max(lens[u], 0), per * page)
        at = np.arange(nn) if pos is None else pos[u]
        k, moves, ww, pp = ref.evict(nn, budget[u], weight[u].astype(np.float32), at, sinks,
                                     None if recent is None else recent[u])
        assert kept[u].item() == k
        assert np.array_equal(wout[u, :nn].cpu().numpy(), ww, equal_nan=True), u
        rest = wout[u, nn:].cpu().numpy()
        assert np.array_equal(rest, weight[u, nn:].astype(np.float32) if in_place else np.full_like(rest, 777.0))
        if pos is not None:
            assert np.array_equal(pout[u, :nn].cpu().numpy(), pp)
            rest = pout[u, nn:].cpu().numpy()
            assert np.array_equal(rest, pos[u, nn:] if in_place else np.full_like(rest, 777))
        for to, src in moves:
            a, b = (int(table[u][i // page]) + i % page for i in (to, src))
            if 0 <= a < pool_rows and 0 <= b < pool_rows:
                for t in before:
                    t[a] = t[b]
    for a, b in zip(got, before):
        assert np.array_equal(a, b)
    if not in_place:                                    # again: the same
        first = kept.clone(), wout.clone()
        call()
        assert torch.equal(kept, first[0]) and torch.equal(wout.view(torch.int32), first[1].view(torch.int32))
        for a, b in zip(pool.bytes(), got):
            assert np.array_equal(a, b)


def weights(r, units, stride, kind):
    if kind == "spread":
        return np.exp(2 * r.standard_normal((units, stride)))
    if kind == "ties":
        return r.integers(0, 4, (units, stride)).astype(float)
    w = r.standard_normal((units, stride))
    w[r.random((units, stride)) < 0.2] = np.nan
    w[r.random((units, stride)) < 0.1] = np.inf
    w[r.random((units, stride)) < 0.1] = -np.inf
    w[r.random((units, stride)) < 0.1] = -0.0
    return w


@pytest.mark.parametrize("dtype", ["fp4", "bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind", ["spread", "ties", "odd"])
@pytest.mark.parametrize("page", [1, 7, 16])
def test_evict(dtype, d, kind, page):
    say("evict", dtype, d, kind, page)
    r = np.random.default_rng(d + page)
    lens = [0, 1, 2, 63, 64, 65, 300, 1025, 700, 40]
    budget = [3, 1, 1, 20, 64, 64, 250, 1024, 0, -2]
    stride = 1025 + 40 + page
    check(dtype, d, page, lens, budget, weights(r, len(lens), stride, kind), seed=page)


@pytest.mark.parametrize("in_place", [False, True])
def test_evict_positions_and_guards(in_place):
    say("evict guards", in_place)
    r = np.random.default_rng(1)
    lens, budget = [200, 200, 500, 90, 128], [50, 10, 499, 45, 64]
    pos = np.stack([r.permutation(600) for _ in lens])
    recent = [500, 300, 590, 2 ** 31 - 1, -5]           # more guarded than the budget holds; none; all
    check("bf16", 128, 16, lens, budget, weights(r, 5, 600, "ties"), pos=pos, sinks=20, recent=recent, in_place=in_place)
    check("fp4", 128, 16, lens, budget, weights(r, 5, 600, "spread"), pos=pos, sinks=4, in_place=in_place)
    check("f32", 64, 16, lens, budget, weights(r, 5, 600, "spread"), sinks=4, recent=[150, 100, 450, 80, 100],
          in_place=in_place)


@pytest.mark.parametrize("n", [2048, 2049, 8000, 16385, 33000, 81920])
def test_evict_lengths(n):
    """Every number of keys per thread, long units included."""
    say("evict length", n)
    r = np.random.default_rng(n)
    lens, budget = [n, n // 3, n - 5], [n // 5, n // 3 - 1, n - 6]
    check("fp4", 64, 64, lens, budget, weights(r, 3, -(-n // 64) * 64 + 64, "spread"), sinks=4, seed=n, extra=0)


def test_evict_many_units():
    say("evict many units")
    r = np.random.default_rng(2)
    lens = r.integers(0, 130, 700).tolist()
    check("bf16", 64, 16, lens, [min(64, max(0, n - 1)) for n in lens], weights(r, 700, 160, "spread"))


@pytest.mark.parametrize("dtype,d", [("fp4", 128), ("fp4", 64), ("f32", 128), ("f32", 64), ("bf16", 128)])
@pytest.mark.parametrize("in_place", [False, True])
def test_evict_units_move_their_own_rows(dtype, d, in_place):
    """Units enough for every CU: one launch selects and moves."""
    say("evict own rows", dtype, d, in_place)
    r = np.random.default_rng(5)
    lens = r.integers(0, 300, 280).tolist()
    pos = np.stack([r.permutation(320) for _ in lens])
    check(dtype, d, 16, lens, [n // 3 for n in lens], weights(r, 280, 320, "spread"), pos=pos, sinks=3,
          recent=[300] * 280, in_place=in_place, seed=9)


def test_evict_far_pool_rows():
    """Pool rows whose byte offsets pass 32 bits."""
    say("evict far rows")
    rows, n, k = 72_000_000, 64, 32
    t = [torch.zeros((rows, w), dtype=torch.uint8, device="cuda") for w in (64, 64, 8)]
    for i, x in enumerate(t):
        x[-n:] = (torch.arange(n, device="cuda") + 10 * i + 1).to(torch.uint8)[:, None]
    w = torch.arange(n, dtype=torch.float32, device="cuda").view(1, n)       # the last half is kept
    kept, out = torch.empty(1, **I32), torch.empty((1, n), device="cuda")
    ws = torch.empty(sg.evict_workspace_size(1, 1, n), dtype=torch.uint8, device="cuda")
    sg.sg_evict(t[0], t[1], cu([[rows - n]]), cu([n]), n, cu([k]), w, kept, out, ws, s_pool=t[2].view(rows, 2, 4))
    assert kept.item() == k
    for i, x in enumerate(t):
        got = x[-n:].cpu().numpy()
        assert (got[:k] == (np.arange(k, n) + 10 * i + 1)[:, None]).all()
        assert not x[:-n].any()
    assert np.array_equal(out[0, :k].cpu().numpy(), np.arange(k, n)) and not out[0, k:].any()


def test_evict_bad_pages():
    """Rows outside the pool are ranked like any other; a move that touches one copies nothing."""
    say("evict bad pages")
    r = np.random.default_rng(7)
    table = (r.permutation(3 * 9) * 16).reshape(3, 9)
    table[0, 1], table[1, 5], table[2, 0], table[2, 8] = -40, 3 * 9 * 16 - 5, 2 ** 31 - 1, 3 * 9 * 16
    check("bf16", 128, 16, [130, 120, 140], [60, 30, 100], weights(r, 3, 160, "spread"), table=table, seed=3)
    check("fp4", 64, 16, [10 ** 6, 120, -3], [60, 30, 100], weights(r, 3, 160, "spread"), table=table, seed=3)


@pytest.mark.parametrize("pool", ["fp4", "bf16"])
@pytest.mark.parametrize("graph", [False, True])
def test_decode_loop(pool, graph):
    """Append a token, attend and accumulate, evict one row: twenty steps of a
    batch at its budget, eager or replayed, against the definitions."""
    say("decode loop", pool, graph)
    B, Hkv, G, d, page, budget, steps = 3, 2, 4, 128, 16, 70, 20
    units, per = B * Hkv, 5
    r = np.random.default_rng(11)
    table = cu((r.permutation(units * per) * page).reshape(units, per))
    rows = units * per * page
    kv = torch.tensor(r.standard_normal((2, units * steps, d)), dtype=torch.float32).to(torch.bfloat16).cuda()
    qs = torch.tensor(r.standard_normal((steps, B, Hkv * G, d)), dtype=torch.float32).to(torch.bfloat16).cuda()
    if pool == "fp4":
        k, v = (torch.zeros((rows, d // 2), dtype=torch.uint8, device="cuda") for _ in range(2))
        s = torch.zeros((rows, 2, d // 32), dtype=torch.uint8, device="cuda")
    else:
        (k, v), s = (torch.zeros((rows, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)), None
    start = r.integers(40, 71, units)
    n = cu(start)
    seed_rows = torch.tensor(r.standard_normal((2, units * per * page, d)), dtype=torch.float32).to(torch.bfloat16).cuda()
    stride = per * page
    w, pos = torch.zeros((units, stride), device="cuda"), torch.full((units, stride), -1, **I32)
    now = torch.zeros((), **I32)

    def append(off, total, n_valid, base, src, at):
        if pool == "fp4":
            sg.sg_fetch_fp4(off, total, None, n_valid, base, src[0], src[1], table, page, at, k, v, s_pool=s)
        else:
            sg.sg_fetch(off, total, None, n_valid, base, src[0], src[1], table, page, at, k, v)

    append(cu(np.concatenate([[0], np.cumsum(start)])), int(start.sum()), None,
           torch.arange(units, dtype=torch.int64, device="cuda") * per * page, seed_rows, torch.zeros(units, **I32))
    for u in range(units):
        pos[u, :start[u]] = torch.arange(int(start[u]), **I32)
    one, base = torch.arange(units + 1, **I32), torch.arange(units, dtype=torch.int64, device="cuda")
    cur_k, cur_v = (torch.empty((units, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q, out = torch.empty_like(qs[0]), torch.empty((B, Hkv * G, d), device="cuda")
    shape = (B, Hkv * G, Hkv, d, per, page)
    size = sg.decode_fp4_workspace_size(*shape, weights=True) if pool == "fp4" else sg.decode_acc_workspace_size(*shape)
    ws = torch.empty(max(size, sg.evict_workspace_size(units, per, page)), dtype=torch.uint8, device="cuda")
    most = cu([budget] * units)
    recent = torch.empty(units, **I32)

    def step():
        append(one, units, None, base, (cur_k, cur_v), n)
        pos.scatter_(1, n[:, None].long(), (now + 1000).expand(units, 1))
        n.add_(1)
        wv, nn, tb = w.view(B, Hkv, stride), n.view(B, Hkv), table.view(B, Hkv, per)
        if pool == "fp4":
            sg.sg_decode_attn_fp4(q, k, v, s, tb, nn, page, out, ws=ws, weight=wv, weight_out=wv, decay=0.95)
        else:
            sg.sg_decode_attn_acc(q, k, v, tb, nn, page, out, wv, ws, weight=wv, decay=0.95)
        recent.copy_((now + 1000 - 3).expand(units))
        sg.sg_evict(k, v, table, n, page, most, w, n, w, ws, pos=pos, pos_out=pos, sinks=4, recent_from=recent, s_pool=s)

    state = [n, w, pos, k, v] + ([s] if s is not None else [])
    g = None
    if graph:
        keep = [t.clone() for t in state]
        cur_k.copy_(kv[0, :units])
        cur_v.copy_(kv[1, :units])
        q.copy_(qs[0])
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        for a, b in zip(state, keep):
            a.copy_(b)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        for a, b in zip(state, keep):
            a.copy_(b)
    for t in range(steps):
        now.fill_(t)
        cur_k.copy_(kv[0, t * units:(t + 1) * units])
        cur_v.copy_(kv[1, t * units:(t + 1) * units])
        q.copy_(qs[t])
        n0, w0, p0 = n.cpu().numpy().copy(), w.cpu().numpy().copy(), pos.cpu().numpy().copy()
        rows0 = [x.cpu().clone() for x in (k, v) + ((s,) if s is not None else ())]
        g.replay() if graph else step()
        torch.cuda.synchronize()
        # the attention saw the rows before and the appended one
        tb = table.cpu().numpy()
        kk, vv = values(rows0)
        new = [x.float().cpu().numpy().astype(np.float64) for x in (cur_k, cur_v)]
        if s is not None:
            new = [ref.decode(*ref.encode(x)) for x in new]
        for u in range(units):
            at = tb[u, n0[u] // page] + n0[u] % page
            kk[at], vv[at] = new[0][u], new[1][u]
            p0[u, n0[u]] = 1000 + t
        want, tol, ww, wtol = ref.attention(q.double().cpu().numpy(), kk, vv, tb.reshape(B, Hkv, per),
                                            (n0 + 1).reshape(B, Hkv), page, d ** -0.5, w0.reshape(B, Hkv, stride),
                                            np.float32(0.95))
        assert (np.abs(out.cpu().numpy() - want) <= tol).all()
        kb, vb = values([x.cpu() for x in (k, v) + ((s,) if s is not None else ())])
        for u in range(units):
            count = int(n0[u]) + 1
            kept = min(budget, count)
            assert n[u].item() == kept
            got_pos = pos[u].cpu().numpy()
            held = got_pos[:kept]
            assert len(set(held.tolist())) == kept and (got_pos[kept:count] == -1).all()
            where = {int(x): i for i, x in enumerate(p0[u, :count])}
            src = np.array([where[int(x)] for x in held])
            b, h = u // Hkv, u % Hkv
            got_w = w[u, :kept].cpu().numpy()
            assert (np.abs(got_w - ww[b, h][src]) <= wtol[b, h][src] + 1e-30).all()
            gone = np.setdiff1d(np.arange(count), src)
            assert ((p0[u, gone] >= 4) & (p0[u, gone] < 1000 + t - 3)).all()
            free = (p0[u, src] >= 4) & (p0[u, src] < 1000 + t - 3)
            if len(gone) and free.any():                # no kept row is lighter than an evicted one
                slack = wtol[b, h].max() * 2
                assert ww[b, h][gone].max() <= ww[b, h][src[free]].min() + slack
            old = ref.pool_rows_of(tb[u], count, page, rows)[src]
            cur = ref.pool_rows_of(tb[u], kept, page, rows)
            assert np.array_equal(kb[cur], kk[old]) and np.array_equal(vb[cur], vv[old])


def values(rows):
    if len(rows) == 3:
        a = [x.numpy() for x in rows]
        return ref.decode(a[0], a[2][:, 0]), ref.decode(a[1], a[2][:, 1])
    return [x.double().numpy() for x in rows]
