"""4-bit rows on the GPU: writing, copying and reading them back (exact), and
attention over them and over float pools with accumulated weights, against the
64-bit definitions."""
import numpy as np
import pytest
import torch

import cache_ref as ref
from gpu_util import cu, say
from paper_2607_28150_amd import smartgen as sg

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def pool4(rows, d, fill=0):
    u8 = dict(dtype=torch.uint8, device="cuda")
    return (torch.full((rows, d // 2), fill, **u8), torch.full((rows, d // 2), fill, **u8),
            torch.full((rows, 2, d // 32), fill, **u8))


def values4(k4, v4, s4):
    k4, v4, s4 = (t.cpu().numpy() for t in (k4, v4, s4))
    return ref.decode(k4, s4[:, 0]), ref.decode(v4, s4[:, 1])


def hard_rows(d, dtype, seed):
    """Rows where rounding and scales can go wrong."""
    r = np.random.default_rng(seed)
    x = r.standard_normal((96, d)) * np.exp(4 * r.standard_normal((96, 1)))
    steps = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 7, 6, -0.25, -5, 0.0, -0.0, 3.5, 1e-3, -7])
    for i in range(8):                                   # halves between codes, at several scales
        x[i] = np.tile(steps, d // 16) * 2.0 ** (3 * i - 12)
    x[8] = 0.0
    x[9], x[9, 0] = 1e-30, 7e-30
    x[10] = np.where(np.arange(d) % 32 == 0, 3.3e38, 1.0)
    x[11] = 2.0 ** -126 * (np.arange(d) % 16) / 4       # normal and subnormal floats
    x[12, 5], x[13, 40], x[14, 0] = np.inf, np.nan, -np.inf
    t = torch.tensor(x, dtype=torch.float32).to(TYPES[dtype])
    return t, t.double().numpy()


def fetch_one(src, pool, s_src=None, s_pool=None, rows=None, page=16, index=None, start=0, base=0, n_valid=None,
              table=None):
    """One index row into a pool whose pages lie in reverse order."""
    total = (rows if rows is not None else src[0].shape[0]) if index is None else index.numel()
    if table is None:
        pages = max(1, -(-pool[0].shape[0] // page))
        table = cu([[p * page for p in reversed(range(pages))]])
    sg.sg_fetch_fp4(cu([0, total]), total, index, n_valid, cu([base], dtype=torch.int64), src[0], src[1], table, page,
                    cu([start]), pool[0], pool[1], s_src=s_src, s_pool=s_pool)
    return table


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [1, 5, 16])
def test_write_and_read_back_exact(dtype, d, page):
    say("write4", dtype, d, page)
    (kt, k), (vt, v) = hard_rows(d, dtype, 1), hard_rows(d, dtype, 2)
    vt, v = vt.flip(0).contiguous(), v[::-1]
    rows = -(-96 // page) * page
    k4, v4, s4 = pool4(rows + 3, d, fill=7)
    table = fetch_one((kt.cuda(), vt.cuda()), (k4, v4), s_pool=s4, page=page,
                      table=cu([[p * page for p in reversed(range(rows // page))]]))
    at = ref.pool_rows_of(table[0].cpu().numpy(), 96, page, rows + 3)
    for got, scale, x in ((k4, s4[:, 0], k), (v4, s4[:, 1], v)):
        codes, scales = ref.encode(x)
        want = ref.decode(codes, scales)
        assert np.array_equal(scale.cpu().numpy()[at], scales)
        assert np.array_equal(ref.decode(got.cpu().numpy()[at], scales), want, equal_nan=True)
    left = np.setdiff1d(np.arange(rows + 3), at)
    for t in (k4, v4, s4):                              # rows that no entry names stay as they were
        assert (t.cpu().numpy()[left] == 7).all()
    # back as values, in either type, and copied into another pool as they are
    index = cu(at)
    for name in ("f32", "bf16"):
        ok, ov = (torch.empty((96, d), dtype=TYPES[name], device="cuda") for _ in range(2))
        fetch_one((k4, v4), (ok, ov), s_src=s4, index=index, page=96, table=cu([[0]]))
        wk, wv = values4(k4, v4, s4)
        assert np.array_equal(ok.double().cpu().numpy(), wk[at], equal_nan=True)
        assert np.array_equal(ov.double().cpu().numpy(), wv[at], equal_nan=True)
    c4 = pool4(96, d)
    fetch_one((k4, v4), (c4[0], c4[1]), s_src=s4, s_pool=c4[2], index=index, page=96, table=cu([[0]]))
    for a, b in zip(c4, (k4, v4, s4)):
        assert np.array_equal(a.cpu().numpy(), b.cpu().numpy()[at])


@pytest.mark.parametrize("d", [64, 128])
def test_write_skips_what_is_out_of_range(d):
    say("write4 skips", d)
    r = np.random.default_rng(5)
    src = torch.tensor(r.standard_normal((40, d)), dtype=torch.float32).cuda()
    page, pool_rows = 4, 30
    lens, valid = [9, 0, 6, 7], [9, 3, 2, 7]
    off = np.concatenate([[0], np.cumsum(lens)])
    index = r.integers(0, 10, off[-1])
    index[2], index[17] = -5, 10 ** 9
    base = [0, 0, 20, 33]                               # the last row's base + 7.. passes the source
    table = np.array([[4, 12, -3], [0, 0, 0], [8, 2 ** 30, 0], [17, 22, 27]])     # no pool row twice
    start = [1, 0, 2, 3]
    k4, v4, s4 = pool4(pool_rows, d, fill=9)
    sg.sg_fetch_fp4(cu(off), int(off[-1]), cu(index), cu(valid), cu(base, dtype=torch.int64), src, src, cu(table), page,
                    cu(start), k4, v4, s_pool=s4)
    wk, ws = np.full((pool_rows, d // 2), 9, np.uint8), np.full((pool_rows, d // 32), 9, np.uint8)
    codes, scales = ref.encode(src.cpu().numpy())
    for row in range(4):
        for i in range(min(lens[row], valid[row])):
            s, lr = base[row] + int(index[off[row] + i]), start[row] + i
            if not 0 <= s < 40 or lr // page >= 3:
                continue
            pr = int(table[row, lr // page]) + lr % page
            if 0 <= pr < pool_rows:
                wk[pr], ws[pr] = codes[s], scales[s]
    assert np.array_equal(ref.decode(k4.cpu().numpy(), s4[:, 0].cpu().numpy()), ref.decode(wk, ws))
    assert torch.equal(k4, v4) and torch.equal(s4[:, 0], s4[:, 1])


def test_write_shapes_of_the_launch():
    """One long index row, many short ones, and a source in pinned host memory."""
    d, g = 128, torch.Generator().manual_seed(3)
    x = torch.randn((5000, d), generator=g).to(torch.bfloat16)
    want = ref.decode(*ref.encode(x[:64].double().numpy()))
    for where in ("device", "host"):
        src = x.cuda() if where == "device" else x.pin_memory()
        say("write4 long row", where)
        k4, v4, s4 = pool4(5000, d)
        fetch_one((src, src), (k4, v4), s_pool=s4, page=5000, table=cu([[0]]))
        say("write4 short rows", where)
        a4, b4, t4 = pool4(5000, d)
        sg.sg_fetch_fp4(torch.arange(5001, dtype=torch.int32, device="cuda"), 5000, None, None,
                        torch.arange(5000, dtype=torch.int64, device="cuda"), src, src,
                        torch.arange(5000, dtype=torch.int32, device="cuda").view(-1, 1), 1,
                        torch.zeros(5000, dtype=torch.int32, device="cuda"), a4, b4, s_pool=t4)
        assert torch.equal(k4, a4) and torch.equal(v4, b4) and torch.equal(s4, t4) and torch.equal(k4, v4)
        assert np.array_equal(values4(k4, v4, s4)[0][:64], want)
        back = torch.empty((5000, d), dtype=torch.bfloat16, device="cuda")
        say("read4 from", where)
        s = (k4, v4, s4) if where == "device" else tuple(t.cpu().pin_memory() for t in (k4, v4, s4))
        fetch_one((s[0], s[1]), (back, back.clone()), s_src=s[2], page=5000, table=cu([[0]]))
        assert np.array_equal(back.double().cpu().numpy(), values4(k4, v4, s4)[0])


# ------------------------------------------------------------------ attention

class Case:
    """A varlen batch over one pool with pages at random places."""

    def __init__(self, lens, G, Hkv, d, page, dtype, pool, seed=0, spread=1.0, extra_pages=1):
        r = np.random.default_rng(seed)
        B, self.page, self.d = len(lens), page, d
        per = max(1, max(-(-n // page) for n in lens)) + extra_pages
        need = B * Hkv * per
        self.table = (r.permutation(need).reshape(B, Hkv, per) * page).astype(np.int32)
        self.n = np.repeat(np.array(lens, np.int32)[:, None], Hkv, axis=1)
        self.pool_rows = need * page
        q = r.standard_normal((B, Hkv * G, d)) * spread
        k, v = r.standard_normal((2, self.pool_rows, d))
        self.q = torch.tensor(q, dtype=torch.float32).to(TYPES[dtype]).cuda()
        self.fp4 = pool == "fp4"
        if self.fp4:
            k4, sk = encode_fast(k)
            v4, sv = encode_fast(v)
            self.pools = [torch.from_numpy(t).cuda() for t in (k4, v4, np.stack([sk, sv], axis=1))]
        else:
            self.pools = [torch.tensor(t, dtype=torch.float32).to(TYPES[pool]).cuda() for t in (k, v)]
        self.r = r

    def values(self):
        if self.fp4:
            return values4(*self.pools)
        return tuple(t.double().cpu().numpy() for t in self.pools)

    def run(self, weight=None, decay=1.0, weights=True, scale=None, in_place=False, stride=None, ws=None):
        B, Hq, d = self.q.shape
        Hkv, per = self.table.shape[1:]
        rows = stride or per * self.page
        shape = (B, Hq, Hkv, d, per, self.page)
        out = torch.full((B, Hq, d), 777.0, device="cuda")
        w = None if weight is None else torch.tensor(weight, dtype=torch.float32, device="cuda")
        wout = (w if in_place else torch.full((B, Hkv, rows), 777.0, device="cuda")) if weights else None
        table, n = cu(self.table), cu(self.n)
        if self.fp4:
            size = sg.decode_fp4_workspace_size(*shape, weights=weights)
            ws = torch.full((max(16, size),), 0xff, dtype=torch.uint8, device="cuda") if ws is None else ws
            sg.sg_decode_attn_fp4(self.q, *self.pools, table, n, self.page, out, ws=ws, weight=w, weight_out=wout,
                                  decay=decay, scale=scale)
        else:
            size = sg.decode_acc_workspace_size(*shape)
            ws = torch.full((max(16, size),), 0xff, dtype=torch.uint8, device="cuda") if ws is None else ws
            sg.sg_decode_attn_acc(self.q, *self.pools, table, n, self.page, out, wout, ws, weight=w, decay=decay,
                                  scale=scale)
        torch.cuda.synchronize()
        return out.cpu().numpy(), None if wout is None else wout.cpu().numpy()

    def check(self, weight=None, decay=1.0, weights=True, scale=None, **kw):
        out, wout = self.run(weight, decay, weights, scale, **kw)
        k, v = self.values()
        want, tol, w, wtol = ref.attention(self.q.double().cpu().numpy(), k, v, self.table, self.n, self.page,
                                           scale or self.d ** -0.5, weight, decay)
        bad = ~(np.abs(out - want) <= tol)
        assert not bad.any(), (np.argwhere(bad)[:4], out[bad][:4], want[bad][:4], tol[bad][:4])
        for (b, h), x in w.items() if weights else ():
            got = wout[b, h, :len(x)]
            bad = ~(np.abs(got - x) <= wtol[b, h] + 1e-37)
            assert not bad.any(), (b, h, np.argwhere(bad)[:4], got[bad][:4], x[bad][:4])
            rest = wout[b, h, len(x):]
            assert np.array_equal(rest, np.full_like(rest, 777.0) if not kw.get("in_place")
                                  else weight[b, h, len(x):].astype(np.float32))
        return out, wout


def encode_fast(x):
    """ref.encode without its loop over blocks (finite rows in the normal range)."""
    b = x.reshape(-1, 32)
    e = np.ceil(np.log2(np.abs(b).max(axis=1) / 7.0))
    a = np.abs(b) / 2.0 ** e[:, None]
    code = np.abs(a[..., None] - ref.MAGNITUDES).argmin(axis=-1).astype(np.uint8) | (np.signbit(b).astype(np.uint8) << 3)
    code = code.reshape(x.shape)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).astype(np.uint8).reshape(*x.shape[:-1], -1)


LENS = {"short": [0, 1, 2, 15, 16, 17, 31, 33], "mid": [127, 128, 129, 0, 300, 640], "one": [1000]}


@pytest.mark.parametrize("lens", list(LENS))
@pytest.mark.parametrize("G,Hkv,d,page,dtype", [
    (4, 2, 128, 16, "bf16"), (1, 3, 128, 7, "bf16"), (8, 1, 128, 1, "f32"), (2, 2, 64, 16, "bf16"), (3, 2, 64, 24, "f32"),
    (5, 1, 128, 16, "f32"), (16, 1, 64, 64, "bf16"), (7, 2, 128, 100, "bf16"), (16, 2, 128, 16, "f32")])
@pytest.mark.parametrize("weights", [False, True])
def test_attention_fp4(lens, G, Hkv, d, page, dtype, weights):
    say("attn4", lens, G, Hkv, d, page, dtype, weights)
    c = Case(LENS[lens], G, Hkv, d, page, dtype, "fp4", seed=G + d)
    w = c.r.random((len(LENS[lens]), Hkv, c.table.shape[2] * page))
    c.check(w if weights else None, 0.9, weights)


@pytest.mark.parametrize("lens", list(LENS))
@pytest.mark.parametrize("G,Hkv,d,page", [(4, 2, 128, 16), (1, 3, 64, 7), (8, 1, 128, 1), (2, 2, 64, 24), (16, 1, 128, 16),
                                          (8, 2, 64, 16)])
@pytest.mark.parametrize("pool", ["bf16", "f32"])
def test_attention_acc(lens, G, Hkv, d, page, pool):
    say("acc", lens, G, Hkv, d, page, pool)
    c = Case(LENS[lens], G, Hkv, d, page, pool, pool, seed=G + d)
    w = c.r.random((len(LENS[lens]), Hkv, c.table.shape[2] * page))
    out, _ = c.check(w, 0.5)
    plain = torch.empty_like(c.q, dtype=torch.float32)
    B, Hq, _ = c.q.shape
    ws = torch.zeros(max(16, sg.decode_workspace_size(B, Hq, Hkv, d, c.table.shape[2], page)), dtype=torch.uint8,
                     device="cuda")
    sg.sg_decode_attn(c.q, *c.pools, cu(c.table), cu(c.n), page, plain, ws=ws)
    assert np.allclose(plain.cpu().numpy(), out, rtol=0, atol=4e-6 * np.abs(out).max() + 1e-30)


@pytest.mark.parametrize("pool", ["fp4", "bf16"])
@pytest.mark.parametrize("units,rows", [(300, 700), (40, 2100), (1, 70000)])
def test_attention_plans(pool, units, rows):
    """Unit counts and lengths of every launch plan: equal parts, split units, one
    very long unit."""
    say("plans", pool, units, rows)
    lens = [rows] if units == 1 else [(rows * (i % 7)) // 6 for i in range(units // 2)]
    c = Case(lens, 4, 1 if units == 1 else 2, 128, 16, "bf16", pool, seed=units)
    a = c.check(None, 1.0)
    b = c.run(None, 1.0)
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])          # fixed order of every sum


@pytest.mark.parametrize("pool", ["fp4", "f32"])
def test_weights_arguments(pool):
    say("weights arguments", pool)
    c = Case([5, 200], 2, 2, 128, 16, "f32", pool, seed=4)
    rows = c.table.shape[2] * 16
    w = c.r.random((2, 2, rows + 9))
    c.check(w, 1.0, stride=rows + 9)
    c.check(w, 0.25, stride=rows + 9, in_place=True)
    a = c.check(None)
    b = c.check(w[..., :rows], 0.0)
    assert np.array_equal(a[1], b[1])                   # decay 0: as if from zeros
    c.check(w[..., :rows], 1.0, scale=0.7)
    total = sum(a[1][i, h, :n].sum() for i, n in enumerate((5, 200)) for h in range(2))
    assert abs(total - 2 * 2 * 2) < 1e-4                # every q head gives out 1


@pytest.mark.parametrize("pool", ["fp4", "bf16"])
def test_reference_is_raised(pool):
    """Logits that keep growing along the rows by more than the headroom."""
    say("growing logits", pool)
    c = Case([600], 4, 1, 128, 16, "bf16", pool, seed=9, spread=4.0)
    k, v = c.values()
    at = ref.pool_rows_of(c.table[0, 0], 600, 16, c.pool_rows)
    k[at] = np.abs(k[at]) * np.sign(c.q[0, 0].double().cpu().numpy()) * (np.arange(600)[:, None] / 60.0)
    if c.fp4:
        codes, scales = ref.encode(k)
        c.pools[0].copy_(torch.from_numpy(codes))
        c.pools[2][:, 0].copy_(torch.from_numpy(scales))
    else:
        c.pools[0].copy_(torch.tensor(k))
    c.check(None)


@pytest.mark.parametrize("pool", ["fp4", "bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_bad_pages_are_left_out(pool, d):
    say("bad pages", pool, d)
    c = Case([40, 70, 33, 20], 2, 2, d, 8, "f32" if pool == "f32" else "bf16", pool, seed=2)
    c.table[0, 0, 1], c.table[1, 1, 3], c.table[2, 0, 0], c.table[3, 1, :] = -5, c.pool_rows, c.pool_rows - 3, 2 ** 31 - 1
    c.n[1, 0], c.n[2, 1] = 10 ** 6, -4                  # clamped to the table, and to nothing
    w = c.r.random((4, 2, c.table.shape[2] * 8))
    c.check(w, 0.5)
    c.n[:] = 0
    out, wout = c.run(None)
    assert (out == 0).all() and (wout == 777).all()


def test_left_out_row_may_stand_on_nan():
    """Left-out rows read pool row 0 in the place of their own: its NaN goes nowhere."""
    say("nan in pool row 0")
    for d in (64, 128):
        c = Case([40, 33], 4, 2, d, 8, "bf16", "fp4", seed=6)
        c.table[c.table == 0] = 8                       # nobody's page
        c.pools[2][0] = 255
        c.table[0, 0, 1], c.table[1, 1, 0] = -9, c.pool_rows + 5
        c.check(None)


@pytest.mark.parametrize("pool", ["fp4", "f32"])
def test_nan_and_infinity(pool):
    say("nan rows", pool)
    c = Case([100, 100, 3], 2, 2, 64, 16, "f32", pool, seed=8)
    rows = [ref.pool_rows_of(c.table[b, h], 100 if b < 2 else 3, 16, c.pool_rows) for b, h in ((0, 0), (1, 1), (2, 0))]
    if c.fp4:
        c.pools[2][rows[0][77], 0, 1] = 255             # a K block
        c.pools[2][rows[1][5], 1, 0] = 255              # a V block
        c.pools[2][rows[2], 0] = 255                    # every K row
    else:
        c.pools[0][rows[0][77], 40] = float("nan")
        c.pools[1][rows[1][5], 3] = float("nan")
        c.pools[0][rows[2]] = float("nan")
    out, w = c.run(None)
    nan = np.isnan(out).reshape(3, 2, 2, 64)
    assert nan[0, 0].all() and not nan[0, 1].any() and not nan[1, 0].any()
    assert nan[1, 1, :, 3].all() and not nan[1, 1, :, 32:].any() and not nan[2, 1].any()
    if c.fp4:
        assert nan[2, 0].all() and np.isnan(w[2, 0, :3]).all()
    assert np.isnan(w[0, 0, :100]).all() and not np.isnan(w[1]).any() and (w[0, 0, 100:] == 777).all()


def test_empty_pool():
    say("empty pool")
    c = Case([10], 4, 1, 128, 16, "bf16", "fp4", seed=1)
    c.pools = [t[:0] for t in c.pools]
    out, w = c.run(np.ones((1, 1, c.table.shape[2] * 16)), 0.5)
    assert (out == 0).all() and (w[0, 0, :10] == 0.5).all() and (w[0, 0, 10:] == 777).all()


def test_extreme_scales():
    """Every scale byte that is stored, small and large values in one set."""
    say("extreme scales")
    c = Case([64], 2, 1, 64, 16, "f32", "fp4", seed=3)
    at = ref.pool_rows_of(c.table[0, 0], 64, 16, c.pool_rows)
    c.pools[2][torch.from_numpy(at).cuda(), 1] = torch.tensor(
        c.r.choice([2, 60, 100, 127, 140, 160], (64, 2)).astype(np.uint8)).cuda()
    c.pools[2][torch.from_numpy(at[:32]).cuda(), 0] = 2
    c.check(None)


def test_far_pool_rows():
    """Pool rows whose byte offsets pass 32 bits (codes of 4.6 GB)."""
    say("far rows")
    d, rows = 128, 72_000_000
    k4, v4, s4 = (torch.zeros((rows, w), dtype=torch.uint8, device="cuda") for w in (64, 64, 8))
    n, page = 200, 16
    first = rows - 16 * 13
    g = torch.Generator().manual_seed(1)
    x, y = (torch.randn((n, d), generator=g) for _ in range(2))
    table = cu([[first + 16 * (12 - p) for p in range(13)]])
    sg.sg_fetch_fp4(cu([0, n]), n, None, None, cu([0], dtype=torch.int64), x.cuda(), y.cuda(), table, page, cu([0]), k4,
                    v4, s_pool=s4.view(rows, 2, 4))
    q = torch.randn((1, 4, d), generator=g).cuda()
    out = torch.empty((1, 4, d), device="cuda")
    ws = torch.empty(max(16, sg.decode_fp4_workspace_size(1, 4, 1, d, 13, page)), dtype=torch.uint8, device="cuda")
    sg.sg_decode_attn_fp4(q, k4, v4, s4.view(rows, 2, 4), table.view(1, 1, 13), cu([[n]]), page, out, ws=ws)
    k, v = (ref.decode(*ref.encode(t.numpy())) for t in (x, y))
    want, tol, _, _ = ref.attention(q.double().cpu().numpy(), k, v, np.arange(0, n, dtype=np.int32).reshape(1, 1, n),
                                    np.array([[n]]), 1, d ** -0.5)
    assert (np.abs(out.cpu().numpy() - want) <= tol).all()
    assert not k4[:first].any()


def test_streams_and_graph():
    """On a side stream, and captured and replayed between eager calls, sharing a
    workspace in stream order."""
    say("graph")
    c = Case([500, 90, 0, 1], 4, 2, 128, 16, "bf16", "fp4", seed=12)
    B, Hq, d = c.q.shape
    table, n = cu(c.table), cu(c.n)
    rows = c.table.shape[2] * 16
    ws = torch.empty(sg.decode_fp4_workspace_size(B, Hq, 2, d, c.table.shape[2], 16, weights=True), dtype=torch.uint8,
                     device="cuda")
    out, w = torch.empty((B, Hq, d), device="cuda"), torch.zeros((B, 2, rows), device="cuda")

    def step():
        sg.sg_decode_attn_fp4(c.q, *c.pools, table, n, 16, out, ws=ws, weight=w, weight_out=w, decay=0.5)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    first, w1 = out.clone(), w.clone()
    want, tol, ww, wtol = ref.attention(c.q.double().cpu().numpy(), *c.values(), c.table, c.n, 16, d ** -0.5)
    assert (np.abs(first.cpu().numpy() - want) <= tol).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        w.copy_(w1)
        out.zero_()
        graph.replay()
        replayed, wr = out.clone(), w.clone()
        w.copy_(w1)
        step()
        torch.cuda.synchronize()
        assert torch.equal(replayed, out) and torch.equal(wr, w) and torch.equal(out, first)


@pytest.mark.parametrize("units,page", [(5000, 16), (4200, 10), (1500, 16), (700, 9)])
@pytest.mark.parametrize("weights", [False, True])
def test_attention_many_units(units, page, weights):
    """More units than one lookup covers (a whole unit per wavefront), and the
    lookup with several units per lane; empty units among them."""
    say("many units", units, page, weights)
    r = np.random.default_rng(units)
    lens = np.where(r.random(units // 2) < 0.3, 0, r.integers(0, 100, units // 2))
    lens[5:5 + min(300, units // 6)] = 0                # a long run of empty ones
    c = Case(lens.tolist(), 4, 2, 64, page, "bf16", "fp4", seed=units, extra_pages=0)
    c.check(None, 1.0, weights)


@pytest.mark.parametrize("page", [16, 24])
def test_attention_short_units_in_a_row(page):
    """Shares that cross from unit to unit at every tile."""
    say("short units", page)
    c = Case([1 + i % 40 for i in range(256)], 3, 2, 128, page, "f32", "fp4", seed=page, extra_pages=3)
    c.check(None, 1.0, True)


@pytest.mark.parametrize("units,page,d,dtype", [(8, 16, 128, "bf16"), (600, 24, 64, "bf16"), (2050, 16, 128, "f32"),
                                                (4096, 10, 64, "bf16")])
@pytest.mark.parametrize("weights", [False, True])
def test_attention_short_units_of_long_tables(units, page, d, dtype, weights):
    """Tables with room for far more rows than any unit has, as a cache has them
    early on: units without a row and shorter than a tile among them."""
    say("short units of long tables", units, page, d, dtype, weights)
    r = np.random.default_rng(units + 1)
    lens = np.where(r.random(units // 2) < 0.3, 0, r.integers(1, 70, units // 2))
    lens[2:2 + units // 8] = 0                          # a run of empty ones
    c = Case(lens.tolist(), 4, 2, d, page, dtype, "fp4", seed=units, extra_pages=0)
    c.table = np.pad(c.table, ((0, 0), (0, 0), (0, -(-800 // page))))
    a = c.check(None, 1.0, weights)
    assert np.array_equal(a[0], c.run(None, 1.0, weights)[0])


@pytest.mark.parametrize("weights", [False, True])
def test_attention_lengths_around_the_plans(weights):
    """Tables on either side of the capacities at which the launch changes, sets of
    nothing up to a full table: the same definition holds."""
    say("tables around the plans", weights)
    for units in (4, 1024):
        for pages in (8, 9, 16, 17, 32, 33):
            lens = [(16 * pages * (i % 5)) // 4 for i in range(units // 2)]
            c = Case(lens, 2, 2, 64, 16, "bf16", "fp4", seed=pages, extra_pages=0)
            c.check(None, 1.0, weights)


def test_outputs_at_any_float():
    say("outputs at any float")
    for pool in ("fp4", "bf16"):
        c = Case([300, 40], 4, 2, 128, 16, "bf16", pool, seed=5)
        B, Hq, d = c.q.shape
        rows, shape = c.table.shape[2] * 16, (2, Hq, 2, d, c.table.shape[2], 16)
        flat, wflat = torch.zeros(B * Hq * d + 3, device="cuda"), torch.zeros(B * 2 * rows + 3, device="cuda")
        out, w = flat[1:1 + B * Hq * d].view(B, Hq, d), wflat[3:].view(B, 2, rows)
        if pool == "fp4":
            ws = torch.empty(sg.decode_fp4_workspace_size(*shape, weights=True), dtype=torch.uint8, device="cuda")
            sg.sg_decode_attn_fp4(c.q, *c.pools, cu(c.table), cu(c.n), 16, out, ws=ws, weight_out=w)
        else:
            ws = torch.empty(sg.decode_acc_workspace_size(*shape), dtype=torch.uint8, device="cuda")
            sg.sg_decode_attn_acc(c.q, *c.pools, cu(c.table), cu(c.n), 16, out, w, ws)
        want, wwant = c.run(None)
        assert np.array_equal(out.cpu().numpy(), want)
        for b, n in enumerate((300, 40)):
            assert np.array_equal(w[b, :, :n].cpu().numpy(), wwant[b, :, :n])


@pytest.mark.parametrize("pool", ["bf16", "f32", "fp4"])
def test_only_nan_rows(pool):
    say("only nan rows", pool)
    c = Case([40, 40], 4, 1, 128, 16, "f32" if pool == "f32" else "bf16", pool, seed=3)
    at = torch.from_numpy(ref.pool_rows_of(c.table[1, 0], 40, 16, c.pool_rows)).cuda()
    if c.fp4:
        c.pools[2][at] = 255
    else:
        c.pools[0][at] = float("nan")
    out, w = c.run(None)
    assert np.isnan(out[1]).all() and np.isnan(w[1, 0, :40]).all()
    assert not np.isnan(out[0]).any() and not np.isnan(w[0]).any()


def test_refused_where_it_would_not_fit():
    """The calls' own checks with tensors on the GPU."""
    say("refusals")
    c = Case([300], 4, 2, 128, 16, "bf16", "fp4", seed=1)
    table, n, out = cu(c.table), cu(c.n), torch.empty((1, 8, 128), device="cuda")
    with pytest.raises(sg.SmartgenError, match="workspace"):
        sg.sg_decode_attn_fp4(c.q, *c.pools, table, n, 16, out)
    with pytest.raises(ValueError, match="contiguous"):
        sg.sg_decode_attn_fp4(c.q.transpose(0, 1).contiguous().transpose(0, 1)[:, ::2], *c.pools, table, n, 16, out)
    with pytest.raises(ValueError, match="n_rows"):
        sg.sg_decode_attn_fp4(c.q, *c.pools, table, n.long(), 16, out)
    with pytest.raises(ValueError, match="pinned"):
        sg.sg_decode_attn_fp4(c.q, c.pools[0].cpu(), *c.pools[1:], table, n, 16, out)
    with pytest.raises(sg.SmartgenError, match="group size"):
        sg.sg_decode_attn_acc(c.q[:, :6].contiguous(), torch.zeros((64, 128), dtype=torch.bfloat16, device="cuda"),
                              torch.zeros((64, 128), dtype=torch.bfloat16, device="cuda"), table, n, 16, out,
                              torch.zeros((1, 2, c.table.shape[2] * 16), device="cuda"),
                              torch.zeros(1 << 20, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("pool", ["fp4", "bf16"])
def test_table_far_longer_than_the_set(pool):
    """A page table of 41 million rows (more chunks of weights than a launch has
    workgroups in y) over a set of a thousand."""
    say("long table", pool)
    page, pages, n, d = 1 << 20, 40, 1000, 64
    r = np.random.default_rng(2)
    k, v = (r.standard_normal((n, d)).astype(np.float32) for _ in range(2))
    q = torch.tensor(r.standard_normal((1, 1, d)), dtype=torch.float32).to(torch.bfloat16).cuda()
    table, rows = torch.zeros((1, 1, pages), dtype=torch.int32, device="cuda"), page * pages
    w, out = torch.full((1, 1, rows), 7.0, device="cuda"), torch.empty((1, 1, d), device="cuda")
    if pool == "fp4":
        (k4, sk), (v4, sv) = ref.encode(k), ref.encode(v)
        k, v = ref.decode(k4, sk), ref.decode(v4, sv)
        ws = torch.empty(sg.decode_fp4_workspace_size(1, 1, 1, d, pages, page, weights=True), dtype=torch.uint8,
                         device="cuda")
        sg.sg_decode_attn_fp4(q, torch.from_numpy(k4).cuda(), torch.from_numpy(v4).cuda(),
                              torch.from_numpy(np.stack([sk, sv], axis=1)).cuda(), table, cu([[n]]), page, out, ws=ws,
                              weight_out=w)
    else:
        kt, vt = (torch.from_numpy(x).to(torch.bfloat16).cuda() for x in (k, v))
        k, v = kt.double().cpu().numpy(), vt.double().cpu().numpy()
        ws = torch.empty(sg.decode_acc_workspace_size(1, 1, 1, d, pages, page), dtype=torch.uint8, device="cuda")
        sg.sg_decode_attn_acc(q, kt, vt, table, cu([[n]]), page, out, w, ws)
    want, tol, ww, wtol = ref.attention(q.double().cpu().numpy(), k, v, np.zeros((1, 1, pages), np.int32),
                                        np.array([[n]]), page, d ** -0.5)
    assert (np.abs(out.cpu().numpy() - want) <= tol).all()
    assert (np.abs(w[0, 0, :n].cpu().numpy() - ww[0, 0]) <= wtol[0, 0]).all() and (w[0, 0, n:] == 7.0).all()
