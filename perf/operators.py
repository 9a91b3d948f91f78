"""Performance cases of the 4-bit cache and of eviction by accumulated attention weight, on one GPU.

Four operators of the decode side.  ``fetch4``: K/V rows are rounded to 4 bits (E2M1 codes, one E8M0 scale per 32
channels) and placed in a paged pool, and read back as values.  ``attn4``: decode attention over such a pool, with or
without the weights that its rows receive.  ``acc``: decode attention over a float32 or bfloat16 pool that accumulates
those weights.  ``evict``: a pool is cut to its budget by accumulated weight.  Shapes are those of the synthetic
workloads (8B- and 70B-shaped GQA heads of 128, the small 8-head model of 64), caches of one row to 32K rows per head,
one request or a varlen batch.  ``listed()`` gives the fixed cases, ``draw()`` others of the same ranges; ``exact()``
recomputes the numbers in 64 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False                      # set by the caller: whether run() calls the framework or computes the plain forms

DEV = "cuda"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 32                       # channels that share a scale
SINKS = 4                        # leading tokens that every query attends to
HEAVY = 100                      # one token in HEAVY is a heavy hitter


def _lib():
    from paper_2607_28150_amd import smartgen
    return smartgen


def listed():
    b8 = dict(dtype="bf16", Hq=32, Hkv=8, d=128)      # Llama-3-8B-shaped attention
    b70 = dict(dtype="bf16", Hq=64, Hkv=8, d=128)     # 70B-shaped attention
    small = dict(dtype="f32", Hq=8, Hkv=8, d=64)      # the small fp32 model
    return [
        # the newest token's row of every head of 64 requests, appended to the cache of one layer
        dict(name="fetch4_append", kind="fetch4", B=64, lo=1, hi=1, N=1, page=16, **b8),
        # the selected 10% of an 8K prompt, every layer (as sequences), on arrival
        dict(name="fetch4_select", kind="fetch4", B=32, lo=819, hi=819, N=8192, page=16, **b8),
        # a ragged batch of the small fp32 model, odd pages
        dict(name="fetch4_f32", kind="fetch4", B=5, lo=37, hi=2048, N=2048, page=24, **small),
        # attention of one layer for one request over its 10%: the smallest decode call
        dict(name="attn4_one", kind="attn4", B=1, lo=819, hi=819, page=16, weights=False, **b8),
        # one layer of 64 requests of different lengths (12% of 2K to 32K tokens)
        dict(name="attn4_batch", kind="attn4", B=64, lo=245, hi=3932, page=16, weights=False, **b8),
        # the same with the weights that an eviction goes by
        dict(name="attn4_batch_weights", kind="attn4", B=64, lo=245, hi=3932, page=16, weights=True, **b8),
        # 16 whole prompts of 8K to 32K tokens, 8 query heads per KV head
        dict(name="attn4_long", kind="attn4", B=16, lo=8192, hi=32768, page=64, weights=False, **b70),
        # the small fp32 model, one query head per KV head, odd pages, with weights
        dict(name="attn4_f32_weights", kind="attn4", B=7, lo=1, hi=2047, page=24, weights=True, **small),
        # accumulated weights over a bfloat16 cache: one request, and the batch
        dict(name="acc_one", kind="acc", B=1, lo=819, hi=819, page=16, **b8),
        dict(name="acc_batch", kind="acc", B=64, lo=245, hi=3932, page=16, **b8),
        # a decode step of 64 requests that hold their 1,024 rows: the newest row stays, the lightest goes
        dict(name="evict_step", kind="evict", B=64, lo=1025, hi=1025, drop=1, keep=0, recent=64, page=16, **b8),
        # eight whole prompts cut to 20% of their rows after the prefill
        dict(name="evict_prompt", kind="evict", B=8, lo=8192, hi=32768, drop=0, keep=2000, recent=256, page=16, **b8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["fetch4", "fetch4", "attn4", "attn4", "attn4", "acc", "acc", "evict", "evict"])
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    d = 64 if rng.random() < 0.3 else 128
    Hkv = rng.choice([1, 2, 4, 8])
    G = rng.choice([1, 2, 4, 4, 8] + ([3, 5, 7, 16] if kind == "attn4" else [16]))
    c = dict(kind=kind, dtype=dtype, Hq=G * Hkv, Hkv=Hkv, d=d, page=rng.choice([1, 16, 16, 24, 64]))
    c["B"] = _log(rng, 1, 64)
    c["hi"] = _log(rng, 1, 32768)
    c["lo"] = rng.choice([0, rng.randint(0, c["hi"]), c["hi"]])
    if kind == "fetch4":
        c["N"] = _log(rng, max(1, c["hi"]), 32768)
    elif kind == "attn4":
        c["weights"] = rng.random() < 0.5
    elif kind == "evict":
        c["hi"] = max(2, c["hi"])
        c["drop"] = 1 if rng.random() < 0.4 else 0
        c["keep"] = rng.randint(300, 9000)
        c["recent"] = rng.choice([0, 16, 64, 256])
    top = {m: max(work(x)[m] for x in listed()) for m in ("bytes", "flops")}
    # no drawn case is larger than the largest listed one, nor are its padded plain arrays
    while any(work(c)[m] > top[m] for m in top) or c["B"] * c["Hkv"] * c["hi"] > 16 * 8 * 32768 or (
            kind == "fetch4" and c["B"] * Hkv * c["N"] * d > 32 * 8 * 8192 * 128):
        c["B"] = c["B"] // 2
    return c


# ------------------------------------------------------------------ sizes

def _lens(c):
    """The sequences' row counts: a fixed spread over [lo, hi] (the same in every run of the case)."""
    r = random.Random("%d %d %d" % (c["B"], c["lo"], c["hi"]))
    return [r.randint(c["lo"], c["hi"]) for _ in range(c["B"])] if c["B"] > 1 else [c["hi"]]


def _budget(c, n):
    return n - 1 if c["drop"] and n > 1 else max(1, n * c["keep"] // 10000) if not c["drop"] else n


def work(c):
    """Bytes: every input read once, every output written once (a 4-bit pool that is written and read back counts for
    both).  Flops: the products of the queries with their keys and the weighted sum of the values."""
    es, d, Hq, Hkv = (4 if c["dtype"] == "f32" else 2), c["d"], c["Hq"], c["Hkv"]
    lens = _lens(c)
    rows = sum(lens)
    row, row4 = 2 * d * es, d + 2 * d // BLOCK        # bytes of a K and V row
    if c["kind"] == "fetch4":
        return {"bytes": max(1, Hkv * rows * (2 * row + 2 * row4 + 8)), "flops": 0}
    if c["kind"] == "evict":
        moved = sum((n - _budget(c, n)) * _budget(c, n) / n for n in lens if n)     # of rows in no order of weight
        return {"bytes": Hkv * (rows * 16 + moved * 2 * row) + 8 * c["B"] * Hkv, "flops": 0}
    by = Hkv * rows * (row4 if c["kind"] == "attn4" else row) + c["B"] * Hq * d * (es + 4)
    if c["kind"] == "acc" or c["weights"]:
        by += 8 * Hkv * rows
    return {"bytes": by, "flops": 4 * Hq * d * rows}


# ------------------------------------------------------------------ 4-bit rows, in 32 bits

def _round4(x):
    """Rows [..., d] rounded to 4 bits: the values (float32) [..., d], their codes (uint8) [..., d / 2], low nibble
    first, and the scale bytes [..., d / 32]."""
    x = x.float()
    b = x.reshape(*x.shape[:-1], x.shape[-1] // BLOCK, BLOCK)
    top = b.abs().amax(dim=-1)
    bits = top.view(torch.int32)
    # the scale 2^e: the smallest with amax <= 7 * 2^e (7, half-way between 6 and 8, still rounds to 6)
    byte = ((bits >> 23) - 2 + ((bits & 0x7fffff) > 0x600000).int()).clamp(2, 252)
    scale = (byte << 23).view(torch.float32)
    inv = ((254 - byte) << 23).view(torch.float32)
    a = (b.abs() * inv[..., None]).clamp(max=6.0)
    step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
    a = torch.round(a / step) * step                  # halves go to the even code
    whole = torch.where(a < 2.0, 2.0 * a, torch.where(a < 4.0, a + 2.0, 0.5 * a + 4.0)).to(torch.uint8)
    neg = torch.signbit(b)
    code = (whole | (neg.to(torch.uint8) << 3)).reshape(x.shape)
    value = (torch.where(neg, -a, a) * scale[..., None]).reshape(x.shape)
    return value, code[..., 0::2] | (code[..., 1::2] << 4), byte.to(torch.uint8)


def _values4(codes, scales):
    """Values (float32) of codes [..., d / 2] under scale bytes [..., d / 32]."""
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    v = torch.stack([table[(codes & 15).long()], table[(codes >> 4).long()]], dim=-1)
    s = (scales.to(torch.int32) << 23).view(torch.float32)
    v = v.reshape(*scales.shape, BLOCK) * s[..., None]
    return v.reshape(*codes.shape[:-1], -1)


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _bytes(n):
    return torch.empty(max(16, int(n)), dtype=torch.uint8, device=DEV)


def _table(c, g):
    """Pages of the sequences' rows at random places of a pool: the table [B][Hkv][pages], the pool's rows.  An entry
    past a sequence's rows repeats its first page (one page behind all others for the sequences without rows)."""
    page, Hkv, lens = c["page"], c["Hkv"], _lens(c)
    need = torch.tensor([-(-n // page) for n in lens], device=DEV)
    per = max(1, int(need.max()))
    has = torch.arange(per, device=DEV)[None, None, :] < need[:, None, None].expand(-1, Hkv, 1)
    total = int(need.sum()) * Hkv
    table = torch.full((len(lens), Hkv, per), total * page, dtype=torch.int32, device=DEV)
    table[has] = torch.randperm(total, generator=g, device=DEV).to(torch.int32) * page
    return torch.where(has, table, table[:, :, :1]).contiguous(), (total + (min(lens) == 0)) * page


def _prepare_fetch4(c, g):
    B, Hkv, d, N, lens = c["B"], c["Hkv"], c["d"], c["N"], _lens(c)
    units = B * Hkv
    table, pool_rows = _table(c, g)
    k, v = (torch.randn((units * N, d), generator=g, device=DEV).to(DT[c["dtype"]]) for _ in range(2))
    count = _i32(lens).repeat_interleave(Hkv)
    off = torch.zeros(units + 1, dtype=torch.int32, device=DEV)
    off[1:] = count.cumsum(0)
    total = sum(lens) * Hkv
    unit = torch.repeat_interleave(torch.arange(units, device=DEV), count, output_size=total)
    i = torch.arange(total, device=DEV) - off[unit]
    # a selection of ascending, distinct tokens: as many per unit as its count, spread over the prompt
    index = (i * (N // max(1, max(lens))) + torch.randint(0, max(1, N // max(1, max(lens))), (total,), generator=g,
                                                           device=DEV)).to(torch.int32)
    at = (table.reshape(units, -1).long()[unit, i // c["page"]] + i % c["page"]).to(torch.int32)
    u8 = dict(dtype=torch.uint8, device=DEV)
    return dict(total=total, off=off, index=index, base=torch.arange(units, device=DEV) * N, k=k, v=v,
                table=table.reshape(units, -1), start=torch.zeros(units, dtype=torch.int32, device=DEV),
                k4=torch.zeros((pool_rows, d // 2), **u8), v4=torch.zeros((pool_rows, d // 2), **u8),
                s4=torch.zeros((pool_rows, 2, d // BLOCK), **u8), at=at, back_off=_i32([0, total]),
                back_base=torch.zeros(1, dtype=torch.int64, device=DEV), back_table=_i32([[0]]), back_start=_i32([0]),
                ok=torch.empty((total, d), dtype=k.dtype, device=DEV), ov=torch.empty((total, d), dtype=k.dtype, device=DEV))


def _rows(c, g, mu, table, pool_rows):
    """K and V rows of a pool: N(0, 1), where the first rows of every head and one row in a hundred lean towards the
    head's mean query (component 4 along it)."""
    B, Hkv, d, page = c["B"], c["Hkv"], c["d"], c["page"]
    k = torch.randn((pool_rows, d), generator=g, device=DEV)
    v = torch.randn((pool_rows, d), generator=g, device=DEV)
    n = max(1, max(_lens(c)))
    pick = torch.cat([torch.arange(min(SINKS, n), device=DEV),
                      torch.randint(0, n, (max(1, n // HEAVY),), generator=g, device=DEV)])
    at = table.long()[:, :, pick // page] + pick % page
    u = (mu / mu.norm(dim=-1, keepdim=True))[:, :, None, :].expand(B, Hkv, pick.numel(), d)
    k[at] += (4.0 - (k[at] * u).sum(-1, keepdim=True)) * u
    return k, v


def _prepare_attention(c, g):
    B, Hq, Hkv, d, dt = c["B"], c["Hq"], c["Hkv"], c["d"], DT[c["dtype"]]
    table, pool_rows = _table(c, g)
    mu = torch.randn((B, Hkv, d), generator=g, device=DEV)
    k, v = _rows(c, g, mu, table, pool_rows)
    q = mu.repeat_interleave(Hq // Hkv, dim=1) + torch.randn((B, Hq, d), generator=g, device=DEV)
    stride = table.shape[2] * c["page"]
    s = dict(q=q.to(dt), table=table, n=_i32(_lens(c))[:, None].expand(B, Hkv).contiguous(),
             o=torch.empty((B, Hq, d), device=DEV), w=None, wout=None, decay=1.0)
    if c["kind"] == "acc" or c["weights"]:
        # weights of some steps before this one
        s.update(w=torch.rand((B, Hkv, stride), generator=g, device=DEV) * (Hq // Hkv / stride), decay=0.98,
                 wout=torch.zeros((B, Hkv, stride), device=DEV))
    if c["kind"] == "acc":
        s.update(k=k.to(dt), v=v.to(dt))
    else:
        (_, k4, sk), (_, v4, sv) = _round4(k), _round4(v)
        s.update(k4=k4, v4=v4, s4=torch.stack([sk, sv], dim=1).contiguous())
    return s


def _prepare_evict(c, g):
    B, Hkv, d, dt, lens = c["B"], c["Hkv"], c["d"], DT[c["dtype"]], _lens(c)
    table, pool_rows = _table(c, g)
    units, stride = B * Hkv, table.shape[2] * c["page"]
    n = _i32(lens).repeat_interleave(Hkv)
    # weights of a long decode: spread over several powers of two, and some rows that no query ever reached
    w = torch.exp(2.0 * torch.randn((units, stride), generator=g, device=DEV))
    w = torch.where(torch.rand((units, stride), generator=g, device=DEV) < 0.05, 0.0, w)
    # the tokens the rows hold: in order after a prefill, in any order once rows have been moved
    pos = torch.arange(stride, device=DEV).expand(units, stride)
    if c["drop"]:
        far = torch.where(pos < n[:, None], torch.rand((units, stride), generator=g, device=DEV), 2.0 + pos)
        pos = far.argsort(dim=1)
    return dict(table=table.reshape(units, -1), n=n, w=w, pos=pos.to(torch.int32).contiguous(),
                budget=_i32([_budget(c, x) for x in lens]).repeat_interleave(Hkv), recent=n - c["recent"],
                kept=torch.empty(units, dtype=torch.int32, device=DEV), wout=torch.zeros((units, stride), device=DEV),
                pout=torch.zeros((units, stride), dtype=torch.int32, device=DEV),
                k=torch.randn((pool_rows, d), generator=g, device=DEV, dtype=dt),
                v=torch.randn((pool_rows, d), generator=g, device=DEV, dtype=dt))


def prepare(c, seed):
    how = {"fetch4": _prepare_fetch4, "attn4": _prepare_attention, "acc": _prepare_attention, "evict": _prepare_evict}
    return dict(how[c["kind"]](c, _gen(seed)), c=c)


# ------------------------------------------------------------------ the plain forms

def _plain_fetch4(c, s):
    count = s["off"][1:] - s["off"][:-1]
    unit = torch.repeat_interleave(torch.arange(count.numel(), device=DEV), count, output_size=s["total"])
    src = s["base"][unit] + s["index"]
    s["ok"][:], s["ov"][:] = _round4(s["k"][src])[0], _round4(s["v"][src])[0]
    return s["ok"], s["ov"]


def _paged(c, table):
    """Pool rows [units..., pages * page] of the logical rows."""
    return (table.long()[..., None] + torch.arange(c["page"], device=DEV)).flatten(-2)


def _plain_attention(c, s):
    B, Hq, Hkv, d = c["B"], c["Hq"], c["Hkv"], c["d"]
    top = max(1, max(_lens(c)))
    at = _paged(c, s["table"])[:, :, :top]
    if c["kind"] == "acc":
        k, v = s["k"][at].float(), s["v"][at].float()
    else:
        k, v = _values4(s["k4"][at], s["s4"][at, 0]), _values4(s["v4"][at], s["s4"][at, 1])
    valid = (torch.arange(top, device=DEV) < s["n"][:, :, None])[:, :, None, :]
    z = torch.matmul(s["q"].float().reshape(B, Hkv, Hq // Hkv, d), k.transpose(2, 3)) * d ** -0.5
    z = z.masked_fill(~valid, -math.inf)
    p = torch.exp(z - z.amax(dim=-1, keepdim=True)).masked_fill(~valid, 0.0)
    total = p.sum(dim=-1, keepdim=True)
    p = p / torch.where(total > 0.0, total, 1.0)
    s["o"].copy_(torch.matmul(p, v).reshape(B, Hq, d))
    if s["w"] is None:
        return s["o"]
    old, new = s["w"][:, :, :top], s["wout"][:, :, :top]
    new.copy_(torch.where(valid[:, :, 0], s["decay"] * old + p.sum(dim=2), new))
    return s["o"], s["wout"]


def _plain_evict(c, s):
    n, w, pos = s["n"][:, None], s["w"], s["pos"]
    row = torch.arange(w.shape[1], device=DEV)[None, :]
    valid = row < n
    k = torch.minimum(s["budget"], s["n"])
    s["kept"].copy_(k)
    k = k[:, None]
    guarded = (pos < SINKS) | (pos >= s["recent"][:, None])
    key = torch.where(guarded, math.inf, w).masked_fill(~valid, -math.inf)
    order = torch.sort(key, dim=1, descending=True, stable=True).indices        # equal weights: the lower row first
    keep = torch.zeros_like(valid).scatter_(1, order, (row < k).expand_as(order).contiguous())
    # the kept rows at and past k go, in order, to the rows below k that are not kept
    move, hole = (keep & (row >= k)).nonzero(as_tuple=True), (~keep & (row < k)).nonzero(as_tuple=True)
    at = _paged(c, s["table"])
    src, dst = at[move], at[hole]
    s["k"][dst], s["v"][dst] = s["k"][src], s["v"][src]
    left = valid & (row < k)
    wout = torch.where(left, w, torch.where(valid, 0.0, s["wout"]))
    pout = torch.where(left, pos, torch.where(valid, -1, s["pout"]))
    wout[hole], pout[hole] = w[move], pos[move]
    s["wout"].copy_(wout)
    s["pout"].copy_(pout)
    return s["kept"], s["wout"], s["pout"], s["k"], s["v"]


# ------------------------------------------------------------------ one pass

def _own_fetch4(c, s):
    sg = _lib()
    sg.sg_fetch_fp4(s["off"], s["total"], s["index"], None, s["base"], s["k"], s["v"], s["table"], c["page"],
                    s["start"], s["k4"], s["v4"], s_pool=s["s4"])
    sg.sg_fetch_fp4(s["back_off"], s["total"], s["at"], None, s["back_base"], s["k4"], s["v4"], s["back_table"],
                    max(1, s["total"]), s["back_start"], s["ok"], s["ov"], s_src=s["s4"])
    return s["ok"], s["ov"]


def _workspace(sg, c, pages):
    shape = (c["B"], c["Hq"], c["Hkv"], c["d"], pages, c["page"])
    if c["kind"] == "evict":
        return _bytes(sg.evict_workspace_size(c["B"] * c["Hkv"], pages, c["page"]))
    if c["kind"] == "acc":
        return _bytes(sg.decode_acc_workspace_size(*shape))
    return _bytes(sg.decode_fp4_workspace_size(*shape, weights=c["weights"]))


def run(s):
    c = s["c"]
    if not own:
        return {"fetch4": _plain_fetch4, "attn4": _plain_attention, "acc": _plain_attention,
                "evict": _plain_evict}[c["kind"]](c, s)
    if c["kind"] == "fetch4":
        return _own_fetch4(c, s)
    sg = _lib()
    if "ws" not in s:            # a program keeps its workspace from call to call
        s["ws"] = _workspace(sg, c, s["table"].shape[-1])
    if c["kind"] == "attn4":
        sg.sg_decode_attn_fp4(s["q"], s["k4"], s["v4"], s["s4"], s["table"], s["n"], c["page"], s["o"], ws=s["ws"],
                              weight=s["w"], weight_out=s["wout"], decay=s["decay"])
        return s["o"] if s["w"] is None else (s["o"], s["wout"])
    if c["kind"] == "acc":
        sg.sg_decode_attn_acc(s["q"], s["k"], s["v"], s["table"], s["n"], c["page"], s["o"], s["wout"], s["ws"],
                              weight=s["w"], decay=s["decay"])
        return s["o"], s["wout"]
    sg.sg_evict(s["k"], s["v"], s["table"], s["n"], c["page"], s["budget"], s["w"], s["kept"], s["wout"], s["ws"],
                pos=s["pos"], pos_out=s["pout"], sinks=SINKS, recent_from=s["recent"])
    return s["kept"], s["wout"], s["pout"], s["k"], s["v"]


# ------------------------------------------------------------------ what is right

def _exact_round4(x):
    """The nearest representable values in 64 bits, from the definition: the scale from the block's largest magnitude,
    then the nearest of the eight magnitudes (half-way values to the one with the even code)."""
    x = x.double()
    b = x.reshape(-1, BLOCK)
    e = torch.ceil(torch.log2(b.abs().amax(dim=1) / 7.0))
    top = b.abs().amax(dim=1)
    e = torch.where(7.0 * torch.exp2(e - 1) >= top, e - 1, torch.where(7.0 * torch.exp2(e) < top, e + 1, e))
    scale = torch.exp2(e.clamp(-125, 125))[:, None]
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=DEV)
    mid = (grid[1:] + grid[:-1]) / 2
    a = b.abs() / scale
    low, high = torch.searchsorted(mid, a), torch.searchsorted(mid, a, right=True)
    code = torch.where((low != high) & (low % 2 == 1), high, low)     # on a border: of the two, the even one
    return (torch.copysign(grid[code], b) * scale).reshape(x.shape)


def _exact_values4(codes, scales):
    code = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).double()
    m, sign = code % 8, torch.where(code >= 8, -1.0, 1.0).double()
    value = torch.where(m < 2, m / 2, (1 + (m % 2) / 2) * torch.exp2(torch.floor(m / 2) - 1))
    return sign * value * torch.exp2(scales.double() - 127).repeat_interleave(BLOCK, dim=-1)


def exact(c, seed):
    if c["kind"] == "evict":
        return None                           # rows and weights are moved, not computed
    s = prepare(c, seed)
    if c["kind"] == "fetch4":
        src = s["index"].long() + torch.repeat_interleave(s["base"], (s["off"][1:] - s["off"][:-1]).long())
        return _exact_round4(s["k"][src]), _exact_round4(s["v"][src])
    G, d, page = c["Hq"] // c["Hkv"], c["d"], c["page"]
    out, weight = torch.zeros((c["B"], c["Hq"], d), dtype=torch.float64, device=DEV), None
    if s["w"] is not None:
        weight = s["wout"].double()
    for b, n in enumerate(_lens(c)):
        if n == 0:
            continue
        i = torch.arange(n, device=DEV)
        at = s["table"][b].long()[:, i // page] + i % page                     # [Hkv][n]
        if c["kind"] == "acc":
            k, v = s["k"][at].double(), s["v"][at].double()
        else:
            k, v = _exact_values4(s["k4"][at], s["s4"][at, 0]), _exact_values4(s["v4"][at], s["s4"][at, 1])
        q = s["q"][b].double().reshape(c["Hkv"], G, d)
        p = torch.softmax((q @ k.transpose(1, 2).contiguous()) * d ** -0.5, dim=-1)
        out[b] = (p @ v).reshape(c["Hq"], d)
        if weight is not None:
            weight[b, :, :n] = s["decay"] * s["w"][b, :, :n].double() + p.sum(dim=1)
    return out if weight is None else (out, weight)
