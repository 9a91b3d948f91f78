"""4-bit rows, accumulated weights and eviction without a GPU: the plain
definitions against hand-worked values, and the host checks of the calls."""
import ctypes

import numpy as np
import pytest
import torch

import cache_ref as ref
from paper_2607_28150_amd import smartgen as sg

P = ctypes.c_void_p(16)   # never dereferenced: every call below fails validation first


@pytest.fixture(scope="module")
def lib():
    return sg.load()


def test_encode_by_hand():
    x = np.zeros((2, 32))
    x[0, :10] = [6, -6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.0]
    x[1, :4] = [7, 3.5, 7.0001, 0.5]
    codes, scales = ref.encode(x)
    assert scales.ravel().tolist() == [127, 128]        # 7.0001 passes 7: the next scale
    v = ref.decode(codes, scales)
    assert v[0, :10].tolist() == [6, -6, 0, 1, 1, 2, 2, 4, 4, 0]
    assert v[1, :4].tolist() == [8, 4, 8, 0]            # 0.5 / 2 is half-way: the even code
    codes, scales = ref.encode(np.array([[7.0] + [0.5] * 31]))
    assert scales.item() == 127 and ref.decode(codes, scales)[0, :2].tolist() == [6, 0.5]
    assert ref.encode(np.zeros((1, 32)))[1].item() == 2
    assert ref.encode(np.full((1, 32), 3.4e38))[1].item() == 252
    assert np.isnan(ref.decode(*ref.encode(np.array([[np.inf] + [1.0] * 31])))).all()


def test_encode_is_nearest():
    r = np.random.default_rng(3)
    x = r.standard_normal((50, 64)) * np.exp(8 * r.standard_normal((50, 1)))
    codes, scales = ref.encode(x)
    got = ref.decode(codes, scales).reshape(50, 2, 32)
    s = 2.0 ** (scales.astype(float) - 127)[..., None]
    grid = np.concatenate([ref.MAGNITUDES, -ref.MAGNITUDES])
    best = np.abs(x.reshape(50, 2, 32, 1) - grid * s[..., None]).min(axis=-1)
    assert np.array_equal(np.abs(x.reshape(50, 2, 32) - got), best)
    top = np.abs(x.reshape(50, 2, 32)).max(axis=-1)
    assert (top <= 7 * s[..., 0]).all() and (top > 3.5 * s[..., 0]).all()


def test_evict_by_hand():
    w = np.array([5, 1, 0, 0, 9, 3, np.nan, 2], np.float32)
    k, moves, wo, po = ref.evict(8, 4, w, np.arange(8), 0, None)
    assert k == 4 and moves == [(1, 4), (2, 5), (3, 7)]
    assert wo.tolist() == [5, 9, 3, 2, 0, 0, 0, 0] and po.tolist() == [0, 4, 5, 7, -1, -1, -1, -1]
    k, moves, wo, po = ref.evict(8, 3, w, np.arange(8), 1, 7)      # rows 0 and 7 are guarded
    assert moves == [(1, 4), (2, 7)] and po[:3].tolist() == [0, 4, 7]
    assert ref.evict(3, 5, w, np.arange(8), 0, None)[1] == []
    assert ref.evict(4, 1, np.zeros(4), np.arange(4), 0, None)[3].tolist() == [0, -1, -1, -1]


def _err(lib):
    return lib.sg_last_error().decode()


def test_fetch_fp4_rejections(lib):
    def call(src=1, dst=2, d=128, rows=1, total=5, base=P, s_src=None, page=16, pages=1, s_pool=P, k=P, src_rows=10):
        return lib.sg_fetch_fp4(None, src, dst, d, rows, P, total, P, None, base, src_rows, k, P, s_src, P, page, pages,
                                P, P, P, s_pool, 10)
    assert call(src=1, dst=0) == sg.SG_EINVAL and "sg_fetch" in _err(lib)
    assert call(src=7) == sg.SG_EINVAL and "dtype" in _err(lib)
    assert call(d=96) == sg.SG_EUNSUPPORTED
    assert call(page=0) == sg.SG_EINVAL and call(pages=0) == sg.SG_EINVAL
    assert call(rows=-1) == sg.SG_EINVAL and call(total=-1) == sg.SG_EINVAL and call(src_rows=-1) == sg.SG_EINVAL
    assert call(base=None) == sg.SG_EINVAL and "null" in _err(lib)
    assert call(s_pool=None) == sg.SG_EINVAL and "scales" in _err(lib)
    assert call(s_src=P) == sg.SG_EINVAL
    assert call(src=2, dst=1, s_pool=None) == sg.SG_EINVAL
    assert call(k=ctypes.c_void_p(24)) == sg.SG_EINVAL and "aligned" in _err(lib)
    assert call(rows=0) == sg.SG_OK and call(total=0) == sg.SG_OK


def test_decode_fp4_rejections(lib):
    def call(dt=1, B=1, Hq=32, Hkv=8, d=128, scale=0.1, q=P, page=16, pages=4, win=None, decay=1.0, wout=None,
             stride=64, ws=P, wsb=1 << 30, pool=10):
        return lib.sg_decode_attn_fp4(None, dt, B, Hq, Hkv, d, scale, q, P, P, P, pool, P, P, page, pages, P, win, decay,
                                      wout, stride, ws, wsb)
    assert call(dt=2) == sg.SG_EINVAL and "dtype" in _err(lib)
    assert call(Hq=6, Hkv=4) == sg.SG_EINVAL
    assert call(Hq=136) == sg.SG_EUNSUPPORTED and "group" in _err(lib)
    assert call(d=96) == sg.SG_EUNSUPPORTED
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert call(scale=scale) == sg.SG_EINVAL and "scale" in _err(lib)
    assert call(page=0) == sg.SG_EINVAL and call(page=1 << 16, pages=1 << 16) == sg.SG_EINVAL
    assert call(pool=1 << 31) == sg.SG_EUNSUPPORTED
    assert call(q=None) == sg.SG_EINVAL and "null" in _err(lib)
    assert call(q=ctypes.c_void_p(18)) == sg.SG_EINVAL and "aligned" in _err(lib)
    assert call(win=P) == sg.SG_EINVAL and "weight_out" in _err(lib)
    assert call(wout=P, stride=63) == sg.SG_EINVAL
    assert call(wout=P, decay=1.5) == sg.SG_EINVAL and call(wout=P, decay=float("nan")) == sg.SG_EINVAL
    assert call(wout=P, wsb=100) == sg.SG_EWORKSPACE
    assert call(pages=1024, ws=None, wsb=0) == sg.SG_EWORKSPACE
    assert call(B=0) == sg.SG_OK
    assert sg.decode_fp4_workspace_size(1, 32, 8, 128, 1, 16) == 0          # one split, no weights
    assert sg.decode_fp4_workspace_size(1, 32, 8, 128, 1, 16, weights=True) == 32 * (130 + 32) * 4
    assert sg.decode_fp4_workspace_size(0, 32, 8, 128, 1, 16, weights=True) == 0


def test_decode_acc_rejections(lib):
    def call(dt=1, Hq=32, d=128, scale=0.1, win=P, decay=1.0, wout=P, stride=64, wsb=1 << 30, ws=P, pages=4):
        return lib.sg_decode_attn_acc(None, dt, 1, Hq, 8, d, scale, P, P, P, 10, P, P, 16, pages, P, win, decay, wout,
                                      stride, ws, wsb)
    assert call(dt=2) == sg.SG_EINVAL
    assert call(Hq=24) == sg.SG_EUNSUPPORTED and "group" in _err(lib)
    assert call(d=80) == sg.SG_EUNSUPPORTED
    assert call(scale=-1.0) == sg.SG_EINVAL
    assert call(wout=None) == sg.SG_EINVAL and "weight_out" in _err(lib)
    assert call(stride=63) == sg.SG_EINVAL
    assert call(decay=-0.1) == sg.SG_EINVAL and "decay" in _err(lib)
    assert call(wsb=64) == sg.SG_EWORKSPACE
    assert call(ws=ctypes.c_void_p(8)) == sg.SG_EINVAL
    assert call(pages=0) == sg.SG_EINVAL
    assert sg.decode_acc_workspace_size(1, 32, 8, 128, 1, 16) == 32 * (130 + 32) * 4


def test_evict_rejections(lib):
    def call(dt=1, units=2, d=128, k=P, s=None, page=16, pages=4, budget=P, w=P, pos=P, stride=64, sinks=4, po=P, ws=P,
             wsb=1 << 20):
        return lib.sg_evict(None, dt, units, d, k, P, s, 100, P, P, page, pages, budget, w, pos, stride, sinks, P, P, P,
                            po, ws, wsb)
    assert call(dt=3) == sg.SG_EINVAL
    assert call(units=-1) == sg.SG_EINVAL and call(sinks=-1) == sg.SG_EINVAL
    assert call(d=32) == sg.SG_EUNSUPPORTED
    assert call(page=0) == sg.SG_EINVAL
    assert call(pages=5121, stride=1 << 20) == sg.SG_EUNSUPPORTED       # 81,936 rows
    assert call(stride=63) == sg.SG_EINVAL
    assert call(budget=None) == sg.SG_EINVAL and "null" in _err(lib)
    assert call(s=P) == sg.SG_EINVAL and call(dt=2) == sg.SG_EINVAL
    assert call(pos=None) == sg.SG_EINVAL and call(po=None) == sg.SG_EINVAL
    assert call(k=ctypes.c_void_p(8)) == sg.SG_EINVAL
    assert call(wsb=100) == sg.SG_EWORKSPACE and call(ws=None, wsb=0) == sg.SG_EWORKSPACE
    assert call(units=0) == sg.SG_OK
    assert sg.evict_workspace_size(2, 4, 16) == 2 * (32 * 8 + 4)


def test_binding_rejections():
    u8, i32 = (lambda *s: torch.zeros(s, dtype=torch.uint8)), (lambda *s: torch.zeros(s, dtype=torch.int32))
    q, table, n, out = torch.zeros(1, 8, 64), i32(1, 8, 2), i32(1, 8), torch.zeros(1, 8, 64)
    with pytest.raises(ValueError, match="scales"):
        sg.sg_decode_attn_fp4(q, u8(4, 32), u8(4, 32), None, table, n, 16, out)
    with pytest.raises(ValueError, match="codes"):
        sg.sg_decode_attn_fp4(q, torch.zeros(4, 64), torch.zeros(4, 64), None, table, n, 16, out)
    with pytest.raises(ValueError, match="rows"):
        sg.sg_decode_attn_fp4(q, u8(4, 32), u8(4, 32), u8(4, 2, 2), table, n, 16, out, weight_out=torch.zeros(1, 8, 31))
    with pytest.raises(ValueError, match="share"):
        sg.sg_decode_attn_acc(q, torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(4, 64, dtype=torch.bfloat16),
                              table, n, 16, out, torch.zeros(1, 8, 32), None)
    with pytest.raises(ValueError, match="together"):
        sg.sg_evict(torch.zeros(4, 64), torch.zeros(4, 64), table, n, 16, n, torch.zeros(8, 32), n,
                    torch.zeros(8, 32), None, pos=i32(8, 32))
    with pytest.raises(ValueError, match="smaller"):
        sg.sg_fetch_fp4(i32(2), 1, None, None, torch.zeros(1, dtype=torch.int64), torch.zeros(4, 64), torch.zeros(4, 64),
                        i32(1, 1), 16, i32(1), u8(4, 32), u8(4, 32), s_pool=u8(3, 2, 2))
    with pytest.raises(ValueError, match="int32"):
        sg.sg_fetch_fp4(i32(2), 1, torch.zeros(1, dtype=torch.int64), None, torch.zeros(1, dtype=torch.int64),
                        torch.zeros(4, 64), torch.zeros(4, 64), i32(1, 1), 16, i32(1), u8(4, 32), u8(4, 32),
                        s_pool=u8(4, 2, 2))
