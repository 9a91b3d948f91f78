"""Limits of the attention calls with weights, of eviction and of their binding, checked
before anything is enqueued (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2607_28150_amd import smartgen as sg

P = ctypes.c_void_p(16)   # never dereferenced: every call below is refused first


@pytest.fixture(scope="module")
def lib():
    return sg.load()


# A launch's dimension holds 2^32 - 1 threads: units times the threads that each takes
# in the attention (4-bit 64, float 256) or in the launch that joins states (128 or more).
@pytest.mark.parametrize("B,Hkv", [(33_554_432, 1), (4_194_304, 8), (60_000_000, 1)])
def test_units_with_weights_4bit(lib, B, Hkv):
    for dt, d in ((0, 64), (1, 128)):
        rc = lib.sg_decode_attn_fp4(None, dt, B, Hkv, Hkv, d, 0.1, P, P, P, P, 10, P, P, 16, 2, P, None, 1.0, P, 32, P,
                                    1 << 62)
        assert rc == sg.SG_EUNSUPPORTED and "units" in lib.sg_last_error().decode()


@pytest.mark.parametrize("B", [16_777_216, 20_000_000, 33_554_432])
def test_units_float(lib, B):
    for dt, d in ((0, 64), (1, 128)):
        rc = lib.sg_decode_attn_acc(None, dt, B, 1, 1, d, 0.1, P, P, P, 10, P, P, 16, 2, P, None, 1.0, P, 32, P, 1 << 62)
        assert rc == sg.SG_EUNSUPPORTED and "units" in lib.sg_last_error().decode()
        rc = lib.sg_decode_attn(None, dt, B, 1, 1, d, 0.1, P, P, P, 10, P, P, 16, 2, P, P, 1 << 62)
        assert rc == sg.SG_EUNSUPPORTED and "units" in lib.sg_last_error().decode()


def test_units_of_many_states(lib):
    """Long sets in pages of one row: several hundred states per unit, which more threads join."""
    rc = lib.sg_decode_attn_acc(None, 1, 5_000_000, 1, 1, 128, 0.1, P, P, P, 10, P, P, 1, 1 << 18, P, None, 1.0, P, 1 << 18,
                                P, 1 << 62)
    assert rc == sg.SG_EUNSUPPORTED and "units" in lib.sg_last_error().decode()


def test_binding_refuses_empty_axes():
    """Rows of no channels and tables of no pages: ValueError, as for any other shape that does not fit."""
    f, u8 = torch.zeros, (lambda *s: torch.zeros(s, dtype=torch.uint8))
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    base = torch.zeros(1, dtype=torch.int64)
    with pytest.raises(ValueError, match="channels"):
        sg.sg_fetch_fp4(i32(2), 1, None, None, base, f(4, 0), f(4, 0), i32(1, 1), 16, i32(1), u8(4, 0), u8(4, 0),
                        s_pool=u8(4, 2, 0))
    for pools, s in ((f(4, 0), None), (u8(4, 0), u8(4, 2, 0))):
        with pytest.raises(ValueError, match="channels"):
            sg.sg_evict(pools, pools, i32(1, 2), i32(1), 16, i32(1), f(1, 32), i32(1), f(1, 32), None, s_pool=s)
    with pytest.raises(ValueError, match="page"):
        sg.sg_evict(f(4, 64), f(4, 64), i32(2, 0), i32(2), 16, i32(2), f(2, 32), i32(2), f(2, 32), None)
    with pytest.raises(ValueError, match="channels"):
        sg.sg_decode_attn_acc(f(1, 8, 0), f(4, 0), f(4, 0), i32(1, 8, 2), i32(1, 8), 16, f(1, 8, 0), f(1, 8, 32), None)
