"""Limits of the attention calls with weights, of eviction and of their binding, checked
before anything is enqueued (no GPU needed)."""
import ctypes

import pytest

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
