"""Scales and caps whose float constants of a kernel are not finite are refused: a score of zero would not be a number."""
import ctypes

import pytest

acc = pytest.importorskip("paper_2605_01255_amd.binding", reason="libacc.so not built")
FINE = (0, -6)   # passed validation (without a GPU the device check refuses)


def _fwd(desc):
    return acc._lib.acc_attn_fwd(ctypes.byref(desc), 0x1000, 0x2000, 0x3000, None, None, None, 0x4000, 0x5000, 0x6000, 1 << 40, None)


def _bwd(desc):
    return acc._lib.acc_attn_bwd(ctypes.byref(desc), 0x1000, 0x2000, 0x3000, None, None, None, 0x4000, 0x5000, 0x7000, 0x8000, 0x9000, 0xA000, 0x6000,
                                 1 << 40, None)


@pytest.mark.parametrize("kw", [dict(scale=3e38), dict(cap=3e38), dict(cap=1.3e38), dict(cap=1e-40), dict(cap=1e-45), dict(scale=1e20, cap=1e-19),
                                dict(scale=1.0, cap=5e-39)], ids=str)
@pytest.mark.parametrize("dtype", [acc.ACC_BF16, acc.ACC_F32])
def test_constants_beyond_float_are_refused(kw, dtype):
    d = acc.make_attn_desc(100, 8, 2, 64, io_dtype=dtype, **kw)
    assert _fwd(d) == -1 and _bwd(d) == -1 and acc.acc_attn_workspace_bytes(d, True) == 0


@pytest.mark.parametrize("kw", [dict(scale=1e38), dict(cap=1e37), dict(cap=1e-30), dict(scale=1e-30, cap=1e-40), dict(scale=1e30, cap=1e30)], ids=str)
def test_far_ones_are_not(kw):
    d = acc.make_attn_desc(100, 8, 2, 64, **kw)
    assert _fwd(d) in FINE and _bwd(d) in FINE
