"""Sizes at the ends of what the header allows for the 8-bit checkpoints, before anything touches a GPU."""
import ctypes

import pytest

acc = pytest.importorskip("paper_2605_01255_amd.binding", reason="libacc.so not built")
FINE = (0, -6)   # passed validation (without a GPU the device check refuses)


def _pack(n, c, ld=0):
    return acc._lib.acc_act8_pack(ctypes.byref(acc.make_act8_desc(n, c, ldx=ld)), 0x1000, 0x2000, 0x3000, None)


def _gated(n, f, ldg=0, ldh=0):
    d = ctypes.byref(acc.make_gated_desc(n, f, ldg=ldg, ldh=ldh))
    a = acc._lib.acc_gated_fwd_act8(d, *range(0x1000, 0x8000, 0x1000), None)
    b = acc._lib.acc_gated_bwd_act8(d, *range(0x1000, 0x9000, 0x1000), None)
    assert (a in FINE) == (b in FINE)
    return a


@pytest.mark.parametrize("call", [_pack, _gated])
def test_elements_of_one_call(call):
    # n (in whole blocks) times c (in whole 64 channels) below 2^37
    assert call(1 << 30, 128) == -2 and call(1 << 30, 120) == -2 and call((1 << 30) - 31, 128) == -2
    assert call((1 << 30) - 64, 128) in FINE and call(1 << 30, 64) in FINE and call(1 << 16, (1 << 21) - 64) in FINE
    assert call(1 << 16, 1 << 21) == -2


def test_row_strides():
    assert _pack(4, 64, 1 << 24) in FINE and _pack(4, 64, (1 << 24) + 8) == -2
    assert _gated(4, 64, 1 << 24, 1 << 24) in FINE and _gated(4, 64, ldg=(1 << 24) + 8) == -2 and _gated(4, 64, ldh=(1 << 24) + 8) == -2
