"""The table's calls take every batch that the header promises: n up to 2^30 tokens, n times d below 2^35."""
import ctypes

import pytest

acc = pytest.importorskip("paper_2605_01255_amd.binding", reason="libacc.so not built")
FINE = (0, -6)   # passed validation (without a GPU the device check refuses)


@pytest.mark.parametrize("dtype", [0, 1], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,d", [(1 << 29, 8), (1 << 30, 8), (1 << 29, 40), (1 << 30, 24), ((1 << 29) - 1, 64), ((1 << 35) // 72 - 1, 72), ((1 << 35) // 264, 264),
                                 ((1 << 35) // 520, 520), ((1 << 35) // 1368, 1368), ((1 << 35) // 2056, 2056), ((1 << 23) - 1, 4096), ((1 << 35) // 4104, 4104),
                                 ((1 << 19) - 1, 1 << 16)])
def test_batches_of_the_promised_range_are_taken(n, d, dtype):
    assert n * d < 1 << 35
    desc = acc.make_embed_desc(n, d, 1 << 21, io_dtype=dtype)
    size = acc.acc_embed_workspace_bytes(desc)
    assert size >= 4 * n
    assert acc._lib.acc_embed_fwd(ctypes.byref(desc), 0x1000, 0x2000, 0x3000, None) in FINE
    assert acc._lib.acc_embed_bwd(ctypes.byref(desc), 0x2000, 0x3000, 0x4000, 0x5000, size, None) in FINE


def test_batches_far_beyond_it_are_refused():
    for n, d in ((1 << 30, 1 << 16), (1 << 30, 4096), ((1 << 30) + 1, 8)):
        desc = acc.make_embed_desc(n, d, 1000)
        assert acc.acc_embed_workspace_bytes(desc) == 0
        assert acc._lib.acc_embed_fwd(ctypes.byref(desc), 0x1000, 0x2000, 0x3000, None) == -2
