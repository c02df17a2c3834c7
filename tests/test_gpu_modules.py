"""The modules' handling of what they are given: devices, alignment, empty batches, weights without a gradient."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mods():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_01255_amd import autograd as ag
    return torch, ag


@pytest.mark.parametrize("compressor", ["rp", "rsvd", "e4m3", "int8"])
def test_a_layer_on_two_devices_is_refused(mods, compressor):
    torch, ag = mods
    x, w = torch.zeros(8, 16, device="cuda"), torch.zeros(24, 16, device="cuda")
    for args in ((x, w.cpu(), None), (x.cpu(), w, None), (x, w, torch.zeros(24))):
        with pytest.raises(ValueError, match="one GPU"):
            ag.CompressedLinearFunction.apply(*args, 8, 0, compressor)
