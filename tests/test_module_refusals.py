"""What the modules refuse before anything touches a GPU: the calls here are made on the CPU, and none of them gets as far as memory."""
import pytest

torch = pytest.importorskip("torch")
ag = pytest.importorskip("paper_2605_01255_amd.autograd", reason="libacc.so not built")


@pytest.mark.parametrize("width", [8, 32, 15, 0])
def test_features_that_are_not_the_matrixs(width):
    """Rows twice as wide are not two tokens each: there are targets for half of those."""
    x, w, t = torch.zeros(4, width), torch.zeros(50, 16), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="features"):
        ag.LinearCrossEntropyFunction.apply(x, w, t)
    m = ag.LinearCrossEntropy(16, 50, dtype=torch.float32)
    with pytest.raises(ValueError, match="features"):
        m(x, t)


@pytest.mark.parametrize("compressor", ["rp", "rsvd", "e4m3", "int8"])
def test_layers_that_are_not_on_a_gpu(compressor):
    """A pointer into host memory, or into another GPU's, is none that a kernel may be given."""
    x, w = torch.zeros(8, 16), torch.zeros(24, 16)
    with pytest.raises(ValueError, match="one GPU"):
        ag.CompressedLinearFunction.apply(x, w, None, 8, 0, compressor)
    with pytest.raises(ValueError, match="one GPU"):
        ag.CompressedLinearFunction.apply(x, w.to("meta"), None, 8, 0, compressor)
    with pytest.raises(ValueError):
        ag.LinearCrossEntropyFunction.apply(x, w, torch.zeros(8, dtype=torch.int64))
    with pytest.raises(ValueError):
        ag.CompressedSwiGLUFunction.apply(x)


def test_low_rank_compressors_need_a_rank():
    for compressor in ("rp", "rsvd"):
        with pytest.raises(TypeError, match="rank"):
            ag.CompressedLinear(64, 32, compressor=compressor)
        for rank in (0, -8):
            with pytest.raises(ValueError, match="rank"):
                ag.CompressedLinear(64, 32, rank, compressor=compressor)
        assert ag.CompressedLinear(64, 32, 16, compressor=compressor).rank == 16
    with pytest.raises(TypeError, match="rank"):
        ag.CompressedLinear(64, 32)
    for compressor in ("e4m3", "int8"):
        assert ag.CompressedLinear(64, 32, compressor=compressor).rank == 0
