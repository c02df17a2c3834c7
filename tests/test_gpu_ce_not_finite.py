"""What is not finite in the cross entropy's backward pass: in rows that have no gradient it reaches nothing, in others everything."""
import pytest

pytestmark = pytest.mark.gpu

from test_gpu_ce import Case, acc  # noqa: F401  (acc: the fixture)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,piece", [(40, 0), (333, 256), (1500, 0)])
@pytest.mark.parametrize("ignored", [0.0, 0.4])
def test_rows_whose_target_lies_beyond_the_vocabulary_reach_no_gradient(acc, n, piece, ignored, dtype):  # noqa: F811
    """The gradients are those of the same tokens without a loss, bit for bit, whatever the rows, their losses and their gradients hold."""
    import torch
    c = Case(acc, n, 136, 700, dtype, piece=piece, ignored=ignored)
    beyond = torch.tensor([0, 7, 31, n // 2, n - 1], device="cuda")
    c.targets[beyond] = -1
    clean = c.backward(c.forward()[1])
    c.targets[beyond] = torch.tensor([700, 701, 1 << 31, 1 << 40, (1 << 63) - 1], device="cuda")
    c.X[beyond[:4], torch.arange(4, device="cuda")] = torch.tensor([float("nan"), float("inf"), -float("inf"), 3e38], device="cuda").to(c.tdt)
    c.dloss[beyond[1:3]] = torch.tensor([float("nan"), float("inf")], device="cuda")
    loss, stats = c.forward()
    assert bool(torch.isnan(loss[beyond]).all()) and bool(torch.isfinite(loss[c.targets < 700]).all())
    for a, b in zip(clean, c.backward(stats)):
        assert torch.equal(a, b)
    assert not c.backward(stats)[0][beyond].any()
