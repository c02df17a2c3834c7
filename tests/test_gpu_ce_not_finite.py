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


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,piece", [(40, 0), (333, 256)])
@pytest.mark.parametrize("what", ["infinite logit", "NaN in its row", "nothing but minus infinity"])
def test_a_log_sum_exp_that_is_not_finite_makes_its_gradients_nan(acc, n, piece, what, dtype):  # noqa: F811
    """One token's row; the input gradients of the others stay as they are, bit for bit."""
    import torch
    c = Case(acc, n, 64, 600, dtype, piece=piece)
    c.X[:, 0] = 0.0
    c.W[:, 0] = 0.0
    c.targets[9] = 3
    clean = c.backward(c.forward()[1])
    if what == "infinite logit":        # of column 11 alone; its other logits are finite
        c.X[9, 0] = 3e38
        c.W[11, 0] = 16.0
    elif what == "NaN in its row":
        c.X[9, 5] = float("nan")
    else:
        c.X[9, 0] = -3e38
        c.W[:, 0] = 16.0
    loss, stats = c.forward()
    assert not bool(torch.isfinite(stats[0, 9])) and not bool(torch.isfinite(loss[9])) and int((~torch.isfinite(loss)).sum()) == 1
    dX, dW = c.backward(stats)
    assert bool(torch.isnan(dX[9]).all()) and bool(torch.isnan(dW).all())
    if what == "NaN in its row":        # W is the same
        others = torch.arange(n, device="cuda") != 9
        assert torch.equal(dX[others], clean[0][others])
    assert int(torch.isnan(dX).any(1).sum()) == 1
