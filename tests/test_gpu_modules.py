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


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_slices_that_are_not_aligned_for_the_8_bit_layer(mods, dtype, fmt):
    """An input and a weight that start inside a longer vector, against copies of them."""
    torch, ag = mods
    tdt = getattr(torch, dtype)
    torch.manual_seed(0)
    xs, ws, g = (torch.randn(k, device="cuda").to(tdt) for k in (77 * 72 + 1, 40 * 72 + 3, 77 * 40))
    assert xs[1:].data_ptr() % 16 and ws[3:].data_ptr() % 16
    got = []
    for x, w in ((xs[1:], ws[3:]), (xs[1:].clone(), ws[3:].clone())):
        x, w = x.reshape(7, 11, 72).detach().requires_grad_(), w.reshape(40, 72).detach().requires_grad_()
        y = ag.CompressedLinearFunction.apply(x, w, None, 0, 0, fmt)
        y.backward(g.reshape(7, 11, 40))
        got.append((y.detach(), x.grad, w.grad))
    for a, b in zip(*got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("bias", [False, True])
def test_an_empty_batch_for_the_8_bit_layer(mods, fmt, bias):
    torch, ag = mods
    lin = ag.CompressedLinear(72, 40, bias=bias, compressor=fmt, device="cuda")
    x = torch.zeros(3, 0, 72, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    y = lin(x)
    assert y.shape == (3, 0, 40) and y.dtype == torch.bfloat16
    y.sum().backward()
    assert x.grad.shape == (3, 0, 72) and lin.weight.grad.shape == (40, 72) and not lin.weight.grad.any()
    if bias:
        assert lin.bias.grad.shape == (40,) and not lin.bias.grad.any()
    with torch.no_grad():
        lin.weight.grad = None
    lin(x.detach()).sum().backward()
    assert not lin.weight.grad.any()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_no_checkpoint_is_kept_for_a_gradient_that_nobody_forms(mods, fmt, monkeypatch):
    """A frozen weight's layer keeps the weight alone, an evaluation pass makes no checkpoint; outputs and input gradients stay."""
    torch, ag = mods
    torch.manual_seed(0)
    lin = ag.CompressedLinear(136, 264, compressor=fmt, device="cuda")
    x, g = (torch.randn(77, k, device="cuda", dtype=torch.bfloat16) for k in (136, 264))
    a = x.clone().requires_grad_()
    y = lin(a)
    y.backward(g)
    db = lin.bias.grad
    lin.bias.grad = None

    def none(*args, **kw):
        raise AssertionError("a checkpoint was made")

    monkeypatch.setattr(ag.acc, "alloc_act8", none)
    lin.weight.requires_grad_(False)
    b, saved = x.clone().requires_grad_(), []
    with torch.autograd.graph.saved_tensors_hooks(lambda z: (saved.append((tuple(z.shape), z.dtype)), z)[1], lambda z: z):
        y2 = lin(b)
    assert saved == [((264, 136), torch.bfloat16)]
    y2.backward(g)
    assert torch.equal(y, y2) and torch.equal(a.grad, b.grad) and torch.equal(db, lin.bias.grad)
    lin.weight.requires_grad_(True)
    with torch.no_grad():
        assert torch.equal(y, lin(x))


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_the_cross_entropys_input_gradient_holds_no_more_than_it_is(mods, dtype):
    """Of rows far apart: the gradient's memory is that of its elements, its bits those for dense rows."""
    torch, ag = mods
    torch.manual_seed(0)
    tdt = getattr(torch, dtype)
    wide, w = torch.randn(50, 4096, device="cuda").to(tdt), torch.randn(301, 72, device="cuda").to(tdt)
    t = torch.randint(0, 301, (50,), device="cuda")
    got = []
    for x in (wide[:, :72], wide[:, :72].contiguous()):
        x = x.detach().requires_grad_()
        (dx,) = torch.autograd.grad(ag.LinearCrossEntropyFunction.apply(x, w, t).sum(), x)
        assert dx.is_contiguous() and dx.untyped_storage().nbytes() == 50 * 72 * dx.element_size()
        got.append(dx)
    assert torch.equal(*got)
