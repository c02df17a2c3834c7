"""The modules over 8-bit checkpoints and the cross entropy, alone and as one training step.

Tolerances: half a step of bfloat16 is 2^-8 of a value, of float32 2^-24; a float sum of k terms is off by at most k 2^-24 of the
sum of magnitudes.  Each operator's gradient is held to its formula for the gradient that arrived at it in the very pass."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from oracle import train_oracle as orc

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def mods():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_01255_amd import autograd as ag
    return torch, ag


def _f64(t):
    return t.detach().cpu().double().numpy()


def _product_close(got, a, b, half, extra=0.0):
    """got = a @ b with operands known exactly."""
    want = a @ b
    bound = half * 1.01 * np.abs(want) + (a.shape[1] + 8) * U * (np.abs(a) @ np.abs(b)) + extra
    off = np.abs(_f64(got) - want)
    assert np.all(off <= bound), float(np.max(off / bound))


def _kept(x, fmt):
    return orc.act8_unpack(*orc.act8_pack(x, fmt), fmt)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_linear_module_keeps_the_checkpoint_alone(mods, dtype, fmt):
    torch, ag = mods
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    torch.manual_seed(0)
    lin = ag.CompressedLinear(136, 264, bias=True, compressor=fmt, device="cuda", dtype=tdt)
    x = torch.randn(3, 41, 136, device="cuda", dtype=tdt, requires_grad=True)
    saved = []
    with torch.autograd.graph.saved_tensors_hooks(lambda z: (saved.append((tuple(z.shape), z.dtype)), z)[1], lambda z: z):
        y = lin(x)
    assert ((123, 136), torch.uint8) in saved and ((4, 136), torch.uint8) in saved
    assert all(entry == ((264, 136), tdt) or entry[1] == torch.uint8 for entry in saved)
    g = torch.randn_like(y) * 0.1
    y.backward(g)
    X, W, dY = _f64(x).reshape(-1, 136), _f64(lin.weight), _f64(g).reshape(-1, 264)
    _product_close(x.grad.reshape(-1, 136), dY, W, HALF[dtype])
    _product_close(lin.weight.grad, dY.T, _kept(X, fmt), HALF[dtype])
    db = dY.sum(0)
    assert np.all(np.abs(_f64(lin.bias.grad) - db) <= HALF[dtype] * 1.01 * np.abs(db) + 123 * U * np.abs(dY).sum(0))
    # gradients that nobody asks for are not formed
    w = lin.weight.detach()
    y = ag.CompressedLinearFunction.apply(x.detach().requires_grad_(), w, None, 0, 0, fmt)
    y.sum().backward()
    y = ag.CompressedLinearFunction.apply(x.detach(), w.requires_grad_(), None, 0, 0, fmt)
    y.backward(g)
    assert torch.equal(w.grad, lin.weight.grad)


def test_refusals(mods):
    torch, ag = mods
    x = torch.randn(4, 64, device="cuda", dtype=torch.bfloat16)
    w = torch.randn(32, 64, device="cuda", dtype=torch.bfloat16)
    t = torch.zeros(4, dtype=torch.int64, device="cuda")
    with pytest.raises(ValueError):
        ag.CompressedLinearFunction.apply(x, w, None, 0, 0, "int4")
    with pytest.raises(ValueError):
        ag.CompressedLinear(64, 32, compressor="int8", factored_grad=True, device="cuda")(x)
    with pytest.raises(ValueError):
        ag.CompressedSwiGLU("fp8")
    with pytest.raises(TypeError):
        ag.CompressedSwiGLUFunction.apply(x.half())
    with pytest.raises(ValueError):
        ag.CompressedSwiGLUFunction.apply(x[:, :33])
    with pytest.raises(TypeError):
        ag.LinearCrossEntropyFunction.apply(x, w.float(), t)
    with pytest.raises(TypeError):
        ag.LinearCrossEntropyFunction.apply(x, w, t.int())
    with pytest.raises(TypeError):
        ag.LinearCrossEntropyFunction.apply(x, w, t[:3])
    with pytest.raises(ValueError):
        ag.LinearCrossEntropyFunction.apply(x, w, t.cpu())
    with pytest.raises(ValueError):
        ag.LinearCrossEntropy(64, 32, reduction="max")
    from paper_2605_01255_amd.binding import AccError
    with pytest.raises(AccError):
        ag.CompressedSwiGLU()(torch.randn(4, 24, device="cuda", dtype=torch.bfloat16))     # 12 channels
    with pytest.raises(AccError):
        ag.LinearCrossEntropyFunction.apply(x[:, :60].contiguous(), w[:, :60].contiguous(), t)


@pytest.mark.parametrize("n", [0, 1, 77])
def test_gated_module(mods, n):
    torch, ag = mods
    torch.manual_seed(1)
    wide = torch.randn(n, 600, device="cuda", dtype=torch.float32)
    for x in (wide[:, :528], wide[:, 8:536].contiguous(), wide.t().contiguous().t()[:, :528]):
        x = x.detach().requires_grad_()
        h = ag.CompressedSwiGLU("e4m3")(x)
        g = torch.randn(n, 528, device="cuda")[:, :264]
        h.backward(g)
        G, V, dH = _f64(x)[:, :264], _f64(x)[:, 264:], _f64(g)
        want = orc.gated(G, V)
        room = lambda x: (np.abs(x) + 8) * 2.0 ** -22  # noqa: E731  (sigmoid's error, relative, with the operations after it)
        assert h.shape == (n, 264) and np.all(np.abs(_f64(h) - want) <= (room(G) + U) * np.abs(want))
        if n:
            Gq, Vq = _kept(G, "e4m3"), _kept(V, "e4m3")
            dg, du = orc.gated_bwd(dH, Gq, Vq)
            s = 1 / (1 + np.exp(-Gq))
            got = _f64(x.grad)
            assert np.all(np.abs(got[:, 264:] - du) <= (room(Gq) + U) * np.abs(du))
            assert np.all(np.abs(got[:, :264] - dg) <= (room(Gq) + U) * np.abs(dH * Vq) * s * (1 + np.abs(Gq) * (1 - s)))
        else:
            assert x.grad.shape == (0, 528)


@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
def test_cross_entropy_module_against_torch(mods, reduction):
    """float32 against torch's own in float64: 2^-14 of the largest value is over a thousand roundings."""
    torch, ag = mods
    torch.manual_seed(2)
    m = ag.LinearCrossEntropy(72, 333, ignore_index=5, reduction=reduction, device="cuda", dtype=torch.float32)
    x = torch.randn(4, 31, 72, device="cuda", requires_grad=True)
    t = torch.randint(0, 333, (4, 31), device="cuda")
    t[0, :9] = 5
    loss = m(x, t)
    (loss if reduction != "none" else (loss * 0.5).sum()).backward()
    x64, w64 = x.detach().double().requires_grad_(), m.weight.detach().double().requires_grad_()
    ref = torch.nn.functional.cross_entropy((x64 @ w64.t()).reshape(-1, 333), t.reshape(-1), ignore_index=5, reduction=reduction)
    (ref if reduction != "none" else (ref * 0.5).sum()).backward()
    for a, b in ((loss, ref.reshape(loss.shape)), (x.grad, x64.grad), (m.weight.grad, w64.grad)):
        assert float((a.detach().double() - b.detach()).abs().max()) <= 2.0 ** -14 * float(b.detach().abs().max())


def test_cross_entropy_of_nothing_and_of_strided_rows(mods):
    torch, ag = mods
    w = torch.randn(50, 64, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    x = torch.randn(0, 64, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    loss = ag.LinearCrossEntropyFunction.apply(x, w, torch.zeros(0, dtype=torch.int64, device="cuda"))
    loss.sum().backward()
    assert loss.shape == (0,) and x.grad.shape == (0, 64) and not w.grad.any()
    wide = torch.randn(9, 96, device="cuda", dtype=torch.bfloat16)
    t = torch.randint(0, 50, (9,), device="cuda")
    got = []
    for view in (wide[:, :64], wide[:, :64].contiguous()):
        view = view.detach().requires_grad_()
        w.grad = None
        loss = ag.LinearCrossEntropyFunction.apply(view, w, t)
        loss.sum().backward()
        got.append((loss.detach(), view.grad, w.grad))
    for a, b in zip(*got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("kinds", [("int8", "int8", "e4m3"), ("rp", "e4m3", "int8"), ("e4m3", "int8", "rsvd")])
def test_a_training_step(mods, kinds):
    """The MLP of a decoder layer with its residual and the loss, on another stream than the default one.  What each operator gives
    back is held to its formula for what arrived at it."""
    torch, ag = mods
    up, act, down = kinds
    torch.manual_seed(3)
    d, f, v, n = 192, 264, 517, 200
    rank = lambda c: 64 if c in ("rp", "rsvd") else 0  # noqa: E731
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        l1 = ag.CompressedLinear(d, 2 * f, rank(up), bias=False, compressor=up, device="cuda")
        glu = ag.CompressedSwiGLU(act)
        l2 = ag.CompressedLinear(f, d, rank(down), bias=False, compressor=down, device="cuda")
        with torch.no_grad():
            l1.weight.mul_(5.0)
            l2.weight.mul_(5.0)
        ce = ag.LinearCrossEntropy(d, v, device="cuda")
        x = torch.randn(4, n // 4, d, device="cuda", dtype=torch.bfloat16, requires_grad=True)
        t = torch.randint(0, v, (4, n // 4), device="cuda")
        t[:, :7] = -100
        gu = l1(x)
        h = glu(gu)
        y = l2(h)
        out = x + y
        for z in (gu, h, y, out):
            z.retain_grad()
        loss = ce(out, t)
        loss.backward()
    stream.synchronize()
    flat = lambda z: _f64(z).reshape(-1, z.shape[-1])  # noqa: E731
    X, GU, H, O = flat(x), flat(gu), flat(h), flat(out)
    dGU, dH, dY, dO = (flat(z.grad) for z in (gu, h, y, out))
    T = t.cpu().numpy().reshape(-1)
    counted = T >= 0
    # the loss and its gradients
    want, lse = orc.linear_ce(O, _f64(ce.weight), T)
    want = want[counted].mean()
    assert abs(float(loss.detach()) - want) <= 2.0 ** -18 * abs(want)   # float sums of 192 and of a few hundred terms of this size
    g = np.where(counted, 1.0 / counted.sum(), 0.0)
    dx, dw = orc.linear_ce_bwd(O, _f64(ce.weight), T, g)
    p = np.exp(O @ _f64(ce.weight).T - lse[:, None])
    onehot = np.zeros_like(p)
    onehot[np.arange(n)[counted], T[counted]] = 1
    adz = np.abs(p - onehot) * g[:, None]
    room = (2.0 ** -8 + 2.0 ** -14) * adz       # dz as an operand; 2^-14: logits of float sums, exponentials
    assert np.all(np.abs(dO - dx) <= (room @ np.abs(_f64(ce.weight))) * 1.01 + 2.0 ** -8 * np.abs(dx) * 1.01 + 1e-12)
    assert np.all(np.abs(_f64(ce.weight.grad) - dw) <= (room.T @ np.abs(O)) * 1.01 + 2.0 ** -8 * np.abs(dw) * 1.01 + 1e-12)
    assert not dO[~counted].any()
    # the linears: input gradients exact, weight gradients from what they kept
    _product_close(h.grad.reshape(-1, f), dY, _f64(l2.weight), HALF["bf16"])
    for name, lin, inp, dout in ((down, l2, H, dY), (up, l1, X, dGU)):
        if name in ("int8", "e4m3"):
            _product_close(lin.weight.grad, dout.T, _kept(inp, name), HALF["bf16"])
        else:
            assert torch.isfinite(lin.weight.grad).all() and lin.weight.grad.any()
    # the activation between them
    Gq, Uq = _kept(GU[:, :f], act), _kept(GU[:, f:], act)
    dg, du = orc.gated_bwd(dH, Gq, Uq)
    s = 1 / (1 + np.exp(-Gq))
    inner = (np.abs(Gq) + 8) * 2.0 ** -22
    assert np.all(np.abs(dGU[:, :f] - dg) <= 2.0 ** -8 * 1.01 * np.abs(dg) + inner * np.abs(dH * Uq) * s * (1 + np.abs(Gq) * (1 - s)) + 1e-38)
    assert np.all(np.abs(dGU[:, f:] - du) <= (2.0 ** -8 * 1.01 + inner) * np.abs(du) + 1e-38)
    # x: through the layer and around it
    into = dGU @ _f64(l1.weight)
    total = into + dO
    assert np.all(np.abs(flat(x.grad) - total) <= 2.0 ** -8 * 1.01 * (np.abs(into) + np.abs(total)) + (2 * f + 8) * U * (np.abs(dGU) @ np.abs(_f64(l1.weight))) + 1e-12)


def test_slices_that_are_not_aligned(mods):
    """Shifted labels and gradients that arrive as slices of a longer vector, against copies of them."""
    torch, ag = mods
    torch.manual_seed(5)
    x = torch.randn(2, 77, 72, device="cuda", dtype=torch.bfloat16)
    w0 = torch.randn(301, 72, device="cuda", dtype=torch.bfloat16)
    ids, g = torch.randint(0, 301, (155,), device="cuda"), torch.randn(155, device="cuda")
    assert ids[1:].data_ptr() % 16 and g[1:].data_ptr() % 16
    got = []
    for labels, weight in ((ids[1:], g[1:]), (ids[1:].clone(), g[1:].clone())):
        a, w = x.detach().requires_grad_(), w0.detach().requires_grad_()
        first = torch.zeros(1, device="cuda", requires_grad=True)
        loss = ag.LinearCrossEntropyFunction.apply(a, w, labels.reshape(2, 77))
        (torch.cat([first, loss.reshape(-1)]) * torch.cat([g[:1], weight])).sum().backward()   # its gradient starts at the second element
        got.append((loss.detach(), a.grad, w.grad))
    for a, b in zip(*got):
        assert torch.equal(a, b)
    flat = torch.randn(9 * 144 + 3, device="cuda")
    h = [ag.CompressedSwiGLUFunction.apply(f.reshape(9, 144), "int8") for f in (flat[3:], flat[3:].clone())]
    assert torch.equal(*h)


def test_second_derivatives_are_refused(mods):
    torch, ag = mods
    x = torch.randn(8, 64, device="cuda", requires_grad=True)
    w = torch.randn(32, 64, device="cuda", requires_grad=True)
    t = torch.zeros(8, dtype=torch.int64, device="cuda")
    for y in (ag.CompressedLinearFunction.apply(x, w, None, 0, 0, "int8"), ag.CompressedSwiGLUFunction.apply(x, "e4m3"),
              ag.LinearCrossEntropyFunction.apply(x, w, t)):
        (dx,) = torch.autograd.grad((y * y).sum(), x, create_graph=True)
        with pytest.raises(RuntimeError):
            dx.sum().backward()


def test_two_streams_at_once(mods):
    """Calls that share nothing on two streams, against the same calls one after the other."""
    torch, ag = mods
    torch.manual_seed(4)
    x = [torch.randn(300, 144, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    w = torch.randn(700, 144, device="cuda", dtype=torch.bfloat16) * 0.1
    t = torch.randint(0, 700, (300,), device="cuda")

    def step(a):
        a, b = a.detach().requires_grad_(), w.detach().requires_grad_()
        loss = ag.LinearCrossEntropyFunction.apply(a, b, t)
        h = ag.CompressedSwiGLUFunction.apply(a, "int8")
        torch.autograd.backward([loss.sum(), h.float().sum()])
        return loss.detach(), h.detach(), a.grad, b.grad

    want = [step(a) for a in x]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        got = [None, None]
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[k] = step(x[k])
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            for p, q in zip(a, b):
                assert torch.equal(p, q)
