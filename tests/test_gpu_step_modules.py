"""The modules of a training step's attention, table and clipping: against their formulas, and all of them together."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ag():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_01255_amd import autograd
    return autograd


def _plain_attention(x, heads, kv, causal, documents, prefix=None, window=0, cap=0.0, slopes=None, scale=None):
    """float32 by torch's own operators; documents: (first, end)."""
    import torch
    n, width = x.shape
    d = width // (heads + 2 * kv)
    q, k, v = (t.reshape(n, -1, d).transpose(0, 1) for t in x.split((heads * d, kv * d, kv * d), 1))
    k, v = k.repeat_interleave(heads // kv, 0), v.repeat_interleave(heads // kv, 0)
    z = (q @ k.transpose(1, 2).contiguous()) * (scale or 1 / math.sqrt(d))
    if cap:
        z = cap * torch.tanh(z / cap)
    i = torch.arange(n, device=x.device)
    if slopes is not None:
        z = z - slopes.view(-1, 1, 1) * (i[:, None] - i).abs()
    seen = torch.zeros(n, n, dtype=torch.bool, device=x.device)
    for e, (a, b) in enumerate(documents):
        inside = (i >= a) & (i < b)
        m = inside[:, None] & inside
        if causal:
            near = i[:, None] >= i
            if window:
                near &= i[:, None] - i < window
            if prefix is not None:
                near |= i < a + int(prefix[e])
            m &= near
        seen |= m
    p = torch.softmax(z.masked_fill(~seen, -1e30), 2) * seen
    return (p @ v).transpose(0, 1).reshape(n, heads * d)


@pytest.mark.parametrize("kw", [dict(heads=4, kv_heads=2), dict(heads=3, causal=False, slopes=True), dict(heads=4, kv_heads=1, cap=10.0, window=20),
                                dict(heads=2, scale=0.2, slopes=[0.5, 0.01])], ids=str)
@pytest.mark.parametrize("form", ["sequences", "documents", "rows apart"])
def test_attention_module(ag, kw, form):
    import torch
    att = ag.DocumentAttention(**kw, device="cuda")
    width = (att.heads + 2 * att.kv_heads) * 32
    torch.manual_seed(1)
    x = torch.randn(2, 60, width, device="cuda")
    if form == "rows apart":
        x = torch.randn(2, 60, width + 32, device="cuda")[..., :width]
    x.requires_grad_(True)
    starts = torch.tensor([0, 10, 10, 95], dtype=torch.int32, device="cuda") if form == "documents" else None
    documents = [(0, 10), (10, 10), (10, 95)] if form == "documents" else [(0, 60), (60, 120)]
    y = att(x, starts)
    g = torch.randn_like(y)
    dx, = torch.autograd.grad(y, x, g)
    x2 = x.detach().reshape(120, width).clone().requires_grad_(True)
    want = _plain_attention(x2, att.heads, att.kv_heads, att.causal, documents, window=att.window, cap=att.cap, slopes=att.slopes, scale=att.scale)
    dwant, = torch.autograd.grad(want, x2, g.reshape(120, -1))
    # both in float: some 2^-24 sqrt(terms) of the largest magnitudes, a hundred roundings of them
    assert float((y.reshape(120, -1) - want).abs().max()) < 100 * 2.0 ** -24 * float(want.abs().max()) * 4
    assert float((dx.reshape(120, width) - dwant).abs().max()) < 100 * 2.0 ** -24 * float(dwant.abs().max()) * 4


def test_attention_prefix_and_edges(ag):
    import torch
    att = ag.DocumentAttention(2, 1)
    x = torch.randn(3, 20, 4 * 16, device="cuda").requires_grad_(True)
    prefix = torch.tensor([5, 0, 100], device="cuda")
    y = att(x, prefix=prefix)
    want = _plain_attention(x.detach().reshape(60, 64), 2, 1, True, [(0, 20), (20, 40), (40, 60)], prefix=[5, 0, 20])
    assert float((y.reshape(60, 32) - want).abs().max()) < 400 * 2.0 ** -24 * float(want.abs().max())
    for bad in (dict(prefix=prefix[:2]), dict(starts=torch.tensor([0], device="cuda")), dict(starts=torch.tensor([0, 60])), dict(starts=torch.tensor([0.0, 1.0], device="cuda"))):
        with pytest.raises(ValueError):
            att(x, **bad)
    empty = att(torch.empty(0, 20, 64, device="cuda", requires_grad=True))
    assert empty.shape == (0, 20, 32)
    empty.sum().backward()
    one = att.to(torch.bfloat16)(torch.randn(1, 64, device="cuda", dtype=torch.bfloat16))   # one row attends to itself
    assert one.shape == (1, 32)
    with pytest.raises(RuntimeError):   # no second derivatives
        g, = torch.autograd.grad(y.sum(), x, create_graph=True)
        g.sum().backward()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_embedding_module(ag, dtype):
    import torch
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    table = ag.Embedding(50, 24, scale=3.0, device="cuda", dtype=dt)
    ids = torch.tensor([[3, 49, -1], [3, 0, 3]], device="cuda", dtype=torch.int32)
    y = table(ids)
    assert torch.equal(y, torch.where((ids >= 0).unsqueeze(2), table.weight.detach().float()[ids.clamp_min(0).long()] * 3.0, 0.0).to(dt))
    g = torch.randn(2, 3, 48, device="cuda").to(dt)[..., :24]   # rows apart
    y.backward(g)
    want = torch.zeros(50, 24, device="cuda", dtype=torch.float64)
    want.index_add_(0, ids[ids >= 0].long(), g[ids >= 0].double() * 3.0)
    step = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -22
    assert bool(((table.weight.grad.double() - want).abs() <= step * want.abs() + 2.0 ** -21 * float(g.abs().max()) * 9).all())
    table.weight.grad = None
    table(torch.empty(0, 4, dtype=torch.int64, device="cuda")).sum().backward()
    assert not table.weight.grad.any()
    with torch.no_grad():
        assert table(ids).requires_grad is False


def test_clipping(ag):
    import torch
    torch.manual_seed(0)
    ps = [torch.nn.Parameter(torch.randn(s, device="cuda")) for s in ((30, 40), (7,), (16, 16))]
    for p in ps:
        p.grad = torch.randn_like(p)
    ps[2].grad = torch.randn(16, 16, device="cuda").t()       # not contiguous
    ps.append(torch.nn.Parameter(torch.ones(5, device="cuda")))   # no gradient
    start = [p.grad.clone() for p in ps[:3]]
    want = math.sqrt(sum(float(g.double().square().sum()) for g in start))
    norm = ag.clip_grad_norm_(ps + ps[:1], 2.0)               # (the same parameter twice counts once)
    assert abs(float(norm) - want) <= 2.0 ** -23 * want
    for p, g in zip(ps, start):
        assert torch.allclose(p.grad, g * (2.0 / (want + 1e-6)), rtol=2.0 ** -21, atol=0.0)
    assert not ps[2].grad.is_contiguous()
    before = [p.grad.clone() for p in ps[:3]]
    assert float(ag.clip_grad_norm_(ps, 100.0)) < 2.001       # nothing to clip
    assert all(torch.equal(p.grad, g) for p, g in zip(ps, before))


def test_clipping_factored_gradients(ag):
    """The norm is that of the gradient the factors stand for, the optimizer's step that of the clipped one."""
    import torch
    torch.manual_seed(0)
    lin = ag.CompressedLinear(64, 128, rank=16, bias=False, device="cuda", factored_grad=True)
    lin(torch.randn(256, 64, device="cuda").bfloat16()).square().sum().backward()
    left, gr = (t.clone() for t in lin.grad_factors)
    dense = gr.double() @ left.double().t()
    other = torch.nn.Parameter(torch.zeros(10, device="cuda"))
    other.grad = torch.full((10,), 2.0, device="cuda")
    want = math.sqrt(float(dense.square().sum()) + 40.0)
    norm = ag.clip_grad_norm_([other], 0.5, modules=[lin, lin])
    assert abs(float(norm) - want) <= 1e-5 * want             # sums of 256 float products over 16 x 16 places
    by = (0.5 / (torch.tensor(want, dtype=torch.float64) + 1e-6)).float()
    assert torch.equal(lin.grad_factors[0], left)
    assert bool(((lin.grad_factors[1].double() - gr.double() * float(by)).abs() <= (2.0 ** -8 + 1e-5) * (gr.double() * float(by)).abs()).all())
    ag.LowRankAdamW([lin], lr=1e-3).step()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_decoder_step_of_all_of_them(ag, dtype):
    """Table, projections, attention, gated activation, the tied vocabulary's loss, clipping and both optimizers: one step's gradients
    against torch's own operators in float64 on the same weights (compressors that keep the input whole)."""
    import torch
    torch.manual_seed(0)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    v, d, heads, kv, f = 211, 64, 4, 2, 96
    ids = torch.randint(0, v, (2, 48), device="cuda")
    ids[1, 40:] = -1                                           # padding
    targets = torch.cat((ids[:, 1:], torch.full((2, 1), -1, device="cuda")), 1)
    table = ag.Embedding(v, d, scale=8.0, device="cuda", dtype=dt)
    qkv = ag.CompressedLinear(d, (heads + 2 * kv) * 16, bias=False, compressor="int8", device="cuda", dtype=dt)
    att = ag.DocumentAttention(heads, kv, cap=20.0, slopes=True, device="cuda")
    out = ag.CompressedLinear(heads * 16, d, bias=False, compressor="int8", device="cuda", dtype=dt)
    up = ag.CompressedLinear(d, 2 * f, bias=False, compressor="int8", device="cuda", dtype=dt)
    act = ag.CompressedSwiGLU("int8")
    down = ag.CompressedLinear(f, d, bias=False, compressor="int8", device="cuda", dtype=dt)
    head = ag.LinearCrossEntropy(d, v, device="cuda", dtype=dt)
    head.weight = table.weight                                 # tied
    weights = {"table": table.weight, "qkv": qkv.weight, "out": out.weight, "up": up.weight, "down": down.weight}
    with torch.no_grad():
        for w in weights.values():
            w.copy_(torch.randn_like(w, dtype=torch.float32) * 0.1)

    def loss_of():
        x = table(ids)
        x = x + out(att(qkv(x)))
        x = x + down(act(up(x)))
        return head(x, targets)

    loss = loss_of()
    loss.backward()
    plain = {k: w.detach().double().requires_grad_(True) for k, w in weights.items()}
    x = torch.where((ids >= 0).unsqueeze(2), plain["table"][ids.clamp_min(0)] * 8.0, 0.0)
    a = _plain_attention((x @ plain["qkv"].t()).reshape(96, -1), heads, kv, True, [(0, 48), (48, 96)], cap=20.0, slopes=att.slopes.double())
    x = x + a.reshape(2, 48, -1) @ plain["out"].t()
    gate, upper = (x @ plain["up"].t()).chunk(2, 2)
    x = x + (torch.nn.functional.silu(gate) * upper) @ plain["down"].t()
    logits = x @ plain["table"].t()
    want = torch.nn.functional.cross_entropy(logits[targets >= 0], targets[targets >= 0])
    want.backward()
    # bfloat16: some ten roundings of 2^-8 on the way of every value, float: the checkpoints' 0.4 % in the weights' gradients
    assert abs(float(loss) - float(want)) < (0.02 if dtype == "bf16" else 1e-5) * float(want)
    for name, w in weights.items():
        rel = float((w.grad.double() - plain[name].grad).norm() / plain[name].grad.norm())
        assert rel < (0.08 if dtype == "bf16" else 0.02), (name, rel)

    opt = torch.optim.AdamW(weights.values(), lr=1e-2)
    before = float(loss)
    norm = ag.clip_grad_norm_(weights.values(), 1.0)
    assert math.isfinite(float(norm))
    opt.step()
    opt.zero_grad()
    again = loss_of()
    assert math.isfinite(float(again)) and float(again) != before


def test_a_captured_step(ag):
    """Table, attention and clipping in one graph, replayed on other inputs beside the program's own passes over the same weights."""
    import torch
    table = ag.Embedding(60, 4 * 32, device="cuda")
    attend = ag.DocumentAttention(2, 1, cap=15.0, slopes=True, device="cuda")
    ids, starts = torch.randint(0, 60, (130,), device="cuda"), torch.tensor([0, 50, 130], device="cuda")
    g = torch.randn(130, 64, device="cuda").to(torch.bfloat16)

    def step():
        table.weight.grad = None
        y = attend(table(ids), starts)
        table.weight.grad, = torch.autograd.grad(y, table.weight, g)
        norm = ag.clip_grad_norm_(table.parameters(), 0.25)
        return y.detach(), table.weight.grad, norm

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(4):
        ids.copy_(torch.randint(-1, 60, (130,), device="cuda"))
        starts.copy_(torch.tensor([k, 40 + 20 * k, 130 - k], device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k
