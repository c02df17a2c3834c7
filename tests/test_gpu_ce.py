"""The vocabulary's cross entropy on the GPU against its formulas in 64 bits.

Tolerances, worst cases with u = 2^-24: a logit is off by at most e_z = (d + 8) u sum |x| |w| (a float sum of d terms in any order); a
sum of exponentials that is formed in pieces of a few hundred terms and those added by (v / 64 + 64) u of itself, its logarithm by as
much, and by 4 u of its own size; exp's argument, rounded to u of itself, moves it by |z| u.  So lse is off by
e_l = max e_z + (v / 64 + 64) u + 8 u (1 + |lse|), a loss by e_l + e_z of its target, dz by |p g| (e_z + e_l + 16 u (1 + |z - lse|)), and
where it is an operand in bfloat16 by 2^-8 of itself.  dX and dW: the error of dz times the other operand, (terms + 8) u sum of
magnitudes, and their own rounding of 2^-8 (bfloat16) or u."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from oracle import train_oracle as orc

U = 2.0 ** -24


@pytest.fixture(scope="module")
def acc():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_01255_amd import binding
    return binding


class Case:
    def __init__(self, acc, n, d, v, dtype, dw=None, piece=0, ignored=0.0, pad=0, add=False, seed=0, scale=1.0):
        import torch
        self.acc, self.n, self.d, self.v, self.add = acc, n, d, v, add
        self.b16 = dtype == "bf16"
        self.tdt = torch.bfloat16 if self.b16 else torch.float32
        self.dwt = torch.bfloat16 if (dw or dtype) == "bf16" else torch.float32
        g = torch.Generator(device="cuda").manual_seed(seed + n + d + v)
        rnd = lambda r, c, s: (torch.randn(r, c, generator=g, device="cuda") * s).to(self.tdt)  # noqa: E731

        def rows(r, s):
            t = torch.full((r, d + pad), float("nan"), dtype=self.tdt, device="cuda")
            t[:, :d] = rnd(r, d, s)
            return t

        self.X, self.W = rows(n, 1.0), rows(v, scale * 1.5 / d ** 0.5)
        t = torch.randint(0, v, (n,), generator=g, device="cuda")
        self.targets = torch.where(torch.rand(n, generator=g, device="cuda") < ignored, -100, t)
        self.dloss = torch.randn(n, generator=g, device="cuda") / n
        self.before = (torch.randn(v, d, generator=g, device="cuda") * 1e-3).to(self.dwt)
        self.pad = pad
        code = lambda t: acc.ACC_BF16 if t == torch.bfloat16 else acc.ACC_F32  # noqa: E731
        self.desc = acc.make_ce_desc(n, d, v, ldx=d + pad, ldw=d + pad, piece=piece, io_dtype=code(self.tdt), dw_dtype=code(self.dwt),
                                     flags=acc.ACC_FLAG_DW_ACCUMULATE if add else 0)

    def forward(self):
        import torch
        loss, stats = torch.full((self.n,), 7.0, device="cuda"), torch.full((2, self.n), 7.0, device="cuda")
        ws = torch.full((self.acc.acc_linear_ce_workspace_bytes(self.desc, False) + 256,), 0xFF, dtype=torch.uint8, device="cuda")
        self.acc.acc_linear_ce_fwd(self.desc, self.X, self.W, self.targets, loss, stats, ws, ws_bytes=ws.numel() - 256)
        assert bool((ws[-256:] == 0xFF).all())
        return loss, stats

    def backward(self, stats, dx=True, dw=True):
        import torch
        dX = torch.full((self.n, self.d + self.pad), 7.0, dtype=self.tdt, device="cuda") if dx else None
        dW = (self.before.clone() if self.add else torch.full((self.v, self.d), 7.0, dtype=self.dwt, device="cuda")) if dw else None
        ws = torch.full((self.acc.acc_linear_ce_workspace_bytes(self.desc, True) + 256,), 0xFF, dtype=torch.uint8, device="cuda")   # NaN bits
        self.acc.acc_linear_ce_bwd(self.desc, self.X, self.W, self.targets, stats, self.dloss, dX, dW, ws, ws_bytes=ws.numel() - 256)
        assert bool((ws[-256:] == 0xFF).all())
        if dx and self.pad:
            assert bool((dX[:, self.d:] == 7.0).all())
        return dX[:, :self.d] if dx else None, dW

    def want(self):
        """Values in float64 and how far they may be off."""
        import torch
        keep = self.targets >= 0
        x = torch.where(keep.unsqueeze(1), self.X[:, :self.d].double(), 0.0)
        w = self.W[:, :self.d].double()
        rows = torch.arange(self.n, device="cuda")
        inside = keep & (self.targets < self.v)
        t = torch.where(inside, self.targets, 0)
        z, ez = x @ w.t(), (self.d + 8) * U * (x.abs() @ w.abs().t())
        lse = torch.logsumexp(z, 1)
        el = ez.amax(1) + (self.v / 64 + 64) * U + 8 * U * (1 + lse.abs())
        loss = torch.where(keep, lse - z[rows, t], 0.0)
        loss = torch.where(keep & ~inside, float("nan"), loss)
        eloss = el + ez[rows, t] + 2 * U * loss.abs().nan_to_num()
        g = torch.where(inside, self.dloss.double(), 0.0).unsqueeze(1)
        p = torch.exp(z - lse.unsqueeze(1))
        edz = (p * g).abs() * (ez + el.unsqueeze(1) + 16 * U * (1 + (z - lse.unsqueeze(1)).abs()))
        dz = p * g
        dz[rows, t] = torch.where(inside, torch.expm1(z[rows, t] - lse) * g[:, 0], dz[rows, t])
        if self.b16:
            edz = edz * (1 + 2.0 ** -8) + 2.0 ** -8 * dz.abs()
        half = lambda t: 2.0 ** -8 if t == torch.bfloat16 else U  # noqa: E731
        adz = dz.abs() + edz
        dx, dw = dz @ w, dz.t() @ x
        edx = edz @ w.abs() + (self.v + 8) * U * (adz @ w.abs())
        edw = edz.t() @ x.abs() + (self.n + 8) * U * (adz.t() @ x.abs())
        if self.add:
            dw = dw + self.before.double()
            edw = edw + U * (dw.abs() + self.before.double().abs())
        edx = edx + half(self.tdt) * (dx.abs() + edx)
        edw = edw + half(self.dwt) * (dw.abs() + edw)
        return dict(loss=(loss, eloss), lse=(torch.where(keep, lse, 0.0), el), dx=(dx, edx), dw=(dw, edw))

    def check(self):
        import torch
        print("ce", self.n, self.d, self.v, self.tdt, self.dwt, "piece", self.desc.piece, "add", self.add, flush=True)
        loss, stats = self.forward()
        dX, dW = self.backward(stats)
        torch.cuda.synchronize()
        want = self.want()
        for name, got in (("loss", loss), ("lse", stats[0]), ("dx", dX), ("dw", dW)):
            value, off = want[name]
            got = got.double()
            assert torch.equal(torch.isnan(got), torch.isnan(value)), name
            ratio = ((got - value).abs() / (off + 1e-37)).nan_to_num()
            assert float(ratio.max()) <= 1.0, (name, float(ratio.max()), int((ratio > 1).sum()))
        ignored = self.targets < 0
        assert bool((loss[ignored] == 0).all()) and bool((stats[:, ignored] == 0).all()) and bool((dX[ignored] == 0).all())
        return loss, stats, dX, dW


SHAPES = [
    dict(n=1, d=8, v=1), dict(n=1, d=64, v=5), dict(n=1, d=2048, v=3001), dict(n=2, d=72, v=257), dict(n=63, d=136, v=1000, pad=8),
    dict(n=65, d=264, v=2049, ignored=0.3, piece=256), dict(n=129, d=520, v=777, ignored=0.5, pad=24, add=True),
    dict(n=255, d=64, v=4099, piece=1024, add=True), dict(n=300, d=1032, v=1283, ignored=0.9),
    dict(n=515, d=520, v=10007, ignored=0.1, piece=2560), dict(n=1000, d=128, v=512, ignored=0.2),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(f"{k}{v}" for k, v in s.items()))
def test_losses_and_gradients(acc, shape, dtype):
    Case(acc, dtype=dtype, **shape).check()


@pytest.mark.parametrize("shape", [
    dict(n=3000, d=1024, v=20011, ignored=0.4), dict(n=2048, d=2048, v=16384, piece=4096), dict(n=4100, d=512, v=32000, ignored=0.96),
    dict(n=2049, d=1032, v=9001, pad=16, add=True, dw="f32")], ids=lambda s: "-".join(f"{k}{v}" for k, v in s.items()))
def test_large_bfloat16(acc, shape):
    Case(acc, dtype="bf16", **shape).check()


def test_losses_of_a_matrix_beyond_four_gib(acc):
    """More of W than one buffer resource reaches, with a ragged last K tile; targets at both ends.  By the terms above a logit is
    off by e_z, and a log-sum-exp by that and (2^21 / 64 + 64) u < 2^-8 / 2, and 8 u of its own size, under 2^-8 / 2 as well."""
    import torch
    n, d, v = 5, 1032, (1 << 21) - 3
    torch.manual_seed(9)
    x = (torch.randn(n, d, device="cuda") * 0.05).to(torch.bfloat16)
    w = torch.empty(v, d, device="cuda", dtype=torch.bfloat16).normal_()
    t = torch.tensor([0, v - 1, v // 2, -1, (1 << 20) + 77], device="cuda")
    desc = acc.make_ce_desc(n, d, v)
    loss, stats = torch.full((n,), 7.0, device="cuda"), torch.full((2, n), 7.0, device="cuda")
    ws = torch.empty(acc.acc_linear_ce_workspace_bytes(desc, False), dtype=torch.uint8, device="cuda")
    acc.acc_linear_ce_fwd(desc, x, w, t, loss, stats, ws)
    torch.cuda.synchronize()
    x64, z, off = x.double(), [], 0.0
    for v0 in range(0, v, 1 << 18):
        part = w[v0:v0 + (1 << 18)].double().t().contiguous()
        z.append(x64 @ part)
        off = max(off, float((x64.abs() @ part.abs()).max()))
    z = torch.cat(z, 1)
    bound = 2 * (d + 8) * U * off + 2.0 ** -8
    keep = t >= 0
    lse = torch.where(keep, torch.logsumexp(z, 1), 0.0)
    zt = torch.where(keep, z.gather(1, t.clamp(min=0)[:, None])[:, 0], 0.0)
    assert float((stats[0].double() - lse).abs().max()) <= bound
    assert float((stats[1].double() - zt).abs().max()) <= bound
    assert float((loss.double() - (lse - zt)).abs().max()) <= bound and float(loss[3]) == 0.0


@pytest.mark.parametrize("rest", [100, 300])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_tokens_than_a_run(acc, dtype, rest):
    Case(acc, (1 << 18) + rest, 8, 77, dtype, dw="f32", ignored=0.3).check()


@pytest.mark.parametrize("dtype,dw", [("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("add", [False, True])
def test_gradient_of_the_other_type(acc, dtype, dw, add):
    Case(acc, 200, 136, 523, dtype, dw=dw, ignored=0.2, add=add).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_against_the_oracle(acc, dtype):
    import torch
    c = Case(acc, 70, 72, 301, dtype, ignored=0.3)
    want = c.want()
    f64 = lambda t: t.double().cpu().numpy()  # noqa: E731
    x, w, t = f64(c.X), f64(c.W), c.targets.cpu().numpy()
    loss, lse = orc.linear_ce(x, w, t)
    dx, dw = orc.linear_ce_bwd(x, w, t, f64(c.dloss))
    for name, value in (("loss", loss), ("dx", dx), ("dw", dw)):
        np.testing.assert_allclose(f64(want[name][0]), value, rtol=1e-10, atol=1e-14)
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_without_a_loss_are_read_into_nothing(acc, dtype):
    import torch
    c = Case(acc, 333, 136, 700, dtype, ignored=0.4)
    clean = c.check()
    ignored = c.targets < 0
    c.X[ignored, 0] = float("nan")
    c.X[ignored, 1] = float("inf")
    c.dloss[ignored] = float("nan")
    again = c.forward()
    grads = c.backward(again[1])
    for a, b in zip(clean, (*again, *grads)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("add", [False, True])
def test_nothing_but_rows_without_a_loss(acc, dtype, add):
    import torch
    c = Case(acc, 70, 64, 300, dtype, ignored=1.0, add=add)
    c.X[:] = float("nan")
    loss, stats = c.forward()
    dX, dW = c.backward(stats)
    assert not loss.any() and not stats.any() and not dX.any()
    assert torch.equal(dW, c.before) if add else not dW.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_targets_beyond_the_vocabulary(acc, dtype):
    import torch
    c = Case(acc, 90, 72, 130, dtype, ignored=0.2, piece=256)
    c.targets[5], c.targets[40], c.targets[77] = 130, 1 << 40, -(1 << 40)
    loss, _, dX, _ = c.check()
    assert torch.isnan(loss[[5, 40]]).all() and loss[77] == 0 and not dX[[5, 40, 77]].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_logits(acc, dtype):
    """Logits of several hundreds: losses stay finite, and a token that is certain has no gradient left."""
    import torch
    c = Case(acc, 64, 64, 400, dtype, scale=100.0)
    z = c.X.double() @ c.W.double().t()
    c.targets[:32] = z[:32].argmax(1)
    assert float(z.abs().max()) > 300
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_is_not_finite_stays_in_its_row(acc, dtype):
    import torch
    c = Case(acc, 40, 64, 300, dtype)
    c.X[7, 3] = float("nan")
    c.X[9] = 0
    loss, stats = c.forward()
    assert torch.isnan(loss[7]) and torch.isnan(stats[0, 7]) and int(torch.isnan(loss).sum()) == 1
    assert abs(float(loss[9]) - np.log(300)) < 1e-4
    c.W[11, 2] = float("inf")
    loss, _ = c.forward()
    z = (c.X.float() @ c.W.float().t())
    ref = torch.logsumexp(z, 1) - z.gather(1, c.targets.unsqueeze(1))[:, 0]
    assert torch.equal(torch.isfinite(loss), torch.isfinite(ref))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_gradient_at_a_time_and_again_gives_the_same_bits(acc, dtype):
    import torch
    c = Case(acc, 700, 264, 3000, dtype, ignored=0.3, piece=1024)
    loss, stats = c.forward()
    both = c.backward(stats)
    loss2, stats2 = c.forward()
    assert torch.equal(loss, loss2) and torch.equal(stats, stats2)
    assert torch.equal(both[0], c.backward(stats, dw=False)[0]) and torch.equal(both[1], c.backward(stats, dx=False)[1])


def test_gradient_against_differences(acc):
    """Float32: the loss moves along a direction as the gradients say."""
    import torch
    c = Case(acc, 33, 64, 150, "f32", ignored=0.2)
    _, stats = c.forward()
    dX, dW = (t.double() for t in c.backward(stats))
    vx, vw = torch.randn_like(c.X), torch.randn_like(c.W) * 0.1
    x0, w0, h = c.X.clone(), c.W.clone(), 2.0 ** -7

    def at(s):
        c.X, c.W = x0 + s * h * vx, w0 + s * h * vw
        return float((c.forward()[0].double() * c.dloss.double()).sum())

    slope = (at(1) - at(-1)) / (2 * h)
    want = float((dX * vx).sum() + (dW * vw).sum())
    # float32 losses of about 5, weighted by 1 / n: 33 * 5 * 2^-21 / 33 over the step of 2^-6; the third derivative times h^2 / 6
    at2 = (at(2) - at(-2)) / (4 * h)
    assert abs(slope - want) <= abs(at2 - slope) + 5 * 2.0 ** -21 / h


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_and_replayed(acc, dtype):
    """Targets change between replays, so the number of tokens with a loss does."""
    import torch
    c = Case(acc, 300, 136, 1001, dtype, piece=512)
    d = c.desc
    bufs = [dict(loss=torch.empty(c.n, device="cuda"), stats=torch.empty(2, c.n, device="cuda"), dX=torch.empty_like(c.X), dW=torch.empty_like(c.W),
                 ws=torch.empty(acc.acc_linear_ce_workspace_bytes(d, True), dtype=torch.uint8, device="cuda")) for _ in range(2)]

    def step(b):
        acc.acc_linear_ce_fwd(d, c.X, c.W, c.targets, b["loss"], b["stats"], b["ws"])
        acc.acc_linear_ce_bwd(d, c.X, c.W, c.targets, b["stats"], c.dloss, b["dX"], b["dW"], b["ws"])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(bufs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(bufs[0])
    for r, share in enumerate((0.0, 0.5, 1.0, 0.1)):
        c.X.copy_(torch.randn_like(c.X))
        t = torch.randint(0, c.v, (c.n,), device="cuda")
        c.targets.copy_(torch.where(torch.rand(c.n, device="cuda") < share, -1, t))
        graph.replay()
        step(bufs[1])
        torch.cuda.synchronize()
        for k in ("loss", "stats", "dX", "dW"):
            assert torch.equal(bufs[0][k], bufs[1][k]), (r, k)
