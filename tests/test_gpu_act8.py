"""8-bit activation checkpoints on the GPU: bytes and scales bit for bit, what reads them against the oracle in 64 bits.

Tolerances.  Half a step of bfloat16 is 2^-8 of the value (finfo.eps / 2), of float32 2^-24.  A float32 sum of k terms is off by
at most k 2^-24 sum |terms| whatever its order.  sigmoid in float32: exp's argument is rounded to 2^-24 of itself, so exp and
sigmoid are off by (|g| + 8) 2^-23 of themselves at most, the few other operations included."""
import ctypes

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

import gpu_util as gu
from oracle import train_oracle as orc

FORMATS = ["e4m3", "int8"]


@pytest.fixture(scope="module")
def acc():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_01255_amd import binding
    return binding


def _types(acc, dtype, fmt):
    import torch
    return (acc.ACC_BF16, torch.bfloat16) if dtype == "bf16" else (acc.ACC_F32, torch.float32), acc.ACC_ACT8_E4M3 if fmt == "e4m3" else acc.ACC_ACT8_INT8


def _hard_values(rng, n, c):
    """Normal data with channels of every magnitude, zeros, infinities, NaN and the ends of the range in it."""
    x = rng.normal(0, 1, (n, c)) * 2.0 ** rng.integers(-130, 120, (1, c))
    kinds = rng.integers(0, 12, (n, c))
    x = np.where(kinds == 0, 0.0, x)
    x = np.where(kinds == 1, -0.0, x)
    odd = rng.random((n, c)) < 0.01
    x = np.where(odd, rng.choice([np.inf, -np.inf, np.nan, 3.38e38, -3.4e38, 1e-40], (n, c)), x)
    x[:, 0] = 0.0
    if c > 8:
        x[:, 8] = np.nan
    return x.astype(np.float32)


def _guarded(torch, shape, dtype, value):
    """A view with 64 elements of `value` before and after it."""
    n = int(np.prod(shape))
    buf = torch.full((n + 128,), value, dtype=dtype, device="cuda")
    return buf, buf[64:64 + n].view(shape)


def _guards_hold(buf, value):
    return bool((buf[:64] == value).all()) and bool((buf[-64:] == value).all())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,c,ld", [(1, 8, 8), (31, 120, 120), (32, 128, 128), (33, 136, 272), (77, 520, 520), (300, 1032, 1040), (64, 256, 256)])
def test_pack_and_unpack_are_exact(acc, n, c, ld, dtype, fmt):
    import torch
    print(f"pack {n} {c} {ld} {dtype} {fmt}", flush=True)
    (code, tdt), f = _types(acc, dtype, fmt)
    x = torch.full((n, ld), float("nan"), dtype=tdt, device="cuda")
    x[:, :c] = torch.from_numpy(_hard_values(np.random.default_rng(n * c), n, c)).to(tdt).cuda()
    desc = acc.make_act8_desc(n, c, ldx=ld, io_dtype=code, format=f)
    blocks = -(-n // 32)
    qb, q = _guarded(torch, (n, c), torch.uint8, 0xA5)
    eb, e = _guarded(torch, (blocks, c), torch.uint8, 0xA5)
    acc.acc_act8_pack(desc, x, q, e)
    back = torch.full((n, ld), 7.0, dtype=tdt, device="cuda")
    acc.acc_act8_unpack(desc, q, e, back)
    torch.cuda.synchronize()
    want_q, want_e = orc.act8_pack(x[:, :c].cpu().double().numpy(), fmt)
    np.testing.assert_array_equal(e.cpu().numpy(), want_e)
    np.testing.assert_array_equal(q.cpu().numpy(), want_q)
    assert _guards_hold(qb, 0xA5) and _guards_hold(eb, 0xA5)
    np.testing.assert_array_equal(back[:, :c].cpu().double().numpy(), orc.act8_unpack(want_q, want_e, fmt))
    assert bool((back[:, c:] == 7.0).all())


@pytest.mark.parametrize("fmt", FORMATS)
def test_every_bfloat16_value_and_every_code(acc, fmt):
    import torch
    (code, tdt), f = _types(acc, "bf16", fmt)
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = bits.reshape(-1, 256).cuda()               # 256 x 256: a block's rows are 32 values 512 apart in the order of the bits
    desc = acc.make_act8_desc(256, 256, format=f)
    q, e = acc.alloc_act8(desc)
    acc.acc_act8_pack(desc, x, q, e)
    want_q, want_e = orc.act8_pack(x.cpu().double().numpy(), fmt)
    np.testing.assert_array_equal(e.cpu().numpy(), want_e)
    np.testing.assert_array_equal(q.cpu().numpy(), want_q)
    # every code under every scale a checkpoint holds
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8).repeat(32, 1).cuda()
    for first in (27, 100, 127, 248 - 32):
        scales = (first + torch.arange(256, dtype=torch.int32) % 32).to(torch.uint8).reshape(1, 256).cuda()
        out = torch.empty(32, 256, device="cuda")
        one = acc.make_act8_desc(32, 256, io_dtype=acc.ACC_F32, format=f)
        acc.acc_act8_unpack(one, codes, scales, out)
        np.testing.assert_array_equal(out.cpu().double().numpy(), orc.act8_unpack(codes.cpu().numpy(), scales.cpu().numpy(), fmt).astype(np.float32))


@pytest.mark.parametrize("fmt", FORMATS)
def test_rounding_of_ties(acc, fmt):
    """Blocks whose largest element is the format's limit, so that e = 0, filled with the middles between neighbouring values."""
    import torch
    v = np.unique(orc.VALUES[fmt][np.isfinite(orc.VALUES[fmt])])
    mids = (v[1:] + v[:-1]) / 2
    mids = np.concatenate([mids, np.nextafter(mids.astype(np.float32), np.float32(1e9)), np.nextafter(mids.astype(np.float32), np.float32(-1e9))])
    c = -(-len(mids) // 31 // 8) * 8 + 8
    x = np.full((32, c), orc.LIMIT[fmt], dtype=np.float32)
    x[1:].reshape(-1)[:len(mids)] = mids
    f = _types(acc, "f32", fmt)[1]
    desc = acc.make_act8_desc(32, c, io_dtype=acc.ACC_F32, format=f)
    q, e = acc.alloc_act8(desc)
    acc.acc_act8_pack(desc, torch.from_numpy(x).cuda(), q, e)
    want_q, want_e = orc.act8_pack(x, fmt)
    assert (want_e == 127).all()
    np.testing.assert_array_equal(e.cpu().numpy(), want_e)
    np.testing.assert_array_equal(q.cpu().numpy(), want_q)


def _gated_inputs(acc, n, f, dtype, stacked, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    both = (torch.randn(n, 2 * f, generator=g, device="cuda") * 3).to(tdt)
    both[:, 0] = -80.0          # far out on either side: sigmoid underflows towards 0 and reaches 1
    both[:, 1] = 80.0
    dh = torch.randn(n, f, generator=g, device="cuda").to(tdt)
    if stacked:
        return both[:, :f], both[:, f:], dh, 2 * f
    return both[:, :f].contiguous(), both[:, f:].contiguous(), dh, f


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,f,stacked", [(1, 8, False), (1, 264, True), (33, 136, False), (70, 520, True), (257, 128, True)])
def test_gated_activation(acc, n, f, stacked, dtype, fmt):
    import torch
    print(f"gated {n} {f} {stacked} {dtype} {fmt}", flush=True)
    (code, tdt), af = _types(acc, dtype, fmt)
    G, U, dH, ldg = _gated_inputs(acc, n, f, dtype, stacked, n + f)
    ldh = f + 8
    wide = torch.zeros(n, ldh, dtype=tdt, device="cuda")
    wide[:, :f] = dH
    desc = acc.make_gated_desc(n, f, ldg=ldg, ldh=ldh, io_dtype=code, format=af)
    kept = acc.alloc_gated_act8(desc)
    H = torch.full((n, ldh), 7.0, dtype=tdt, device="cuda")
    acc.acc_gated_fwd_act8(desc, G, U, H, *kept)
    f64 = lambda t: t.cpu().double().numpy()  # noqa: E731
    g, u, dh = f64(G), f64(U), f64(dH)
    for t, q, e in ((g, *kept[:2]), (u, *kept[2:])):
        want_q, want_e = orc.act8_pack(t, fmt)
        np.testing.assert_array_equal(q.cpu().numpy(), want_q)
        np.testing.assert_array_equal(e.cpu().numpy(), want_e)
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    inner = lambda x: (np.abs(x) + 8) * 2.0 ** -23  # noqa: E731

    def close(got, want, parts, x):
        assert np.all(np.abs(f64(got) - want) <= half * np.abs(want) * 1.01 + 2 * inner(x) * parts + 1e-45), float(np.max(np.abs(f64(got) - want)))

    close(H[:, :f], orc.gated(g, u), np.abs(orc.gated(g, u)), g)
    assert bool((H[:, f:] == 7.0).all())
    gq, uq = (orc.act8_unpack(kept[k].cpu().numpy(), kept[k + 1].cpu().numpy(), fmt) for k in (0, 2))
    dg_want, du_want = orc.gated_bwd(dh, gq, uq)
    s = 1 / (1 + np.exp(-gq))
    for again in (True, False):
        out = torch.full((n, 4 * f), 7.0, dtype=tdt, device="cuda")
        alone = torch.full((2, n, f), 7.0, dtype=tdt, device="cuda")
        dG, dU = (out[:, :f], out[:, f:2 * f]) if stacked else (alone[0], alone[1])
        desc_b = acc.make_gated_desc(n, f, ldg=4 * f if stacked else f, ldh=ldh, io_dtype=code, format=af)
        H2 = torch.full((n, ldh), 7.0, dtype=tdt, device="cuda")
        acc.acc_gated_bwd_act8(desc_b, wide, *kept, dG, dU, H2 if again else None)
        torch.cuda.synchronize()
        close(dG, dg_want, np.abs(dh * uq) * s * (1 + np.abs(gq) * (1 - s)), gq)
        close(dU, du_want, np.abs(du_want), gq)
        if again:
            close(H2[:, :f], orc.gated(gq, uq), np.abs(orc.gated(gq, uq)), gq)
            assert bool((H2[:, f:] == 7.0).all())
        else:
            assert bool((H2 == 7.0).all())
        if stacked:
            assert bool((out[:, 2 * f:] == 7.0).all())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("n,d_in,d_out,dtype,dw,w_out_in,pad,add", [
    (1, 8, 8, "bf16", "bf16", True, 0, False),
    (33, 72, 40, "bf16", "f32", False, 8, False),
    (300, 136, 264, "bf16", "bf16", True, 16, True),
    (777, 520, 264, "bf16", "f32", True, 0, True),
    (2049, 1032, 776, "bf16", "bf16", False, 8, False),
    (4100, 2048, 2048, "bf16", "bf16", True, 0, False),
    (5000, 4096, 4096, "bf16", "bf16", False, 0, False),
    (1, 8, 8, "f32", "f32", False, 0, False),
    (130, 72, 40, "f32", "f32", True, 8, True),
    (515, 264, 520, "f32", "bf16", True, 0, False),
])
def test_linear_layer(acc, n, d_in, d_out, dtype, dw, w_out_in, pad, add, fmt):
    import torch
    print(f"linear {n} {d_in} {d_out} {dtype} {dw} {w_out_in} {pad} {add} {fmt}", flush=True)
    (code, tdt), af = _types(acc, dtype, fmt)
    dcode, ddt = _types(acc, dw, fmt)[0]
    g = torch.Generator(device="cuda").manual_seed(n)

    def rows(r, c, scale):
        t = torch.full((r, c + pad), float("nan"), dtype=tdt, device="cuda")
        t[:, :c] = (torch.randn(r, c, generator=g, device="cuda") * scale).to(tdt)
        return t

    X, dY = rows(n, d_in, 1.0), rows(n, d_out, 0.1)
    W = rows(d_out, d_in, 0.1) if w_out_in else rows(d_in, d_out, 0.1)
    X[:, 3] *= 20
    flags = (acc.ACC_FLAG_W_OUT_IN if w_out_in else 0) | (acc.ACC_FLAG_DW_ACCUMULATE if add else 0)
    desc = acc.make_desc(n, d_in, d_out, 8, io_dtype=code, dw_dtype=dcode, ldx=d_in + pad, ldw=W.shape[1], ldy=d_out + pad, flags=flags)
    Y, dX = torch.full((n, d_out + pad), 7.0, dtype=tdt, device="cuda"), torch.full((n, d_in + pad), 7.0, dtype=tdt, device="cuda")
    q, e = acc.alloc_act8(acc.make_act8_desc(n, d_in, io_dtype=code, format=af))
    acc.acc_linear_fwd_act8(desc, af, X, W, Y, q, e)
    before = torch.randn(*((d_out, d_in) if w_out_in else (d_in, d_out)), generator=g, device="cuda").to(ddt)
    dW = before.clone()
    need = acc.acc_linear_act8_workspace_bytes(desc)
    wsb, ws = _guarded(torch, (need,), torch.uint8, 0xA5)
    acc.acc_linear_bwd_act8(desc, af, dY, W, q, e, dX, dW, ws)
    torch.cuda.synchronize()
    assert _guards_hold(wsb, 0xA5)
    if pad:
        assert bool((Y[:, d_out:] == 7.0).all()) and bool((dX[:, d_in:] == 7.0).all())
    f64 = lambda t, c: t[:, :c].double()  # noqa: E731  (products of float64 on the GPU: a library step)
    x, dy, w = f64(X, d_in), f64(dY, d_out), f64(W, W.shape[1] - pad)
    w = w.t() if w_out_in else w
    xq = torch.from_numpy(orc.act8_unpack(q.cpu().numpy(), e.cpu().numpy(), fmt)).cuda()
    half = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}

    def close(got, want, terms, k, t, extra=0.0):
        bound = half[t] * want.abs() * 1.01 + (k + 8) * 2.0 ** -24 * terms + extra
        assert bool(((got.double() - want).abs() <= bound).all()), float(((got.double() - want).abs() / bound).max())

    close(Y[:, :d_out], x @ w, x.abs() @ w.abs(), d_in, dtype)
    close(dX[:, :d_in], dy @ w.t(), dy.abs() @ w.abs().t(), d_out, dtype)
    want, terms = xq.t() @ dy, xq.abs().t() @ dy.abs()
    if w_out_in:
        want, terms = want.t(), terms.t()
    if add:
        want, terms = want + before.double(), terms + before.double().abs()
    close(dW, want, terms, n, dw)
    # one output at a time gives the same bits, and a linear that shares the input leaves the checkpoint alone
    dX2, dW2 = torch.full_like(dX, 7.0), before.clone()
    acc.acc_linear_bwd_act8(desc, af, dY, W, None, None, dX2, None, None)
    acc.acc_linear_bwd_act8(desc, af, dY, None, q, e, None, dW2, ws)
    assert torch.equal(dX, dX2) and torch.equal(dW, dW2)
    Y2 = torch.full_like(Y, 7.0)
    skip = acc.make_desc(n, d_in, d_out, 8, io_dtype=code, dw_dtype=dcode, ldx=d_in + pad, ldw=W.shape[1], ldy=d_out + pad,
                         flags=(flags & acc.ACC_FLAG_W_OUT_IN) | acc.ACC_FLAG_SKIP_SKETCH)
    acc.acc_linear_fwd_act8(skip, af, X, W, Y2, None, None)
    assert torch.equal(Y, Y2)


def test_linear_layer_over_more_tokens_than_a_product(acc):
    """Rows of dY so far apart that 4 GiB hold fewer tokens than there are: the weight gradient is a sum of two products.
    Its operands are exact in bfloat16, so it is off by (n + 8) 2^-24 of the sum of magnitudes and its own rounding."""
    import torch
    n, d_in, d_out, ldy = 2121, 136, 72, 1 << 20
    g = torch.Generator(device="cuda").manual_seed(3)
    wide = torch.empty(n, ldy, dtype=torch.bfloat16, device="cuda")
    dY = wide[:, :d_out]
    dY.copy_(torch.randn(n, d_out, generator=g, device="cuda"))
    X = torch.randn(n, d_in, generator=g, device="cuda").to(torch.bfloat16)
    q, e = acc.alloc_act8(acc.make_act8_desc(n, d_in, format=acc.ACC_ACT8_INT8))
    acc.acc_act8_pack(acc.make_act8_desc(n, d_in, format=acc.ACC_ACT8_INT8), X, q, e)
    xq = torch.from_numpy(orc.act8_unpack(q.cpu().numpy(), e.cpu().numpy(), "int8")).cuda()
    for w_out_in in (False, True):
        desc = acc.make_desc(n, d_in, d_out, 8, ldy=ldy, dw_dtype=acc.ACC_F32, flags=acc.ACC_FLAG_W_OUT_IN if w_out_in else 0)
        dW = torch.full((d_out, d_in) if w_out_in else (d_in, d_out), 7.0, device="cuda")
        wsb, ws = _guarded(torch, (acc.acc_linear_act8_workspace_bytes(desc),), torch.uint8, 0xA5)
        acc.acc_linear_bwd_act8(desc, acc.ACC_ACT8_INT8, wide, None, q, e, None, dW, ws)
        torch.cuda.synchronize()
        assert _guards_hold(wsb, 0xA5)
        want, terms = xq.t() @ dY.double(), xq.abs().t() @ dY.double().abs()
        got = dW.double().t() if w_out_in else dW.double()
        assert bool(((got - want).abs() <= (n + 8) * 2.0 ** -24 * terms + 2.0 ** -24 * want.abs()).all())


def test_captured_and_replayed(acc):
    """One graph of a whole step on a side stream, replayed on new inputs with eager work between, against eager calls."""
    import torch
    n, d, f = 260, 256, 136
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    X, W, dY, G, U, dH = rnd(n, d), rnd(d, d), rnd(n, d), rnd(n, f), rnd(n, f), rnd(n, f)
    desc = acc.make_desc(n, d, d, 8, flags=acc.ACC_FLAG_W_OUT_IN)
    gd = acc.make_gated_desc(n, f, format=acc.ACC_ACT8_INT8)

    def buffers():
        return dict(Y=torch.empty_like(X), dX=torch.empty_like(X), dW=torch.empty_like(W), H=torch.empty_like(G), dG=torch.empty_like(G), dU=torch.empty_like(G))

    def step(o, qe, kept, ws):
        acc.acc_linear_fwd_act8(desc, acc.ACC_ACT8_INT8, X, W, o["Y"], *qe)
        acc.acc_linear_bwd_act8(desc, acc.ACC_ACT8_INT8, dY, W, *qe, o["dX"], o["dW"], ws)
        acc.acc_gated_fwd_act8(gd, G, U, o["H"], *kept)
        acc.acc_gated_bwd_act8(gd, dH, *kept, o["dG"], o["dU"])

    one = acc.make_act8_desc(n, d)
    state = [(buffers(), acc.alloc_act8(one), acc.alloc_gated_act8(gd), torch.empty(acc.acc_linear_act8_workspace_bytes(desc), dtype=torch.uint8, device="cuda"))
             for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*state[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*state[0])
    for r in range(4):
        for t in (X, dY, G, U, dH):
            t.copy_(rnd(*t.shape))
        graph.replay()
        step(*state[1])
        torch.cuda.synchronize()
        for k in state[0][0]:
            assert torch.equal(state[0][0][k], state[1][0][k]), (r, k)


def test_status_of_a_refused_call_leaves_the_outputs(acc):
    import torch
    t = torch.full((64, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    desc = acc.make_act8_desc(64, 64, ldx=60)
    assert acc._lib.acc_act8_unpack(ctypes.byref(desc), t.data_ptr(), t.data_ptr(), t.data_ptr(), None) == -2
    torch.cuda.synchronize()
    assert bool((t == 7.0).all())
