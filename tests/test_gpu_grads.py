"""The norm over gradients and their scaling through the C ABI against float64.

Dense squares are summed in double: the norm is off by its rounding to float alone.  Of a factored gradient the two sums over rows are float
sums of at most 2048 products: each element is off by at most 2048 x 2^-24 of the sum of magnitudes, and the norm by what that makes of
sum (L^T L) o (G^T G), over twice the norm."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def acc():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_01255_amd import binding
    return binding


def _randn(shape, dtype, seed, size=1.0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * size).to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def _norm(acc, tensors, factors, max_norm=1.0, stream=None):
    import torch
    out = torch.full((2,), 7.0, device="cuda")
    t = acc.make_grad_list(tensors)
    ws = torch.empty(acc.acc_grad_norm_workspace_bytes(t, factors), dtype=torch.uint8, device="cuda").fill_(0xFF)
    acc.acc_grad_norm(t, factors, max_norm, out, ws, stream=stream)
    torch.cuda.synchronize()
    return [float(x) for x in out]


def _no_factors(acc):
    return acc.make_factor_list([], [])


def _exact(tensors):
    return math.sqrt(sum(float(t.double().square().sum()) for t in tensors))


SIZES = [1, 2, 7, 8, 9, 255, 2048, 2049, 65535, 65536, 65537, 200003]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", SIZES)
def test_one_tensor(acc, n, dtype):
    t = _randn((n,), dtype, n)
    norm, by = _norm(acc, [t], _no_factors(acc), 0.5)
    want = _exact([t])
    assert abs(norm - want) <= 2.0 ** -23 * want
    assert abs(by - min(1.0, 0.5 / (want + 1e-6))) <= 2.0 ** -23


@pytest.mark.parametrize("count", [0, 1, 63, 64, 65, 200])
def test_any_number_of_tensors_of_both_types(acc, count):
    import torch
    ts = [_randn((SIZES[i % len(SIZES)] % 5000,), ("bf16", "f32")[i % 2], i, 10.0 ** (i % 5 - 2)) for i in range(count)]
    ts.insert(count // 2, torch.empty(0, device="cuda"))
    norm, by = _norm(acc, ts, _no_factors(acc), 3.0)
    want = _exact(ts)
    assert abs(norm - want) <= 2.0 ** -23 * want and abs(by - min(1.0, 3.0 / (want + 1e-6))) <= 2.0 ** -23


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("offset", [0, 1, 3, 4, 7])
def test_tensors_that_start_anywhere(acc, offset, dtype):
    import torch
    whole = _randn((70000,), dtype, 5)
    t = whole[offset:offset + 66001]
    norm, by = _norm(acc, [t], _no_factors(acc))
    want = _exact([t])
    assert abs(norm - want) <= 2.0 ** -23 * want
    kept = whole.clone()
    acc.acc_grad_scale(acc.make_grad_list([t]), torch.full((1,), 0.25, device="cuda"))
    torch.cuda.synchronize()
    assert torch.equal(whole[:offset], kept[:offset]) and torch.equal(whole[offset + 66001:], kept[offset + 66001:])
    assert torch.equal(t, kept[offset:offset + 66001] * 0.25)


@pytest.mark.parametrize("size", [1e-30, 1e-22, 1e19, 1e38])
def test_squares_beyond_float(acc, size):
    t = _randn((3000,), "f32", 2, 1.0).clamp(-3, 3) * size
    norm, _ = _norm(acc, [t], _no_factors(acc))
    want = _exact([t])
    assert norm == math.inf if want > 3.4028235e38 else abs(norm - want) <= 2.0 ** -23 * want


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_what_is_not_finite_shows(acc, what, dtype):
    t = _randn((70000,), dtype, 3)
    t[69999] = what
    norm, by = _norm(acc, [_randn((100,), dtype, 1), t], _no_factors(acc))
    if math.isnan(what):
        assert math.isnan(norm) and math.isnan(by)
    else:
        assert norm == math.inf and by == 0.0


def test_no_gradient_and_zeros(acc):
    import torch
    assert _norm(acc, [], _no_factors(acc)) == [0.0, 1.0]
    assert _norm(acc, [torch.zeros(1000, device="cuda")], _no_factors(acc), 0.5) == [0.0, 1.0]
    assert _norm(acc, [torch.ones(4, device="cuda")], _no_factors(acc), math.inf) == [2.0, 1.0]
    assert _norm(acc, [torch.ones(4, device="cuda")], _no_factors(acc), 0.0) == [2.0, 0.0]


def _pair(acc, d_in, d_out, r, dtype, oi, seed=0, pad=0):
    left = _randn((d_in, r + pad), dtype, seed, 3.0)[:, :r]
    gr = _randn((d_out, r + pad) if oi else (r, d_out + pad), dtype, seed + 1, 0.1)
    return left, gr[:, :r] if oi else gr[:, :d_out]


def _factor_bound(left, gr, oi):
    x, y = left.double(), gr.double() if oi else gr.double().t()
    a, b, aa, bb = x.t() @ x, y.t() @ y, x.abs().t() @ x.abs(), y.abs().t() @ y.abs()
    square = float((x @ y.t()).square().sum())
    return square, 2048 * 2.0 ** -24 * float((aa * b.abs() + a.abs() * bb + 2048 * 2.0 ** -24 * aa * bb).sum())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("oi", [True, False])
@pytest.mark.parametrize("d_in,d_out,r,pad", [(8, 8, 8, 0), (64, 128, 16, 0), (520, 264, 32, 8), (2048, 72, 128, 0), (2056, 4104, 136, 0), (300 * 8, 1000, 256, 16),
                                              (72, 40, 264, 8)])
def test_one_factored_gradient(acc, d_in, d_out, r, pad, oi, dtype):
    left, gr = _pair(acc, d_in, d_out, r, dtype, oi, pad=pad)
    norm, _ = _norm(acc, [], acc.make_factor_list([left], [gr], acc.ACC_FLAG_W_OUT_IN if oi else 0))
    square, bound = _factor_bound(left, gr, oi)
    assert abs(norm ** 2 - square) <= bound + 2.0 ** -22 * square, (norm, math.sqrt(square))


def test_many_factored_gradients_and_tensors_together(acc):
    import torch
    lists, square, bound = {True: ([], []), False: ([], [])}, 0.0, 0.0
    for i in range(41):
        oi, dtype = i % 3 != 0, ("bf16", "f32")[i % 2]
        left, gr = _pair(acc, 8 * (i + 1), 8 * (50 - i), (8, 16, 136)[i % 3], dtype, oi, seed=10 * i)
        lists[oi][0].append(left)
        lists[oi][1].append(gr)
        s, b = _factor_bound(left, gr, oi)
        square, bound = square + s, bound + b
    tables = [acc.make_factor_list(*lists[oi], acc.ACC_FLAG_W_OUT_IN if oi else 0) for oi in (True, False)]
    both = (acc.AccGradFactors * 41)(*tables[0], *tables[1])
    dense = [_randn((1000,), "bf16", 3), _randn((77777,), "f32", 4, 0.1)]
    norm, by = _norm(acc, dense, both, 2.0)
    square += _exact(dense) ** 2
    assert abs(norm ** 2 - square) <= bound + 2.0 ** -22 * square
    assert abs(by - 2.0 / (norm + 1e-6)) <= 2.0 ** -22 * by
    assert torch.cuda.is_available()


def test_factors_whose_product_vanishes(acc):
    """Columns of the left factor that the right one has zeros for."""
    left, gr = _pair(acc, 256, 128, 16, "f32", True)
    left[:, 8:] = 0.0
    gr[:, :8] = 0.0
    assert _norm(acc, [], acc.make_factor_list([left], [gr], acc.ACC_FLAG_W_OUT_IN)) == [0.0, 1.0]


@pytest.mark.parametrize("src,dst", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
def test_scaling_into_other_tensors(acc, src, dst):
    import torch
    ts = [_randn((n,), src, n) for n in SIZES]
    outs = [torch.full((n,), math.nan, dtype=torch.bfloat16 if dst == "bf16" else torch.float32, device="cuda") for n in SIZES]
    kept = [t.clone() for t in ts]
    by = torch.tensor([0.3], device="cuda")
    acc.acc_grad_scale(acc.make_grad_list(ts, outs), by)
    torch.cuda.synchronize()
    for t, k, o in zip(ts, kept, outs):
        assert torch.equal(t, k) and torch.equal(o, (k.float() * by).to(o.dtype))   # one product in float, one rounding
    by.fill_(1.0)
    acc.acc_grad_scale(acc.make_grad_list(ts, outs), by)
    torch.cuda.synchronize()
    assert all(torch.equal(o, t.to(o.dtype)) for t, o in zip(ts, outs))


def test_in_place_and_the_same_bits_in_a_graph(acc):
    import torch
    ts = [_randn((n,), ("bf16", "f32")[n % 2], n, 0.1) for n in SIZES * 8]
    left, gr = _pair(acc, 512, 256, 64, "bf16", True)
    factors, start = acc.make_factor_list([left], [gr], acc.ACC_FLAG_W_OUT_IN), [t.clone() for t in ts] + [gr.clone()]
    table, everything = acc.make_grad_list(ts), acc.make_grad_list(ts + [gr])
    out = torch.empty(2, device="cuda")
    ws = torch.empty(acc.acc_grad_norm_workspace_bytes(table, factors), dtype=torch.uint8, device="cuda")

    def step():
        acc.acc_grad_norm(table, factors, 1.0, out, ws)
        acc.acc_grad_scale(everything, out[1:])

    def reset():
        for t, s in zip(ts + [gr], start):
            t.copy_(s)

    step()
    torch.cuda.synchronize()
    first, norm = [t.clone() for t in ts + [gr]], out.clone()
    assert float(norm[1]) < 1.0 and all(torch.equal(t, (s.float() * norm[1]).to(s.dtype)) for t, s in zip(first, start))
    reset()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    del table, everything, factors   # the graph has the tables
    for _ in range(3):
        reset()
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, norm) and all(torch.equal(a, b) for a, b in zip(first, ts + [gr]))
        _norm(acc, [start[0]], _no_factors(acc))   # the program's own work between the replays
