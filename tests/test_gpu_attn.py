"""Attention over documents through the C ABI against float64, every element within its bound of roundings."""
import pytest

pytestmark = pytest.mark.gpu

from attn_util import Case


@pytest.fixture(scope="module")
def acc():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_01255_amd import binding
    return binding


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 333])
def test_one_causal_document_of_any_length(acc, n, dtype):
    c = Case(n, 4, 2, 64, dtype)
    c.check(c.run(acc))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [8, 16, 40, 64, 72, 80, 96, 104, 120, 128])
def test_channels_of_a_head(acc, d, dtype):
    c = Case(150, 3, 3, d, dtype, cuts=[0, 90, 150])
    c.check(c.run(acc))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv", [(1, 1), (2, 1), (6, 2), (8, 1), (5, 5), (9, 3)])
def test_heads_that_share_keys(acc, heads, kv, dtype):
    c = Case(140, heads, kv, 32, dtype, causal=heads % 2 == 0)
    c.check(c.run(acc))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cuts", [[0, 0, 1, 3, 3, 64, 70, 200, 200], [5, 40, 41, 190], [200, 200], [0, 0], [7, 200], [0, 193], list(range(0, 201)),
                                  sorted([0] * 70 + list(range(0, 200, 3)) + [150] * 40), [0] * 4300 + [100, 200] + [200] * 90], ids=str)
def test_documents(acc, cuts, dtype):
    """Empty ones, ones of one row, rows of none (zeros), more of them than are looked through at once."""
    c = Case(200, 2, 1, 64, dtype, cuts=cuts)
    out = c.run(acc)
    c.check(out)
    import torch
    none = torch.ones(200, dtype=torch.bool)
    none[cuts[0]:cuts[-1]] = False
    assert not out["o"][none.cuda()].any() and not out["dqkv"][none.cuda()].any() and bool((out["lse"][:, none.cuda()] == -torch.inf).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n,seq", [(150, 50), (150, 64), (257, 128), (5, 9), (300, 1)])
def test_sequences_of_one_length(acc, n, seq, causal, dtype):
    c = Case(n, 2, 2, 40, dtype, seq=seq, causal=causal)
    c.check(c.run(acc))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 2, 31, 64, 100, 260, 10 ** 9])
def test_windows(acc, window, dtype):
    c = Case(270, 2, 1, 64, dtype, cuts=[3, 30, 270], window=window)
    c.check(c.run(acc))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("prefix", [[0, 0, 0], [1, 200, 7], [130, -5, 10 ** 12], [64, 32, 1]])
def test_prefixes(acc, prefix, dtype):
    c = Case(300, 2, 1, 64, dtype, cuts=[0, 180, 290, 300], prefix=prefix)
    c.check(c.run(acc))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap,bias,window,causal,scale", [(30.0, False, 0, True, 0.0), (5.0, False, 0, False, 0.3), (0.0, True, 0, True, 0.0), (0.0, True, 0, False, 0.0),
                                                          (20.0, True, 40, True, 0.5), (0.0, False, 0, True, 1e-3), (1e-3, False, 0, True, 0.0)])
def test_caps_biases_and_scales(acc, cap, bias, window, causal, scale, dtype):
    c = Case(200, 4, 2, 64, dtype, cuts=[0, 120, 200], cap=cap, bias=bias, window=window, causal=causal, scale=scale, size=2.0)
    c.check(c.run(acc))


def test_large_scores(acc):
    """Logits of some hundreds: one key takes everything, and nothing overflows."""
    c = Case(160, 2, 1, 64, "f32", size=8.0)
    c.check(c.run(acc))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_is_not_finite_stays_in_its_document(acc, dtype):
    import torch
    c = Case(260, 2, 1, 64, dtype, cuts=[10, 60, 90, 200], bias=True)
    clean = c.run(acc)
    c.qkv[65], c.dO[70] = float("nan"), float("inf")
    c.qkv[80, ::3] = float("inf")
    for rows in (slice(0, 10), slice(200, 260)):   # of no document
        c.qkv[rows], c.dO[rows] = float("nan"), float("nan")
    out = c.run(acc)
    others = torch.tensor([i for i in range(260) if not 60 <= i < 90])
    for name in ("o", "dqkv"):
        assert torch.equal(out[name][others], clean[name][others]), name
    assert torch.equal(out["lse"][:, others], clean["lse"][:, others])
    assert bool(torch.isnan(out["o"][65:90]).all())   # rows that see what is not a number


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_only_its_rows_are_written(acc, dtype):
    """Outputs that are column blocks of a wider matrix: the gaps stay as they were."""
    import torch
    c = Case(70, 2, 1, 40, dtype)
    t, wide = c.to_gpu(), c.outputs()
    dense = c.run(acc)
    ld = 4 * 40 + 16
    desc = acc.make_attn_desc(70, 2, 1, 40, ldq=160, ldk=160, ldv=160, ldo=2 * 40 + 8, io_dtype=c.desc(acc).io_dtype)
    o = torch.full((70, 88), 7.0, dtype=c.tdt, device="cuda")
    do = torch.full((70, 88), float("nan"), dtype=c.tdt, device="cuda")
    do[:, :80] = t["dO"]
    ws = torch.empty(acc.acc_attn_workspace_bytes(desc, True), dtype=torch.uint8, device="cuda")
    q, k, v = c.split(t["qkv"])
    acc.acc_attn_fwd(desc, q, k, v, None, None, None, o, wide["lse"], ws)
    dq, dk, dv = (torch.full((70, 160), 7.0, dtype=c.tdt, device="cuda") for _ in range(3))
    acc.acc_attn_bwd(desc, q, k, v, None, None, None, o, wide["lse"], do, dq, dk, dv, ws)
    assert torch.equal(o[:, :80], dense["o"]) and bool((o[:, 80:] == 7.0).all()) and ld
    for got, want, width in zip((dq, dk, dv), c.split(dense["dqkv"]), (80, 40, 40)):
        assert torch.equal(got[:, :width], want) and bool((got[:, width:] == 7.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_twice_the_same_bits_on_another_stream_and_in_a_graph(acc, dtype):
    import torch
    c = Case(500, 8, 2, 64, dtype, cuts=[0, 100, 500], cap=20.0)
    first = c.run(acc)
    side = torch.cuda.Stream()
    t, out = c.to_gpu(), c.outputs()
    ws = torch.empty(acc.acc_attn_workspace_bytes(c.desc(acc), True), dtype=torch.uint8, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    c.call(acc, t, out, ws, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(out[k], first[k]) for k in first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.call(acc, t, out, ws)
    for _ in range(3):
        for x in out.values():
            x.fill_(float("nan"))
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[k], first[k]) for k in first)
        c.run(acc)   # the program's own work between the replays
    t["qkv"].copy_(t["qkv"] * 0.5)
    graph.replay()
    torch.cuda.synchronize()
    c.qkv = c.qkv * 0.5
    again = c.run(acc)
    assert all(torch.equal(out[k], again[k]) for k in again)


def test_gradients_against_differences(acc):
    """The derivative of sum(O . dO) along a random direction, from two forward passes in float32."""
    import torch
    c = Case(60, 4, 2, 24, "f32", cuts=[0, 25, 60], cap=15.0, bias=True, size=1.5)
    out = c.run(acc)
    g = torch.Generator().manual_seed(3)
    way = torch.randn(c.qkv.shape, generator=g)
    step = 2.0 ** -7
    base, ends = c.qkv.clone(), []
    for sign in (1, -1):
        c.qkv = base + sign * step * way
        ends.append(float((c.run(acc, backward=False)["o"].cpu().double() * c.dO.double()).sum()))
    slope = (ends[0] - ends[1]) / (2 * step)
    want = float((out["dqkv"].cpu().double() * way.double()).sum())
    # the third derivative's part is step^2 of the value's size; the outputs' errors 2^-22 of sum |O dO| over the step
    scale = float((out["dqkv"].cpu().double() * way.double()).abs().sum())
    assert abs(slope - want) < 5e-3 * scale, (slope, want, scale)
