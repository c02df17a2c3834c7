"""Attention through the C ABI at the sizes where the work-groups' shape and number change, with offsets beyond 32 bits, and with two captured
graphs on one workspace; float64 bounds as in the other tests of it."""
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


# (sizes, whether the forward pass has each row's keys in parts)
@pytest.mark.parametrize("kw,parts", [
    (dict(n=520, heads=72, kv=72, d=72), False),                                          # whole rows, 128 of them a work-group
    (dict(n=520, heads=72, kv=72, d=40), False),                                          # the keys' gradients: 64 rows
    (dict(n=520, heads=72, kv=9, d=104, cap=20.0), False),                                # in parts, of 128 rows
    (dict(n=520, heads=72, kv=9, d=40, cap=20.0, bias=True), False),                      # the keys' gradients alone in parts
    (dict(n=520, heads=72, kv=72, d=40, cuts=[3, 9, 70, 71, 200, 260, 300, 340, 400, 455, 510]), False),   # short documents: 64 rows
    (dict(n=520, heads=72, kv=72, d=40, dtype="f32"), False),
    (dict(n=300, heads=72, kv=72, d=40, dtype="f32", causal=False), True),
    (dict(n=1030, heads=16, kv=16, d=24, window=200), False),
    (dict(n=1030, heads=16, kv=16, d=24, window=600), True),
    (dict(n=1030, heads=16, kv=4, d=24, prefix=[700]), True),
    (dict(n=2100, heads=1, kv=1, d=128), True),                                           # as many parts as there are
    (dict(n=2100, heads=1, kv=1, d=128, dtype="f32", cuts=[0, 1, 2099]), True),
], ids=lambda x: str(x))
def test_work_groups_of_every_shape_and_number(acc, kw, parts):
    c = Case(**kw)
    assert (acc.acc_attn_workspace_bytes(c.desc(acc), False) > 0) == parts
    c.check(c.run(acc))


def test_offsets_beyond_32_bits(acc):
    """Rows 2^18 elements apart, 4.4 GB from the first to the last: the same bits as from rows one after another."""
    import torch
    n, ld = 8400, 1 << 18
    c = Case(n, 2, 1, 64, cuts=[0, 100, n - 300, n], window=150)
    dense = c.run(acc)
    t, out = c.to_gpu(), c.outputs()
    wide = torch.empty(n, ld, dtype=c.tdt, device="cuda")
    back = torch.empty(n, ld, dtype=c.tdt, device="cuda")
    q, k, v = (wide[:, a:b] for a, b in ((0, 128), (ld - 128, ld - 64), (ld - 64, ld)))
    o, do = wide[:, 1024:1152], wide[:, 4096:4224]
    for to, x in zip((q, k, v, do), (*c.split(t["qkv"]), t["dO"])):
        to.copy_(x)
    dq, dk, dv = (back[:, a:b] for a, b in ((0, 128), (ld - 128, ld - 64), (ld - 64, ld)))
    desc = acc.make_attn_desc(n, 2, 1, 64, ldq=ld, ldk=ld, ldv=ld, ldo=ld, docs=3, window=150, io_dtype=acc.ACC_BF16, flags=acc.ACC_ATTN_CAUSAL)
    ws = torch.empty(acc.acc_attn_workspace_bytes(desc, True), dtype=torch.uint8, device="cuda")
    acc.acc_attn_fwd(desc, q, k, v, t["starts"], None, None, o, out["lse"], ws)
    acc.acc_attn_bwd(desc, q, k, v, t["starts"], None, None, o, out["lse"], do, dq, dk, dv, ws)
    assert torch.equal(o, dense["o"]) and torch.equal(out["lse"], dense["lse"])
    for got, want in zip((dq, dk, dv), c.split(dense["dqkv"])):
        assert torch.equal(got, want)


def test_two_graphs_on_one_workspace(acc):
    """Nothing is kept there from one call for the next."""
    import torch
    cases = [Case(700, 4, 2, 64, cuts=[0, 100, 650]), Case(300, 8, 1, 32, "f32", causal=False, cap=9.0)]
    want = [c.run(acc) for c in cases]
    ws = torch.empty(max(acc.acc_attn_workspace_bytes(c.desc(acc), True) for c in cases), dtype=torch.uint8, device="cuda")
    held, graphs = [(c.to_gpu(), c.outputs()) for c in cases], []
    for c, (t, out) in zip(cases, held):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            c.call(acc, t, out, ws)
    for order in ((0, 1), (1, 0), (0, 0, 1)):
        for _, out in held:
            for x in out.values():
                x.fill_(float("nan"))
        for k in order:
            graphs[k].replay()
        torch.cuda.synchronize()
        for (_, out), first in zip(held, want):
            assert all(torch.equal(out[k], first[k]) for k in first)
        cases[0].run(acc)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_columns_between_the_heads_hold_anything(acc, dtype):
    """Rows of q, k, v, O and dO whose gaps are not numbers: the same bits as from dense rows."""
    import torch
    c = Case(150, 2, 2, 40, dtype, cuts=[0, 90, 150], cap=12.0)
    dense = c.run(acc)
    t, lse = c.to_gpu(), torch.empty(2, 150, device="cuda")
    wide = lambda: torch.full((150, 96), float("nan"), dtype=c.tdt, device="cuda")  # noqa: E731
    q, k, v, do, o, dq, dk, dv = (wide() for _ in range(8))
    for to, x in zip((q, k, v, do), (*c.split(t["qkv"]), t["dO"])):
        to[:, :80] = x
    desc = acc.make_attn_desc(150, 2, 2, 40, ldq=96, ldk=96, ldv=96, ldo=96, docs=2, cap=12.0, io_dtype=c.desc(acc).io_dtype, flags=acc.ACC_ATTN_CAUSAL)
    ws = torch.empty(acc.acc_attn_workspace_bytes(desc, True), dtype=torch.uint8, device="cuda")
    acc.acc_attn_fwd(desc, q, k, v, t["starts"], None, None, o, lse, ws)
    acc.acc_attn_bwd(desc, q, k, v, t["starts"], None, None, o, lse, do, dq, dk, dv, ws)
    assert torch.equal(o[:, :80], dense["o"]) and bool(torch.isnan(o[:, 80:]).all()) and torch.equal(lse, dense["lse"])
    for got, want in zip((dq, dk, dv), c.split(dense["dqkv"])):
        assert torch.equal(got[:, :80], want) and bool(torch.isnan(got[:, 80:]).all())


def test_numbers_of_documents_that_do_not_ascend_stay_inside(acc):
    """Every first row is brought into [0, n] before it is used: what lies around the tensors is neither read into results nor written."""
    import torch
    n = 200
    c = Case(n, 2, 1, 64, cuts=[0, 60, n])
    t = c.to_gpu()
    guard = lambda rows, cols: torch.full((rows + 64, cols), 7.0, dtype=c.tdt, device="cuda")  # noqa: E731
    for numbers in ([150, 20, 90], [-5, 1 << 40, 30], [0, -(1 << 50), 1 << 50], [200, 200, 0], [199, 0, 400]):
        starts = torch.tensor(numbers, dtype=torch.int64, device="cuda")
        o, back, lse = guard(n, 128), guard(n, 256), torch.full((2 * n + 64,), 7.0, device="cuda")
        desc = c.desc(acc)
        ws = torch.zeros(acc.acc_attn_workspace_bytes(desc, True), dtype=torch.uint8, device="cuda")
        masks = starts, None, None
        acc.acc_attn_fwd(desc, *c.split(t["qkv"]), *masks, o[32:-32], lse[32:-32], ws)
        acc.acc_attn_bwd(desc, *c.split(t["qkv"]), *masks, o[32:-32], lse[32:-32], t["dO"], *c.split(back[32:-32]), ws)
        torch.cuda.synchronize()
        for x in (o, back, lse):
            assert bool((x[:32] == 7.0).all()) and bool((x[-32:] == 7.0).all()), numbers


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [dict(n=1), dict(n=300, window=1), dict(n=65, seq=1, causal=False), dict(n=140, seq=1, prefix=[1] * 140),
                                dict(n=130, window=1, cuts=[0, 1, 34, 130]), dict(n=40, cuts=list(range(41)), cap=5.0)], ids=str)
def test_rows_that_see_one_key_have_no_gradient_of_their_scores(acc, kw, dtype):
    """Zeros, and not what is left of a difference of two sums."""
    c = Case(heads=4, kv=2, d=72, dtype=dtype, **kw)
    out = c.run(acc)
    c.check(out)
    dq, dk, _ = c.split(out["dqkv"])
    assert not dq.any() and not dk.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [dict(n=200), dict(n=200, window=2), dict(n=200, prefix=[1]), dict(n=200, cuts=[0, 1, 90, 91, 200])], ids=str)
def test_the_first_row_sees_one_key(acc, kw, dtype):
    c = Case(heads=2, kv=1, d=64, dtype=dtype, **kw)
    out = c.run(acc)
    c.check(out)
    first = [a for a, b in c.documents()]
    dq = c.split(out["dqkv"])[0]
    assert not dq[first].any() and bool(dq[first[-1] + 1].any())


@pytest.mark.parametrize("kw", [dict(n=300, seq=2), dict(n=300, seq=3, causal=False), dict(n=256, cuts=sorted({0, 256, *range(0, 256, 5)}), cap=9.0),
                                dict(n=900, window=2), dict(n=900, window=64, bias=True), dict(n=64), dict(n=512, seq=64, causal=False)], ids=str)
def test_rows_of_few_keys_have_delta_from_their_probabilities(acc, kw):
    """Scores of size four, so that dP and delta nearly cancel; bounds without the rounding of O."""
    c = Case(heads=4, kv=2, d=64, size=2.0, **kw)
    c.check(c.run(acc))
