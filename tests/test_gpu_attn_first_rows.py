"""The gradients of a long document's first rows, which see at most 64 keys, against float64 with bounds that leave the rounding of O out.

Row i of a causal document sees the rows up to i (and the prefix), so the first 64 rows' outputs, log-sum-exps and dQ are those of a document of
64 rows; with dO zero behind them dK and dV are too, because rows without dO give none."""
import pytest

pytestmark = pytest.mark.gpu

from attn_util import Case

FEW = 64


@pytest.fixture(scope="module")
def acc():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_01255_amd import binding
    return binding


@pytest.mark.parametrize("kw", [
    dict(n=400, heads=32, kv=8, d=64),                                                        # work-groups of 128 rows
    dict(n=1100, heads=16, kv=4, d=128, cuts=[3, 400, 1090]),                                 # in parts
    dict(n=520, heads=72, kv=72, d=40, cuts=[0, 150, 151, 231, 520], cap=20.0, bias=True),
    dict(n=520, heads=72, kv=9, d=104, seq=130),
    dict(n=520, heads=36, kv=36, d=80, window=100),
    dict(n=520, heads=36, kv=12, d=24, seq=260, prefix=[40, 64]),
    dict(n=300, heads=2, kv=1, d=64),                                                         # of 64 rows
], ids=str)
def test_first_rows_of_long_documents_have_delta_from_their_probabilities(acc, kw):
    """Scores of size four, so that dP and delta nearly cancel."""
    import torch
    c = Case(size=2.0, **kw)
    documents = c.documents()
    rows = torch.cat([torch.arange(a, min(a + FEW, b)) for a, b in documents])
    rest = torch.ones(c.n, dtype=torch.bool)
    rest[rows] = False
    c.dO[rest] = 0
    out = c.run(acc)
    cuts = [0]
    for a, b in documents:
        cuts.append(cuts[-1] + min(b - a, FEW))
    small = {**kw, "n": len(rows), "cuts": cuts, "seq": 0}
    if small.get("prefix"):
        assert max(small["prefix"]) <= FEW
    want = Case(size=2.0, **small)
    want.qkv, want.dO = c.qkv[rows], c.dO[rows]
    at = rows.cuda()
    want.check({"o": out["o"][at], "lse": out["lse"][:, at], "dqkv": out["dqkv"][at]})
    _, dk, dv = c.split(out["dqkv"])
    assert not dk[rest.cuda()].any() and not dv[rest.cuda()].any()
