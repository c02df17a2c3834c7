"""Values of attention with heads of 128 channels, shared keys and full work-groups, thousands of rows: some key heads of a call against float64."""
import pytest

pytestmark = pytest.mark.gpu

from attn_util import Case

FIRST, ROWS, BEHIND = 70, 2300, 1800   # the document that is compared stands between two others


@pytest.fixture(scope="module")
def acc():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_01255_amd import binding
    return binding


@pytest.mark.parametrize("heads,kv,more", [(32, 16, {}), (16, 4, {}), (16, 4, dict(cap=30.0, window=1000)), (32, 16, dict(prefix=[3, 900, 0], cap=50.0)),
                                           (20, 4, dict(causal=False))], ids=str)
def test_key_heads_of_a_large_call(acc, heads, kv, more):
    import torch
    n, d, group = FIRST + ROWS + BEHIND, 128, heads // kv
    c = Case(n, heads, kv, d, cuts=[0, FIRST, FIRST + ROWS, n], **more)
    out = c.run(acc)
    rows = slice(FIRST, FIRST + ROWS)
    for head in (0, kv - 1):
        one = Case(ROWS, group, 1, d, **{**more, **({"prefix": more["prefix"][1:2]} if "prefix" in more else {})})
        pick = lambda t, width: t[rows, head * width:(head + 1) * width]  # noqa: E731
        parts = lambda t: torch.cat([pick(x, w) for x, w in zip(c.split(t), (group * d, d, d))], 1)  # noqa: E731
        one.qkv, one.dO = parts(c.qkv), pick(c.dO, group * d).contiguous()
        one.check({"o": pick(out["o"], group * d), "lse": out["lse"][head * group:(head + 1) * group, rows], "dqkv": parts(out["dqkv"])})
