"""The table's lookup and gradient on more tokens than a launch has work-groups for parts of 32: whole numbers, whose sums are exact in float."""
import pytest

pytestmark = pytest.mark.gpu


def test_more_than_half_a_billion_tokens():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_01255_amd import binding as acc
    n, d, v = (1 << 29) + 77, 8, 5000
    g = torch.Generator(device="cuda").manual_seed(1)
    ids = torch.randint(0, v, (n,), generator=g, device="cuda")
    ids[5::1000] = -1
    ids[(1 << 28):(1 << 28) + (1 << 22)] = 17                    # a word with far more tokens than the others
    W = torch.randn(v, d, generator=g, device="cuda").to(torch.bfloat16)
    pattern = (torch.arange(4, device="cuda").view(4, 1) + torch.arange(d, device="cuda")) % 4
    dY = pattern.to(torch.bfloat16).repeat((n + 3) // 4, 1)[:n]  # row i holds (i + column) mod 4
    desc = acc.make_embed_desc(n, d, v, scale=1.0, dw_dtype=acc.ACC_F32)
    Y = torch.empty(n, d, dtype=torch.bfloat16, device="cuda")
    acc.acc_embed_fwd(desc, W, ids, Y)
    for a in range(0, n, 1 << 22):
        part = ids[a:a + (1 << 22)]
        assert torch.equal(Y[a:a + (1 << 22)], W[part.clamp_min(0)] * (part >= 0).unsqueeze(1)), a
    del Y
    dW = torch.full((v, d), float("nan"), device="cuda")
    ws = torch.empty(acc.acc_embed_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    acc.acc_embed_bwd(desc, ids, dY, dW, ws)
    torch.cuda.synchronize()
    counts = torch.zeros(v, 4, dtype=torch.float64, device="cuda")   # tokens of a word by their number mod 4
    for k in range(4):
        some = ids[k::4]
        counts[:, k] = torch.bincount(some[some >= 0], minlength=v).double()
    want = counts @ pattern.double()
    assert float(want.max()) < 1 << 24 and torch.equal(dW.double(), want)
