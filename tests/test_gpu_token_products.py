"""Every form of the bfloat16 weight gradient over the tokens, each at a size for which the library chooses it (asserted through
plan_util): tiles, stages, parts that a second launch adds up, bfloat16 and float results, written and added to.

The checkpoint is exact in bfloat16, so a result is off by its float sum, (k + 64 parts + 8) 2^-24 of the sum of magnitudes, and its own
rounding, half a step: 2^-8 (bfloat16) or 2^-24."""
import pytest

pytestmark = pytest.mark.gpu

import plan_util as pu

# rows, columns, tokens; tile, whether it is one round, whether there are parts (the persistent kernel, for a bfloat16 result that is
# written alone: below)
FORMS = [
    (64, 64, 40, "64x64", True, False), (512, 2056, 40, "64x64", False, False), (64, 64, 2049, "64x64", True, True),
    (136, 2048, 8192, "64x64", False, True), (512, 512, 8192, "64x64", True, True),
    (512, 2056, 300, "128x64", True, False), (1544, 2048, 40, "128x64", False, False), (2048, 136, 8192, "128x64", True, True),
    (4136, 136, 8192, "128x64", False, True), (512, 512, 32768, "128x64", True, True),
    (1024, 4096, 8192, "128x128", True, False), (1544, 4096, 40, "128x128", False, False), (264, 2048, 16384, "128x128", False, True),
    (1032, 4136, 3387, "192x128", True, False), (136, 57176, 40, "192x128", False, False), (136, 4096, 16384, "192x128", True, True),
    (136, 12072, 7959, "192x128", False, True),
]


def _run(m, n, k, w_out_in, dw, add, seed=0):
    import torch
    from paper_2605_01255_amd import binding as acc
    g = torch.Generator(device="cuda").manual_seed(m + n + k + seed)
    d_out, d_in = (m, n) if w_out_in else (n, m)
    dwt = torch.bfloat16 if dw == "bf16" else torch.float32
    one = acc.make_act8_desc(k, d_in, format=acc.ACC_ACT8_INT8)
    q, e = acc.alloc_act8(one)
    acc.acc_act8_pack(one, torch.randn(k, d_in, generator=g, device="cuda").to(torch.bfloat16), q, e)
    x = torch.empty(k, d_in, device="cuda")
    acc.acc_act8_unpack(acc.make_act8_desc(k, d_in, io_dtype=acc.ACC_F32, format=acc.ACC_ACT8_INT8), q, e, x)
    wide = torch.full((k, d_out + 8), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, :d_out] = torch.randn(k, d_out, generator=g, device="cuda")
    flags = (acc.ACC_FLAG_W_OUT_IN if w_out_in else 0) | (acc.ACC_FLAG_DW_ACCUMULATE if add else 0)
    desc = acc.make_desc(k, d_in, d_out, 8, ldy=d_out + 8, dw_dtype=acc.ACC_BF16 if dw == "bf16" else acc.ACC_F32, flags=flags)
    before = torch.randn(m, n, generator=g, device="cuda").to(dwt)
    buf = torch.full((m * n + 128,), 7.0, dtype=dwt, device="cuda")
    dW = buf[64:-64].view(m, n)
    dW.copy_(before if add else torch.full_like(before, float("nan")))
    need = acc.acc_linear_act8_workspace_bytes(desc)
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")   # NaN bits
    acc.acc_linear_bwd_act8(desc, acc.ACC_ACT8_INT8, wide, None, q, e, None, dW, ws, ws_bytes=need)
    torch.cuda.synchronize()
    assert bool((ws[need:] == 0xFF).all()) and bool((buf[:64] == 7.0).all()) and bool((buf[-64:] == 7.0).all())
    a, b = (wide[:, :d_out].double(), x.double()) if w_out_in else (x.double(), wide[:, :d_out].double())
    want, terms = a.t() @ b, a.abs().t() @ b.abs()
    if add:
        want, terms = want + before.double(), terms + before.double().abs()
    return dW, want, terms


@pytest.mark.parametrize("dw,add", [("bf16", False), ("bf16", True), ("f32", False), ("f32", True)])
@pytest.mark.parametrize("m,n,k,tile,one_round,parts", FORMS, ids=lambda v: str(v))
def test_a_form_of_the_weight_gradient(m, n, k, tile, one_round, parts, dw, add):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    plan = pu.token_product(m, n, k, float_or_sum=add or dw == "f32")
    assert (plan.tile, plan.one_round, plan.parts > 1) == (tile, one_round, parts), plan
    got, want, terms = _run(m, n, k, (m + k) % 16 == 0, dw, add)
    bound = (2.0 ** -8 if dw == "bf16" else 2.0 ** -24) * 1.01 * want.abs() + (k + 64 * plan.parts + 8) * 2.0 ** -24 * terms
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), float((off / bound).max())


@pytest.mark.parametrize("m,n,k", [(4096, 4096, 129), (3848, 4096, 300)])
@pytest.mark.parametrize("w_out_in", [False, True])
def test_the_persistent_form(m, n, k, w_out_in):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    assert pu.token_product(m, n, k).tile == "256x256" and pu.token_product(m, n, k, float_or_sum=True).tile != "256x256"
    got, want, terms = _run(m, n, k, w_out_in, "bf16", False)
    off = (got.double() - want).abs()
    assert bool((off <= 2.0 ** -8 * 1.01 * want.abs() + (k + 72) * 2.0 ** -24 * terms).all())
