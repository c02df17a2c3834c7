"""An MLP's second half through the C calls with nothing kept for its last product: the gated activation's backward call forms H again,
and the last product's weight gradient is taken from a checkpoint made of that.

Tolerances as in test_gpu_act8.py: half a step of bfloat16 is 2^-8 of a value, of float32 2^-24; a float sum of k terms is off by k 2^-24 of
the sum of magnitudes at most."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from oracle import train_oracle as orc


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,f,d", [(1, 8, 16), (77, 136, 72), (300, 520, 264)])
def test_weight_gradient_from_the_activation_formed_again(n, f, d, dtype, fmt):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_01255_amd import binding as acc
    code, tdt, half = (acc.ACC_BF16, torch.bfloat16, 2.0 ** -8) if dtype == "bf16" else (acc.ACC_F32, torch.float32, 2.0 ** -24)
    af = acc.ACC_ACT8_E4M3 if fmt == "e4m3" else acc.ACC_ACT8_INT8
    g = torch.Generator(device="cuda").manual_seed(n + f)
    rnd = lambda r, c, s: (torch.randn(r, c, generator=g, device="cuda") * s).to(tdt)  # noqa: E731
    both, w, dy = rnd(n, 2 * f, 2.0), rnd(d, f, 0.1), rnd(n, d, 0.1)
    gd = acc.make_gated_desc(n, f, ldg=2 * f, io_dtype=code, format=af)
    one = acc.make_act8_desc(n, f, io_dtype=code, format=af)
    lin = acc.make_desc(n, f, d, 8, io_dtype=code, flags=acc.ACC_FLAG_W_OUT_IN | acc.ACC_FLAG_SKIP_SKETCH)
    kept = acc.alloc_gated_act8(gd)
    H, Y = torch.empty(n, f, dtype=tdt, device="cuda"), torch.empty(n, d, dtype=tdt, device="cuda")
    acc.acc_gated_fwd_act8(gd, both[:, :f], both[:, f:], H, *kept)
    acc.acc_linear_fwd_act8(lin, af, H, w, Y, None, None)
    del H
    lin.flags = acc.ACC_FLAG_W_OUT_IN
    dH, dboth, again, dW = torch.empty(n, f, dtype=tdt, device="cuda"), torch.empty_like(both), torch.empty(n, f, dtype=tdt, device="cuda"), torch.empty_like(w)
    acc.acc_linear_bwd_act8(lin, af, dy, w, None, None, dH, None, None)
    acc.acc_gated_bwd_act8(gd, dH, *kept, dboth[:, :f], dboth[:, f:], again)
    q, e = acc.alloc_act8(one)
    acc.acc_act8_pack(one, again, q, e)
    ws = torch.empty(acc.acc_linear_act8_workspace_bytes(lin), dtype=torch.uint8, device="cuda")
    acc.acc_linear_bwd_act8(lin, af, dy, None, q, e, None, dW, ws)
    torch.cuda.synchronize()
    f64 = lambda t: t.cpu().double().numpy()  # noqa: E731
    hq, dY = orc.act8_unpack(*orc.act8_pack(f64(again), fmt), fmt), f64(dy)
    want = dY.T @ hq
    assert np.all(np.abs(f64(dW) - want) <= half * 1.01 * np.abs(want) + (n + 8) * 2.0 ** -24 * (np.abs(dY).T @ np.abs(hq)))
    # what was formed again is the activation of the checkpoints (sigmoid in float32: (|g| + 8) 2^-22 of it)
    gq, uq = (orc.act8_unpack(kept[k].cpu().numpy(), kept[k + 1].cpu().numpy(), fmt) for k in (0, 2))
    h = orc.gated(gq, uq)
    assert np.all(np.abs(f64(again) - h) <= (half * 1.01 + (np.abs(gq) + 8) * 2.0 ** -22) * np.abs(h) + 1e-45)
