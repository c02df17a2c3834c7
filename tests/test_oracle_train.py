"""Pins of oracle/train_oracle.py: the 8-bit formats against PyTorch's casts and hand-made blocks, gradients against differences."""
import numpy as np
import pytest
import torch

from oracle import train_oracle as orc
from paper_2605_01255_amd import inputs


def test_the_tables_hold_the_formats():
    t = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    np.testing.assert_array_equal(orc.VALUES["e4m3"], t.view(torch.float8_e4m3fn).double().numpy())
    finite = [c for c in range(256) if c != 0x80]
    np.testing.assert_array_equal(orc.VALUES["int8"][finite], t.view(torch.int8).double().numpy()[finite])
    assert np.isnan(orc.VALUES["int8"][0x80])


def test_nearest_codes_are_those_of_the_library_casts():
    rng = np.random.default_rng(5)
    y = np.concatenate([rng.uniform(-448, 448, 4000), rng.normal(0, 0.01, 4000), np.arange(-256, 257) / 2.0]).astype(np.float32)
    mids = (orc.VALUES["e4m3"][:0x7E] + orc.VALUES["e4m3"][1:0x7F]) / 2      # every tie
    y = np.concatenate([y, mids, -mids]).astype(np.float32)
    want = torch.from_numpy(y).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(orc._nearest_code(y.astype(np.float64), "e4m3"), want)
    np.testing.assert_array_equal(want, inputs.f32_to_fp8_bits(y))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_the_scale_is_the_least_that_holds_the_block(fmt):
    rng = np.random.default_rng(6)
    x = rng.normal(0, 1, (96, 40)) * 2.0 ** rng.integers(-60, 60, (1, 40))
    x[:32, 0], x[:32, 1] = 0.0, 1e-35
    x[3, 2], x[4, 3] = np.inf, np.nan
    q, e = orc.act8_pack(x, fmt)
    e = e.astype(np.float64) - 127
    for b in range(3):
        big = np.where(np.isfinite(x[32 * b:32 * b + 32]), np.abs(x[32 * b:32 * b + 32]), 0).max(axis=0)
        assert np.all(big <= orc.LIMIT[fmt] * 2.0 ** e[b])
        assert np.all((e[b] == -100) | (big > orc.LIMIT[fmt] * 2.0 ** (e[b] - 1)))
    assert e[0, 0] == e[0, 1] == -100
    back = orc.act8_unpack(q, (e + 127).astype(np.uint8), fmt)
    assert np.isnan(back[3, 2]) and np.isnan(back[4, 3]) and np.isnan(back).sum() == 2
    fine = np.isfinite(x) & np.isfinite(back)
    step = 2.0 ** np.repeat(e, 32, axis=0)
    # half a step: of the integer grid, or 2^-4 of the value and 2^-10 near zero for e4m3
    half = np.broadcast_to(step / 2, x.shape) if fmt == "int8" else np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * step)
    assert np.all(np.abs(back - x)[fine] <= half[fine])


def test_gated_gradients_are_differences():
    rng = np.random.default_rng(7)
    g, u, dh = rng.normal(0, 2, (3, 5, 7))
    dg, du = orc.gated_bwd(dh, g, u)
    h = 1e-6
    np.testing.assert_allclose(dg, dh * (orc.gated(g + h, u) - orc.gated(g - h, u)) / (2 * h), rtol=1e-7, atol=1e-9)
    np.testing.assert_allclose(du, dh * (orc.gated(g, u + h) - orc.gated(g, u - h)) / (2 * h), rtol=1e-7, atol=1e-9)


def test_cross_entropy_is_torchs_and_its_gradients_are_differences():
    rng = np.random.default_rng(8)
    x, w = rng.normal(0, 1, (6, 5)), rng.normal(0, 1, (11, 5))
    t = np.array([0, 10, -100, 4, 4, -1])
    dloss = rng.normal(0, 1, 6)
    loss, lse = orc.linear_ce(x, w, t)
    z = torch.from_numpy(x @ w.T)
    t2 = torch.from_numpy(np.where(t < 0, -100, t))
    np.testing.assert_allclose(loss, torch.nn.functional.cross_entropy(z, t2, reduction="none").numpy(), rtol=1e-12, atol=1e-14)
    np.testing.assert_allclose(lse, torch.logsumexp(z, 1).numpy(), rtol=1e-12)
    dx, dw = orc.linear_ce_bwd(x, w, t, dloss)
    h = 1e-6
    for i, j in ((0, 0), (2, 1), (3, 4), (5, 2)):
        d = np.zeros_like(x)
        d[i, j] = h
        num = dloss @ (orc.linear_ce(x + d, w, t)[0] - orc.linear_ce(x - d, w, t)[0]) / (2 * h)
        assert abs(num - dx[i, j]) <= 1e-7
    for i, j in ((0, 0), (4, 1), (10, 4)):
        d = np.zeros_like(w)
        d[i, j] = h
        num = dloss @ (orc.linear_ce(x, w + d, t)[0] - orc.linear_ce(x, w - d, t)[0]) / (2 * h)
        assert abs(num - dw[i, j]) <= 1e-7
