"""Every form of the cross entropy's bfloat16 products, each at a size for which the library chooses it (asserted through plan_util): the
tiles of the logits, the input gradient's parts, the weight gradient's tiles and parts, some of which lie behind the last token with a
loss.  Tolerances: test_gpu_ce.py."""
import pytest

pytestmark = pytest.mark.gpu

import plan_util as pu
from test_gpu_ce import Case, acc  # noqa: F401  (acc: the fixture)


def _weight_gradient(n, d, v, float_or_sum):
    return pu.token_product(v, d, max(n, 64 if n <= 128 else 192), float_or_sum)


@pytest.mark.parametrize("n,d,v,tile", [(40, 64, 515, "64x128"), (1000, 136, 2049, "128x128"), (1000, 64, 4099, "192x128"), (3000, 136, 4099, "256x256")])
def test_a_tile_of_the_logits(acc, n, d, v, tile):  # noqa: F811
    assert pu.ce_tile(n, v, d) == tile
    Case(acc, n, d, v, "bf16", ignored=0.3).check()


@pytest.mark.parametrize("n,d,v,tile,parts", [
    (77, 64, 300, "64x64", False), (1, 64, 2049, "64x64", True), (1000, 1032, 1003, "128x64", False), (1000, 136, 8191, "128x64", True),
    (3000, 1032, 300, "128x128", False), (700, 1024, 8191, "128x128", True), (2049, 2048, 77, "192x128", False),
    (129, 2048, 20011, "192x128", True), (8200, 2048, 10007, "256x256", False), (3000, 1024, 20011, "256x256", True)])
def test_a_form_of_the_input_gradient(acc, n, d, v, tile, parts):  # noqa: F811
    plan = pu.ce_input_gradient(n, d, v)
    assert (plan.tile, plan.parts > 1) == (tile, parts), plan
    Case(acc, n, d, v, "bf16", ignored=0.1 if n > 1 else 0.0).check()


@pytest.mark.parametrize("dw,add", [("bf16", False), ("bf16", True), ("f32", False), ("f32", True)])
@pytest.mark.parametrize("ignored", [0.0, 0.9])
@pytest.mark.parametrize("n,d,v,tile", [(1500, 64, 77, "64x64"), (8200, 136, 2049, "128x64"), (8200, 1024, 2049, "128x128")])
def test_a_weight_gradient_in_parts(acc, n, d, v, tile, ignored, dw, add):  # noqa: F811
    """With nine tokens in ten left out most parts hold none that takes part."""
    plan = _weight_gradient(n, d, v, add or dw == "f32")
    assert plan.tile == tile and plan.parts > 1, plan
    Case(acc, n, d, v, "bf16", dw=dw, add=add, ignored=ignored).check()


@pytest.mark.parametrize("dw,add", [("bf16", False), ("bf16", True), ("f32", False)])
@pytest.mark.parametrize("n,d,v,tile", [
    (1, 1032, 1003, "64x64"), (257, 1032, 1003, "128x64"), (1, 264, 10007, "128x64"), (1, 264, 20011, "128x128"), (3000, 2048, 2049, "192x128"),
    (129, 520, 20011, "256x256")])
def test_a_weight_gradient_in_one_part(acc, n, d, v, tile, dw, add):  # noqa: F811
    plan = _weight_gradient(n, d, v, add or dw == "f32")
    assert plan.parts == 1 and (plan.tile == tile or (tile == "256x256" and (add or dw == "f32"))), plan
    Case(acc, n, d, v, "bf16", dw=dw, add=add, ignored=0.2 if n > 1 else 0.0).check()
