"""The slopes of DocumentAttention are float32 numbers whatever type the module is cast to."""
import copy

import pytest

torch = pytest.importorskip("torch")
ag = pytest.importorskip("paper_2605_01255_amd.autograd", reason="libacc.so not built")

SLOPES = [2.0 ** (-8.0 * (h + 1) / 12) for h in range(12)]   # not numbers of bfloat16


@pytest.mark.parametrize("cast", [lambda m: m.to(torch.bfloat16), lambda m: m.bfloat16(), lambda m: m.half(), lambda m: m.double(),
                                  lambda m: torch.nn.Sequential(torch.nn.Linear(2, 2), m).to(torch.bfloat16)[1],
                                  lambda m: m.to("cpu", torch.bfloat16), lambda m: copy.deepcopy(m).bfloat16().float()],
                         ids=["to", "bfloat16", "half", "double", "inside", "with a device", "and back"])
@pytest.mark.parametrize("slopes", [True, SLOPES], ids=["usual", "given"])
def test_slopes_stay_as_they_are(cast, slopes):
    att = ag.DocumentAttention(12, slopes=slopes)
    start = att.slopes.clone()
    assert start.dtype == torch.float32
    att = cast(att)
    assert att.slopes.dtype == torch.float32 and torch.equal(att.slopes, start)
    assert att.state_dict()["slopes"].dtype == torch.float32 and "slopes" in dict(att.named_buffers())


def test_slopes_move_with_the_module():
    att = ag.DocumentAttention(12, slopes=True).to("meta", torch.bfloat16)
    assert att.slopes.device.type == "meta" and att.slopes.dtype == torch.float32
    assert ag.DocumentAttention(12).bfloat16().slopes is None
