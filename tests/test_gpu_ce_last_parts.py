"""The input gradient of the cross entropy where the last piece of the vocabulary ends inside a part of the persistent kernel: nothing
behind the vocabulary's matrix is read.  W is the front of a buffer whose other rows are NaN, so that a read of any of them shows in dX
(0 times NaN is NaN).  Tolerances: test_gpu_ce.py."""
import pytest

pytestmark = pytest.mark.gpu

import plan_util as pu
from test_gpu_ce import Case, acc  # noqa: F401  (acc: the fixture)

TOKENS, FEATURES, PIECE = 3000, 1024, 20480


# a last part of one K tile, two (three run), four; a whole part and one, sixteen K tiles behind it
@pytest.mark.parametrize("rest", [37, 100, 232, 4096 + 21, 4096 + 1001])
def test_short_last_part(acc, rest):  # noqa: F811
    import torch
    plan = pu.ce_input_gradient(TOKENS, FEATURES, PIECE)
    assert plan.tile == "256x256" and plan.k_per_part == 4096, plan
    c = Case(acc, TOKENS, FEATURES, PIECE + rest, "bf16", piece=PIECE, ignored=0.2)
    behind = torch.full((c.v + plan.k_per_part + 64, FEATURES), float("nan"), dtype=torch.bfloat16, device="cuda")
    behind[:c.v] = c.W
    c.W = behind[:c.v]
    c.check()
