"""Tables of growing size one after another in a process of its own: each asks for more LDS than the one before."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

_PROGRAM = r"""
import torch
from paper_2605_01255_amd import binding as acc
for v in (140000, 200000, 262144, 131073):
    ids = torch.tensor([v - 1, 5, -1, v - 1, 70000], device="cuda")
    dy = torch.arange(40, device="cuda", dtype=torch.float32).reshape(5, 8)
    dw = torch.full((v, 8), 7.0, device="cuda")
    desc = acc.make_embed_desc(5, 8, v, io_dtype=acc.ACC_F32)
    ws = torch.empty(acc.acc_embed_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    acc.acc_embed_bwd(desc, ids, dy, dw, ws)
    want = torch.zeros(v, 8, device="cuda")
    want[v - 1], want[5], want[70000] = dy[0] + dy[3], dy[1], dy[4]
    assert torch.equal(dw, want), v
    print("words", v, flush=True)
"""


def test_tables_that_grow_in_one_process():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    res = subprocess.run([sys.executable, "-c", _PROGRAM], cwd=ROOT, capture_output=True, text=True, timeout=100)
    assert res.returncode == 0 and res.stdout.count("words") == 4, res.stdout + res.stderr
