"""Refusals of the cross entropy's calls, before anything touches a GPU, and the mirror of their descriptor."""
import ctypes
import os
import re

import pytest

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "acc.h")
acc = pytest.importorskip("paper_2605_01255_amd.binding", reason="libacc.so not built")
FINE = (0, -6)   # passed validation (without a GPU the device check refuses)
OK = dict(n=100, d=64, v=1001)


def test_descriptor_matches_the_header():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    body = re.search(r"typedef struct acc_ce_desc \{(.*?)\} acc_ce_desc;", text, flags=re.S).group(1)
    ctype = {"int64_t": ctypes.c_int64, "int32_t": ctypes.c_int32, "uint32_t": ctypes.c_uint32}
    fields = [(n, ctype[t]) for t, n in re.findall(r"\b(int64_t|int32_t|uint32_t)\s+(\w+)\s*;", body)]
    assert fields == list(acc.AccCeDesc._fields_) and ctypes.sizeof(acc.AccCeDesc) == 64


def _fwd(desc, X=0x1000, W=0x2000, targets=0x3000, loss=0x4000, stats=0x5000, ws=0x6000, size=1 << 40):
    return acc._lib.acc_linear_ce_fwd(ctypes.byref(desc) if desc else None, X, W, targets, loss, stats, ws, size, None)


def _bwd(desc, X=0x1000, W=0x2000, targets=0x3000, stats=0x4000, dloss=0x5000, dX=0x6000, dW=0x7000, ws=0x8000, size=1 << 40):
    return acc._lib.acc_linear_ce_bwd(ctypes.byref(desc) if desc else None, X, W, targets, stats, dloss, dX, dW, ws, size, None)


@pytest.mark.parametrize("bad,status", [
    (dict(n=0), -2), (dict(n=-3), -2), (dict(n=(1 << 30) + 1), -2), (dict(d=0), -2), (dict(d=60), -2), (dict(d=(1 << 16) + 8), -2),
    (dict(v=0), -2), (dict(v=(1 << 21) + 1), -2), (dict(ldx=56), -2), (dict(ldx=68), -2), (dict(ldw=56), -2), (dict(ldw=(1 << 18) + 8), -2),
    (dict(piece=-256), -2), (dict(piece=100), -2), (dict(io_dtype=2), -4), (dict(dw_dtype=-1), -4), (dict(flags=1), -1), (dict(flags=4), -1)], ids=str)
def test_descriptors_are_refused(bad, status):
    d = acc.make_ce_desc(**{**OK, **bad})
    assert _fwd(d) == status and _bwd(d) == status
    assert acc.acc_linear_ce_workspace_bytes(d, False) == acc.acc_linear_ce_workspace_bytes(d, True) == 0


def test_pointers_and_workspaces_are_refused():
    d = acc.make_ce_desc(**OK)
    assert _fwd(None) == -1 and _bwd(None) == -1 and _fwd(d) in FINE and _bwd(d) in FINE
    for name in ("X", "W", "targets", "loss", "stats"):
        assert _fwd(d, **{name: None}) == -1 and _fwd(d, **{name: 0x9008}) == -3, name
    for name in ("X", "W", "targets", "stats", "dloss"):
        assert _bwd(d, **{name: None}) == -1 and _bwd(d, **{name: 0x9008}) == -3, name
    assert _bwd(d, dX=None) in FINE and _bwd(d, dW=None) in FINE and _bwd(d, dX=None, dW=None) == -1
    assert _bwd(d, dX=0x9008) == -3 and _bwd(d, dW=0x9008) == -3 and _fwd(d, ws=0x9008) == -3
    f, b = acc.acc_linear_ce_workspace_bytes(d, False), acc.acc_linear_ce_workspace_bytes(d, True)
    assert 0 < f <= b
    assert _fwd(d, size=f) in FINE and _fwd(d, size=f - 1) == -5 and _fwd(d, ws=None) == -5
    assert _bwd(d, size=b) in FINE and _bwd(d, size=b - 1) == -5 and _bwd(d, ws=None) == -5


def test_the_workspace_does_not_grow_to_the_logits():
    # 65536 tokens over 128000 words: 33 GB of float logits; 2^20 tokens take the workspace of a run of them
    at = lambda n, **kw: acc.acc_linear_ce_workspace_bytes(acc.make_ce_desc(n, 4096, 128000, **kw), True)  # noqa: E731
    assert at(65536) < 6 << 30
    assert at(1 << 20) == at(1 << 19)
    assert at(8192, piece=1024) < at(8192)
    assert acc.acc_linear_ce_workspace_bytes(acc.make_ce_desc(1 << 18, 64, 1 << 21), False) < 8 << 30   # of 2^39 logits
