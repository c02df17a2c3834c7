"""Refusals of the attention calls, before anything touches a GPU, the mirror of their descriptor, and the oracle of their tests."""
import ctypes
import os
import re

import pytest

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "acc.h")
acc = pytest.importorskip("paper_2605_01255_amd.binding", reason="libacc.so not built")
FINE = (0, -6)   # passed validation (without a GPU the device check refuses)
OK = dict(n=100, heads=8, kv_heads=2, d=64)


def test_descriptor_matches_the_header():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    body = re.search(r"typedef struct acc_attn_desc \{(.*?)\} acc_attn_desc;", text, flags=re.S).group(1)
    ctype = {"int64_t": ctypes.c_int64, "int32_t": ctypes.c_int32, "uint32_t": ctypes.c_uint32, "float": ctypes.c_float}
    fields = [(n, ctype[t]) for t, n in re.findall(r"\b(int64_t|int32_t|uint32_t|float)\s+(\w+)\s*;", body)]
    assert fields == list(acc.AccAttnDesc._fields_) and ctypes.sizeof(acc.AccAttnDesc) == 104


PTRS = dict(Q=0x1000, K=0x2000, V=0x3000, starts=None, prefix=None, slopes=None)


def _fwd(desc, O=0x4000, lse=0x5000, ws=0x6000, size=1 << 40, **kw):
    p = {**PTRS, **kw}
    return acc._lib.acc_attn_fwd(ctypes.byref(desc) if desc else None, *p.values(), O, lse, ws, size, None)


def _bwd(desc, O=0x4000, lse=0x5000, dO=0x7000, dQ=0x8000, dK=0x9000, dV=0xA000, ws=0x6000, size=1 << 40, **kw):
    p = {**PTRS, **kw}
    return acc._lib.acc_attn_bwd(ctypes.byref(desc) if desc else None, *p.values(), O, lse, dO, dQ, dK, dV, ws, size, None)


@pytest.mark.parametrize("bad,status", [
    (dict(n=0), -2), (dict(n=-1), -2), (dict(n=(1 << 30) + 1), -2), (dict(heads=0), -2), (dict(heads=7), -2), (dict(kv_heads=0), -2),
    (dict(heads=1 << 16, d=8), -2), (dict(d=0), -2), (dict(d=60), -2), (dict(d=136), -2), (dict(ldq=504), -2), (dict(ldq=516), -2), (dict(ldk=120), -2),
    (dict(ldv=120), -2), (dict(ldo=504), -2), (dict(ldo=(1 << 18) + 8), -2), (dict(docs=-1), -2), (dict(seq=-1), -2), (dict(window=-1), -1),
    (dict(window=5, flags=0), -1), (dict(scale=-1.0), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(cap=-2.0), -1),
    (dict(cap=float("nan")), -1), (dict(cap=float("inf")), -1), (dict(flags=2), -1), (dict(io_dtype=2), -4),
    (dict(n=1 << 30, seq=1), -2), (dict(n=1 << 30, heads=1, kv_heads=1), -2)], ids=str)   # the last two: more threads than a launch has
def test_descriptors_are_refused(bad, status):
    d = acc.make_attn_desc(**{**OK, **bad})
    assert _fwd(d) == status and _bwd(d) == status
    assert acc.acc_attn_workspace_bytes(d, True) == 0


def test_as_many_rows_as_a_launch_has_threads_for():
    d = acc.make_attn_desc(1 << 29, 1, 1, 8)
    assert _fwd(d) in FINE and _bwd(d) in FINE


def test_masks_that_do_not_go_together_are_refused():
    plain, docs = acc.make_attn_desc(**OK), acc.make_attn_desc(**OK, docs=3)
    for call in (_fwd, _bwd):
        assert call(None) == -1
        assert call(plain) in FINE and call(docs, starts=0x9000) in FINE
        assert call(plain, starts=0x9000) == -1 and call(docs) == -1
        assert call(acc.make_attn_desc(**OK, docs=3, seq=5), starts=0x9000) == -2
        assert call(plain, prefix=0x9000) in FINE and call(plain, slopes=0x9000) in FINE
        assert call(acc.make_attn_desc(**OK, flags=0), prefix=0x9000) == -1
        assert call(acc.make_attn_desc(**OK, window=4), prefix=0x9000) == -1
        assert call(docs, starts=0x9008) == call(plain, prefix=0x9008) == call(plain, slopes=0x9004) == -3


def test_pointers_and_workspaces_are_refused():
    d = acc.make_attn_desc(**OK)
    for name in ("Q", "K", "V", "O", "lse"):
        assert _fwd(d, **{name: None}) == -1 and _fwd(d, **{name: 0x9008}) == -3, name
    for name in ("Q", "K", "V", "O", "lse", "dO", "dQ", "dK", "dV"):
        assert _bwd(d, **{name: None}) == -1 and _bwd(d, **{name: 0x9008}) == -3, name
    f, b = acc.acc_attn_workspace_bytes(d, False), acc.acc_attn_workspace_bytes(d, True)
    assert f <= b and b > 0
    assert _fwd(d, size=f) in FINE and _bwd(d, size=b) in FINE and _bwd(d, size=b - 1) == -5 and _bwd(d, ws=None) == -5
    assert _fwd(d, ws=0x9008) == -3 and _bwd(d, ws=0x9008) == -3


def test_the_oracle_agrees_with_differentiation():
    """The test oracle's gradients are those that automatic differentiation of its forward formula gives."""
    import torch
    from attn_util import Case
    c = Case(40, 4, 2, 8, "f32", cuts=[2, 20, 38], cap=3.0, bias=True, prefix=[3, 5], size=1.5)
    want = c.exact()
    qkv = c.qkv.double().requires_grad_(True)
    q, k, v = (t.reshape(40, -1, 8).transpose(0, 1) for t in c.split(qkv))
    k, v = k.repeat_interleave(2, 0), v.repeat_interleave(2, 0)
    i = torch.arange(40)
    z = 3.0 * torch.tanh(q @ k.transpose(1, 2) / 8 ** 0.5 / 3.0) - c.slopes.double().view(-1, 1, 1) * (i[:, None] - i).abs()
    z = z.masked_fill(~c.seen(), -1e300)
    o = (torch.softmax(z, 2) * c.seen()) @ v
    o = o.transpose(0, 1).reshape(40, -1)
    assert float((o - want["o"][0]).abs().max()) < 1e-12
    (o * c.dO.double()).sum().backward()
    for got, name in zip(c.split(qkv.grad), ("dq", "dk", "dv")):
        assert float((got - want[name][0]).abs().max()) < 1e-11, name
