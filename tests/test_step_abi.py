"""Refusals of the table's and the gradients' calls, before anything touches a GPU, and the mirrors of their descriptors."""
import ctypes
import os
import re

import pytest

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "acc.h")
acc = pytest.importorskip("paper_2605_01255_amd.binding", reason="libacc.so not built")
FINE = (0, -6)   # passed validation (without a GPU the device check refuses)
CTYPE = {"int64_t": ctypes.c_int64, "int32_t": ctypes.c_int32, "uint32_t": ctypes.c_uint32, "float": ctypes.c_float, "void*": ctypes.c_void_p}


@pytest.mark.parametrize("name,mirror,size", [("acc_embed_desc", acc.AccEmbedDesc, 64), ("acc_grad_tensor", acc.AccGradTensor, 32),
                                              ("acc_grad_factors", acc.AccGradFactors, 64)])
def test_descriptors_match_the_header(name, mirror, size):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), text, flags=re.S).group(1)
    fields = []
    for line in body.split(";"):
        m = re.match(r"\s*(?:const )?(int64_t|int32_t|uint32_t|float|void\*)\s+(.*)", line, flags=re.S)
        if m:
            fields += [(n.strip(), CTYPE[m.group(1)]) for n in m.group(2).split(",")]
    assert fields == list(mirror._fields_) and ctypes.sizeof(mirror) == size


def _efwd(desc, W=0x1000, ids=0x2000, Y=0x3000):
    return acc._lib.acc_embed_fwd(ctypes.byref(desc) if desc else None, W, ids, Y, None)


def _ebwd(desc, ids=0x2000, dY=0x3000, dW=0x4000, ws=0x5000, size=1 << 40):
    return acc._lib.acc_embed_bwd(ctypes.byref(desc) if desc else None, ids, dY, dW, ws, size, None)


EMBED = dict(n=100, d=64, v=1000)


@pytest.mark.parametrize("bad,status", [
    (dict(n=0), -2), (dict(n=(1 << 30) + 1), -2), (dict(d=0), -2), (dict(d=12), -2), (dict(d=(1 << 16) + 8), -2), (dict(v=0), -2), (dict(v=(1 << 21) + 1), -2),
    (dict(ldw=56), -2), (dict(ldw=68), -2), (dict(ldy=56), -2), (dict(ldy=(1 << 18) + 8), -2), (dict(n=1 << 30, d=1 << 16), -2), (dict(io_dtype=2), -4),
    (dict(dw_dtype=3), -4), (dict(flags=1), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1)], ids=str)
def test_embed_descriptors_are_refused(bad, status):
    d = acc.make_embed_desc(**{**EMBED, **bad})
    assert _efwd(d) == status and _ebwd(d) == status and acc.acc_embed_workspace_bytes(d) == 0


def test_embed_pointers_and_workspaces_are_refused():
    d = acc.make_embed_desc(**EMBED)
    assert _efwd(None) == -1 and _ebwd(None) == -1 and _efwd(d) in FINE and _ebwd(d) in FINE
    for name in ("W", "ids", "Y"):
        assert _efwd(d, **{name: None}) == -1 and _efwd(d, **{name: 0x9008}) == -3, name
    for name in ("ids", "dY", "dW"):
        assert _ebwd(d, **{name: None}) == -1 and _ebwd(d, **{name: 0x9008}) == -3, name
    b = acc.acc_embed_workspace_bytes(d)
    assert b > 0 and _ebwd(d, size=b) in FINE and _ebwd(d, size=b - 1) == -5 and _ebwd(d, ws=None) == -5 and _ebwd(d, ws=0x9008) == -3
    d.reserved = 1
    assert _efwd(d) == -1


def test_the_embedding_workspace_is_a_quarter_of_the_gradient():
    at = lambda n, d: acc.acc_embed_workspace_bytes(acc.make_embed_desc(n, d, 128000))  # noqa: E731
    assert at(16384, 4096) < 16384 * 4096 + (2 << 20)   # of 134 MB of gradients


def _tensor(src=0x1000, dst=0x1000, count=10, dtype=0, dst_dtype=0):
    return acc.AccGradTensor(src, dst, count, dtype, dst_dtype)


def _factors(left=0x1000, gr=0x2000, d_in=64, d_out=32, r=8, ldl=0, ldg=0, dtype=1, flags=4):
    return acc.AccGradFactors(left, gr, d_in, d_out, r, ldl, ldg, dtype, flags)


def _norm(tensors=(), factors=(), max_norm=1.0, out=0x8000, ws=0x9000, size=1 << 50):
    t, f = (acc.AccGradTensor * len(tensors))(*tensors), (acc.AccGradFactors * len(factors))(*factors)
    return acc._lib.acc_grad_norm(t, len(t), f, len(f), max_norm, out, ws, size, None)


def _scale(tensors, factor=0x8000):
    t = (acc.AccGradTensor * len(tensors))(*tensors)
    return acc._lib.acc_grad_scale(t, len(t), factor, None)


@pytest.mark.parametrize("bad,norm,scale", [
    (dict(src=None), -1, -1), (dict(dst=None), None, -1), (dict(count=-1), -2, -2), (dict(count=(1 << 39) + 1), -2, -2), (dict(dtype=2), -4, -4),
    (dict(dst_dtype=7), None, -4), (dict(src=0x1002, dst=0x2000), -3, -3), (dict(dst=0x1002), None, -3), (dict(dtype=1, src=0x1001, dst=0x2000), -3, -3),
    (dict(dtype=1), None, -1), (dict(src=0x1004, dst=0x1004), None, None), (dict(src=None, dst=None, count=0), None, None),
    (dict(dtype=1, src=0x1002, dst=0x2004), None, None)], ids=str)
def test_gradient_tables_are_refused(bad, norm, scale):
    """None: not refused.  The last but two: aligned to its elements is enough; empty tensors need no memory; bfloat16 into float."""
    t = [_tensor(), _tensor(**bad)]
    assert _norm(t) == norm if norm else _norm(t) in FINE
    assert _scale(t) == scale if scale else _scale(t) in FINE
    assert (acc.acc_grad_norm_workspace_bytes((acc.AccGradTensor * 2)(*t), (acc.AccGradFactors * 0)()) == 0) == bool(norm)


@pytest.mark.parametrize("bad,status", [
    (dict(left=None), -1), (dict(gr=None), -1), (dict(left=0x1008), -3), (dict(gr=0x2004), -3), (dict(d_in=0), -2), (dict(d_in=12), -2), (dict(d_out=20), -2),
    (dict(r=0), -2), (dict(r=12), -2), (dict(r=(1 << 13) + 8), -2), (dict(d_in=(1 << 21) + 8), -2), (dict(ldl=4), -2), (dict(ldl=12), -2), (dict(ldg=4), -2),
    (dict(ldg=24, flags=0), -2), (dict(ldg=(1 << 22) + 8), -2), (dict(dtype=2), -4), (dict(flags=8), -1)], ids=str)
def test_factor_tables_are_refused(bad, status):
    assert _norm(factors=[_factors(), _factors(**bad)]) == status


def test_norm_arguments_are_refused():
    t, f = [_tensor()], [_factors(), _factors(flags=0, ldg=40)]
    assert _norm(t, f) in FINE and _norm() in FINE and _norm(t, max_norm=float("inf")) in FINE and _norm(t, max_norm=0.0) in FINE
    assert _norm(t, max_norm=-1.0) == -1 and _norm(t, max_norm=float("nan")) == -1 and _norm(t, out=None) == -1
    assert _norm(t, out=0x8002) == -3 and _norm(t, ws=0x9008) == -3 and _norm(t, ws=None) == -5
    need = acc.acc_grad_norm_workspace_bytes((acc.AccGradTensor * 1)(*t), (acc.AccGradFactors * 2)(*f))
    assert need > 0 and _norm(t, f, size=need) in FINE and _norm(t, f, size=need - 1) == -5
    assert _scale(t, factor=None) == -1 and _scale(t, factor=0x8002) == -3 and _scale(t, factor=0x8004) in FINE and _scale([]) in FINE
    assert acc._lib.acc_grad_norm(None, 1, None, 0, 1.0, 0x8000, 0x9000, 1 << 50, None) == -1
    assert acc._lib.acc_grad_norm(None, -1, None, 0, 1.0, 0x8000, 0x9000, 1 << 50, None) == -1
    assert acc._lib.acc_grad_norm(None, 0, None, 1, 1.0, 0x8000, 0x9000, 1 << 50, None) == -1


def test_modules_refuse_before_the_gpu():
    import torch
    ag = pytest.importorskip("paper_2605_01255_amd.autograd")
    for kw in (dict(heads=3, kv_heads=2), dict(heads=0), dict(heads=2, window=-1), dict(heads=2, window=3, causal=False), dict(heads=2, cap=-1.0),
               dict(heads=2, scale=0.0)):
        with pytest.raises(ValueError):
            ag.DocumentAttention(**kw)
    x = torch.zeros(2, 5, 4 * 16)
    att = ag.DocumentAttention(2, 1)
    with pytest.raises(ValueError):
        att(x)                                            # not on a GPU
    with pytest.raises(ValueError):
        att(torch.zeros(2, 5, 63))
    with pytest.raises(TypeError):
        att(x.half())
    with pytest.raises(ValueError):
        ag.DocumentAttention(2, 1, causal=False)(x, prefix=torch.tensor([1, 1]))
    with pytest.raises(ValueError):
        ag.DocumentAttention(2, 1, window=3)(x, prefix=torch.tensor([1, 1]))
    table = ag.Embedding(10, 16, dtype=torch.float32)
    with pytest.raises(ValueError):
        table(torch.zeros(3, dtype=torch.int64))
    with pytest.raises(TypeError):
        table(torch.zeros(3))
    p = torch.nn.Parameter(torch.zeros(4))
    assert float(ag.clip_grad_norm_([p], 1.0)) == 0.0     # no gradients
    p.grad = torch.ones(4)
    with pytest.raises(ValueError):
        ag.clip_grad_norm_(p, 1.0)
    q = torch.nn.Parameter(torch.zeros(2, 2))
    q.grad = p.grad.view(2, 2)                            # one gradient of two parameters
    with pytest.raises(ValueError, match="share one gradient"):
        ag.clip_grad_norm_([p, q], 1.0)
    p = torch.nn.Parameter(torch.zeros(4, dtype=torch.float64))
    p.grad = torch.ones(4, dtype=torch.float64)
    with pytest.raises(TypeError):
        ag.clip_grad_norm_([p], 1.0)
    with pytest.raises(ValueError):
        acc.make_grad_list([torch.zeros(4, 4).t()])
    with pytest.raises(ValueError):
        acc.make_grad_list([torch.zeros(4)], [torch.zeros(5)])
    with pytest.raises(ValueError):
        acc.make_factor_list([torch.zeros(8, 8)], [torch.zeros(8, 16)], acc.ACC_FLAG_W_OUT_IN)
