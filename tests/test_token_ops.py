"""CPU checks of the token operators' C entry points: descriptors, sizes and refusals, without a launch."""
import ctypes as C
import os
import re

import pytest
import torch

import paper_1805_08691_b200 as q8

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, ARG, UNSUPPORTED, ALIGN, WORKSPACE = 0, 1, 2, 3, 4
F32, F16, BF16, S8, U8, S32 = q8.Q8_F32, q8.Q8_F16, q8.Q8_BF16, q8.Q8_S8, q8.Q8_U8, q8.Q8_S32
P = 4096  # stands for a device address: refused calls never look at it


@pytest.mark.parametrize("name", ["q8_linear_desc", "q8_moe_desc"])
def test_struct_layout_matches_header(name):
    text = open(os.path.join(ROOT, "include", "q8.h")).read()
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), text, flags=re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    fields = []
    for decl in body.split(";"):
        m = re.match(r"\s*(int64_t|int32_t)\s+(.*)", decl.strip(), flags=re.S)
        if m:
            fields += [(f.strip(), 8 if m.group(1) == "int64_t" else 4) for f in m.group(2).split(",")]
    cls = getattr(q8, name)
    assert fields == [(f[0], C.sizeof(f[1])) for f in cls._fields_]
    assert C.sizeof(cls) == sum(n for _, n in fields)
    assert (q8.Q8_F16, q8.Q8_BF16) == (4, 5)


@pytest.mark.parametrize("args,code", [
    ((None, F32, 2, 8, 8, P, 8, P, None), ARG), ((P, F32, 2, 8, 8, None, 8, P, None), ARG), ((P, F32, 2, 8, 8, P, 8, None, None), ARG),
    ((P, F32, 2, 0, 8, P, 8, P, None), ARG), ((P, F32, 2, 8, 7, P, 8, P, None), ARG), ((P, F32, 2, 8, 8, P, 7, P, None), ARG),
    ((P, S8, 2, 8, 8, P, 8, P, None), ARG), ((P, S32, 2, 8, 8, P, 8, P, None), ARG), ((P, 9, 2, 8, 8, P, 8, P, None), ARG),
    ((P + 2, F32, 2, 8, 8, P, 8, P, None), ALIGN), ((P + 1, BF16, 2, 8, 8, P, 8, P, None), ALIGN), ((P, F16, 2, 8, 8, P, 8, P + 2, None), ALIGN),
    ((P, F32, 1 << 60, 8, 8, P, 8, P, None), ARG),
    ((None, F32, 0, 8, 8, None, 8, None, None), OK),
])
def test_quantize_and_dequantize_refusals(args, code):
    assert q8.lib.q8_quantize_tokens(*args) == code
    x, t, n, c, ldx, z, ldz, s, st = args
    assert q8.lib.q8_dequantize_tokens(z, n, c, ldz, s, x, t, ldx, st) == code


def _linear(**k):
    d = q8.q8_linear_desc(0, 0, 0, 4, 64, 32, S8, BF16, 0)
    for n, v in k.items():
        setattr(d, n, v)
    return d


def _run_linear(d, x=P, xs=P, w=P, ws=P, b=None, y=P, work=None, n=0):
    return q8.lib.q8_linear(C.byref(d), x, xs, w, ws, b, y, work, n, None)


def test_linear_refusals():
    for bad in (dict(M=-1), dict(C=0), dict(K=0), dict(C=131072), dict(x_type=U8), dict(x_type=S32), dict(x_type=6), dict(y_type=S8),
                dict(y_type=S32), dict(y_type=-1), dict(ldx=63), dict(ldw=63), dict(ldy=31), dict(ldx=-64), dict(ldw=1 << 62), dict(reserved=1)):
        d = _linear(**bad)
        assert _run_linear(d) == ARG, bad
        assert q8.lib.q8_linear_workspace_bytes(C.byref(d), C.byref(C.c_size_t())) == ARG, bad
    d = _linear()
    assert q8.lib.q8_linear(None, P, P, P, P, None, P, None, 0, None) == ARG
    assert q8.lib.q8_linear_workspace_bytes(None, C.byref(C.c_size_t())) == ARG
    assert q8.lib.q8_linear_workspace_bytes(C.byref(d), None) == ARG
    for missing in ("x", "xs", "w", "ws", "y"):
        assert _run_linear(d, **{missing: None}) == ARG, missing
    f = _linear(x_type=F32)
    assert _run_linear(f) == ARG                     # factors belong to codes
    assert _run_linear(f, x=P + 2, xs=None) == ALIGN
    assert _run_linear(d, y=P + 1) == ALIGN and _run_linear(d, xs=P + 2) == ALIGN and _run_linear(d, ws=P + 1) == ALIGN
    assert _run_linear(d, b=P + 2) == ALIGN and _run_linear(d, work=P + 8, n=1 << 20) == ALIGN
    assert _run_linear(_linear(M=0), x=None, xs=None, y=None) == OK
    assert _run_linear(_linear(M=0, x_type=F16), x=None, xs=None, y=None) == OK
    assert _run_linear(_linear(M=0), w=None) == ARG


def _moe(**k):
    d = q8.q8_moe_desc(0, 0, 4, 64, 32, 8, 2, BF16, 1, 0)
    for n, v in k.items():
        setattr(d, n, v)
    return d


def _run_moe(d, x=P, r=P, wgu=P, sgu=P, wd=P, sd=P, y=P, ids=None, probs=None, work=P, n=1 << 40):
    return q8.lib.q8_moe(C.byref(d), x, r, wgu, sgu, wd, sd, y, ids, probs, work, n, None)


def test_moe_refusals():
    for bad in (dict(T=-1), dict(C=0), dict(I=0), dict(E=0), dict(top_k=0), dict(top_k=9), dict(x_type=S8), dict(x_type=S32), dict(renormalize=2),
                dict(reserved=1), dict(ldx=63), dict(ldy=63), dict(ldx=-1), dict(ldy=1 << 62)):
        d = _moe(**bad)
        assert _run_moe(d) == ARG, bad
        assert q8.lib.q8_moe_workspace_bytes(C.byref(d), C.byref(C.c_size_t())) == ARG, bad
    for bad in (dict(C=131072), dict(I=131072), dict(E=1025), dict(E=64, top_k=33)):
        d = _moe(**bad)
        assert _run_moe(d) == UNSUPPORTED, bad
        assert q8.lib.q8_moe_workspace_bytes(C.byref(d), C.byref(C.c_size_t())) == UNSUPPORTED, bad
    d = _moe()
    for missing in ("x", "r", "wgu", "sgu", "wd", "sd", "y"):
        assert _run_moe(d, **{missing: None}) == ARG, missing
    assert q8.lib.q8_moe(None, *[P] * 10, 1 << 40, None) == ARG
    for odd in (dict(x=P + 1), dict(y=P + 1), dict(r=P + 2), dict(sgu=P + 2), dict(sd=P + 2), dict(ids=P + 2), dict(probs=P + 1), dict(work=P + 128)):
        assert _run_moe(d, **odd) == ALIGN, odd
    need = q8.q8_moe_workspace_bytes(d)
    assert need > 0 and need % 256 == 0
    assert _run_moe(d, n=need - 1) == WORKSPACE and _run_moe(d, work=None) == WORKSPACE
    assert q8.q8_moe_workspace_bytes(_moe(T=0)) == 0
    assert _run_moe(_moe(T=0), x=None, y=None, work=None, n=0) == OK
    # tokens go in groups: the scratch does not grow with their number
    assert q8.q8_moe_workspace_bytes(_moe(T=16)) == q8.q8_moe_workspace_bytes(_moe(T=100000))


def test_binding_refuses_other_tensors():
    x, w, s = torch.zeros(2, 8), torch.zeros(4, 8, dtype=torch.int8), torch.zeros(4)
    for call in (lambda: q8.q8_quantize_tokens(x), lambda: q8.q8_dequantize_tokens(w, s), lambda: q8.q8_linear(x, w, s),
                 lambda: q8.q8_moe(x, x, w, s, w, s, 2)):
        with pytest.raises(TypeError):
            call()
