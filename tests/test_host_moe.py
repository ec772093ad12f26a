"""include/tuna_moe.h without a GPU: what it declares is there, the sizes of workspaces, and what is refused before anything is enqueued."""
import ctypes
import os
import re

import pytest
import torch

import moe_plain as plain
import paper_2411_02581_amd as tuna

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x7000000000                                                 # an address that is never used: every call here is refused or empty
ARG, LARGE, SMALL, OK = tuna.TUNA_ERR_ARG, tuna.TUNA_ERR_TOO_LARGE, tuna.TUNA_ERR_WORKSPACE_TOO_SMALL, tuna.TUNA_OK


def test_library_exports_every_declared_symbol():
    header = open(os.path.join(ROOT, "include", "tuna_moe.h")).read()
    declared = set(re.findall(r"^int\s+(tuna_\w+)\s*\(", header, flags=re.M))
    assert declared == set(tuna.MOE_EXPORTS)
    lib = ctypes.CDLL(tuna.library_path())
    for name in declared:
        assert hasattr(lib, name) and callable(getattr(tuna, name)), name


def test_header_constants_match_the_binding():
    header = open(os.path.join(ROOT, "include", "tuna_moe.h")).read()
    for name, value in re.findall(r"^#define (TUNA_\w+) (-?\d+)", header, flags=re.M):
        assert getattr(tuna, name) == int(value), name


def refused(call, code, **changes):
    """`call` with its arguments by name, some changed, on a stream of its own name."""
    name, args = call
    args = dict(args, **changes)
    assert getattr(tuna, name)(*args.values(), stream=0) == code, (name, changes)


def test_route_refusals():
    c = ("tuna_moe_route", dict(logits=A, type=0, ld=8, n=4, e=8, k=2, flags=0, experts=A, weights=A, slots=A, rows=A, row_bytes=16, sc=A, sd=A, rc=A, rd=A,
                                ws=A, size=1 << 20))
    for ch in (dict(logits=None), dict(logits=A + 2), dict(type=2), dict(type=7), dict(ld=7), dict(n=-1), dict(e=0), dict(e=1025, ld=1025), dict(k=0), dict(k=9),
               dict(k=17, e=32, ld=32), dict(flags=2), dict(experts=None), dict(weights=None), dict(slots=A + 1), dict(rows=None), dict(row_bytes=0),
               dict(sc=None), dict(rd=None), dict(sd=A + 4), dict(ws=None), dict(ws=A + 8)):
        refused(c, ARG, **ch)
    refused(c, LARGE, n=1 << 30)
    refused(c, LARGE, row_bytes=1 << 31)
    refused(c, LARGE, n=8000, row_bytes=1 << 22)
    refused(c, SMALL, size=16)
    g = ("tuna_moe_route_grad", dict(logits=A, type=1, ld=8, n=4, e=8, k=2, flags=1, experts=A, weights=A, dw=A, dl=A, ldd=8))
    for ch in (dict(logits=None), dict(logits=A + 1), dict(dl=None), dict(ldd=7), dict(ld=7), dict(k=9), dict(dw=None), dict(flags=4), dict(n=-1)):
        refused(g, ARG, **ch)
    refused(g, OK, n=0)


def test_quantise_refusals():
    c = ("tuna_fp8_quantize", dict(x=A, type=1, ldx=256, rows=4, cols=256, act=0, slots=None, copies=1, out=4, q=A, ldq=256, s=A, lds=2, kind=0))
    for ch in (dict(x=None), dict(x=A + 1), dict(type=2), dict(ldx=255), dict(rows=-1), dict(cols=-1), dict(act=2), dict(act=1), dict(copies=0), dict(copies=2),
               dict(out=3), dict(slots=A + 2), dict(slots=A, copies=17), dict(q=None), dict(ldq=255), dict(s=A + 2), dict(lds=1), dict(kind=2)):
        refused(c, ARG, **ch)
    refused(c, LARGE, rows=1 << 31, out=1 << 31)
    refused(c, OK, rows=0)
    refused(c, OK, cols=0)
    t = ("tuna_fp8_quantize_columns", dict(x=A, type=0, ldx=100, rows=300, cols=100, g=A, groups=3, q=A, ldq=640, s=A, lds=5, kind=1))
    for ch in (dict(x=None), dict(ldx=99), dict(groups=0), dict(groups=1025), dict(g=None), dict(g=A + 2), dict(ldq=639), dict(lds=4), dict(kind=-1), dict(type=3)):
        refused(t, ARG, **ch)
    refused(t, LARGE, cols=1 << 30, ldx=1 << 30)
    d = ("tuna_moe_swiglu_grad", dict(x=A, type=1, ldx=20, dh=A, ldh=10, rows=3, cols=10, dx=A, ldd=20))
    for ch in (dict(x=None), dict(ldx=19), dict(ldh=9), dict(ldd=19), dict(dx=A + 1), dict(rows=-1), dict(type=2)):
        refused(d, ARG, **ch)


def test_product_refusals():
    c = ("tuna_fp8_matmul", dict(x=A, ldx=256, xs=A, lxs=2, w=A, ldw=256, wg=100 * 256, ws=A, lws=2, wsg=2, kind=0, g=A, groups=4, y=A, yt=1, ldy=100, m=10, n=100,
                                 k=256))
    for ch in (dict(x=None), dict(ldx=255), dict(xs=A + 1), dict(lxs=1), dict(w=None), dict(ldw=255), dict(ws=None), dict(lws=1), dict(kind=2), dict(g=None),
               dict(groups=0), dict(groups=2000), dict(g=A + 1), dict(y=None), dict(yt=2), dict(ldy=99), dict(m=-1), dict(n=-1), dict(k=-1), dict(wg=-1),
               dict(y=A + 1)):
        refused(c, ARG, **ch)
    refused(c, LARGE, m=1 << 31)
    refused(c, LARGE, n=1 << 30, ldy=1 << 30)
    refused(c, OK, m=0)
    refused(c, OK, n=0)
    w = ("tuna_fp8_matmul_grad_w", dict(a=A, la=640, sa=A, lsa=5, b=A, lb=640, sb=A, lsb=5, kind=0, g=A, groups=3, dw=A, dt=0, ld=50, dg=2000, m=300, n=40, k=50))
    for ch in (dict(a=None), dict(la=639), dict(lsa=4), dict(b=None), dict(lb=639), dict(lsb=4), dict(dw=None), dict(dw=A + 2), dict(dt=2), dict(ld=49), dict(dg=1999),
               dict(kind=3), dict(g=None), dict(groups=0), dict(m=-1)):
        refused(w, ARG, **ch)


def test_combine_refusals():
    c = ("tuna_moe_combine", dict(y=A, yt=1, ldy=64, rows=8, slots=A, w=A, n=4, k=2, cols=64, out=A, ot=0, ldo=64))
    for ch in (dict(y=None), dict(yt=2), dict(ldy=63), dict(rows=-1), dict(slots=None), dict(w=A + 1), dict(k=0), dict(k=17), dict(cols=-1), dict(out=A + 2),
               dict(ldo=63), dict(ot=-1), dict(n=-1)):
        refused(c, ARG, **ch)
    refused(c, LARGE, n=1 << 31)
    refused(c, OK, n=0)
    g = ("tuna_moe_combine_grad", dict(d=A, ot=1, ldd=64, y=A, yt=1, ldy=64, rows=8, slots=A, w=A, n=4, k=2, cols=64, dy=A, lddy=64, dw=A))
    for ch in (dict(d=None), dict(ldd=63), dict(y=None), dict(dy=None), dict(lddy=63), dict(dw=None), dict(k=17), dict(rows=-1)):
        refused(g, ARG, **ch)


def test_few_refusals():
    rc, size = tuna.tuna_moe_few_workspace(4, 64, 48, 8, 2)
    assert rc == OK and size > 0
    c = ("tuna_moe_few", dict(x=A, ldx=64, n=4, h=64, l=A, lt=0, ldl=8, e=8, k=2, flags=1, w1=A, s1=A, w2=A, s2=A, f=48, wt=2, kind=0, out=A, ot=1, ldo=64, ws=A, size=size))
    for ch in (dict(x=None), dict(ldx=63), dict(n=65), dict(n=-1), dict(h=-1), dict(l=None), dict(ldl=7), dict(lt=2), dict(e=0), dict(k=9), dict(flags=2), dict(w1=None),
               dict(s1=None), dict(s2=A + 2), dict(wt=0), dict(wt=1), dict(kind=2), dict(f=0), dict(out=None), dict(ldo=63), dict(ot=2), dict(ws=None), dict(ws=A + 4)):
        refused(c, ARG, **ch)
    refused(c, SMALL, size=size - 1)
    refused(c, OK, n=0)
    assert tuna.tuna_moe_few_workspace(65, 64, 48, 8, 2)[0] == ARG
    assert tuna.tuna_moe_route_workspace(1 << 30, 8, 4, True)[0] == LARGE


def test_binding_refuses_tensors_that_do_not_fit():
    with pytest.raises(TypeError):
        tuna.tuna_moe_route(torch.zeros(4, 8), 0, 8, 4, 8, 2, 0, A, A, A, A, 1, None, None, None, None, A, 1 << 20, stream=0)


# ------------------------------------------------------------------------------------------------ the definitions the GPU tests compare with


def test_plain_e4m3_is_the_types():
    codes = torch.arange(256, dtype=torch.uint8)
    v = plain.from_e4m3(codes)
    t = codes.view(torch.float8_e4m3fn).double()
    assert torch.equal(v.isnan(), t.isnan()) and torch.equal(v[~v.isnan()], t[~t.isnan()])
    x = torch.randn(4000, generator=torch.Generator().manual_seed(0)).double() * 100
    x = torch.cat([x.clamp(-460, 460), v[~v.isnan()], (v[1:126] + v[2:127]) / 2])
    assert torch.equal(plain.to_e4m3(x), x.float().to(torch.float8_e4m3fn).view(torch.uint8))


@pytest.mark.parametrize("renorm", [False, True])
def test_plain_route_gradient_is_the_derivative(renorm):
    x = torch.randn(5, 9, generator=torch.Generator().manual_seed(1)).double().requires_grad_()
    d = torch.randn(5, 3, generator=torch.Generator().manual_seed(2)).double()
    p, experts, weights = plain.route(x.detach(), 3, renorm)
    s = torch.softmax(x, 1)
    w = s.gather(1, experts)
    w = w / w.sum(1, keepdim=True) if renorm else w
    assert torch.allclose(w.detach(), weights)
    (w * d).sum().backward()
    assert torch.allclose(x.grad, plain.route_grad(p, experts, weights, d, renorm))


def test_plain_swiglu_gradient_is_the_derivative():
    x = torch.randn(3, 10, generator=torch.Generator().manual_seed(3)).double().requires_grad_()
    d = torch.randn(3, 5, generator=torch.Generator().manual_seed(4)).double()
    (plain.swiglu(x) * d).sum().backward()
    assert torch.allclose(x.grad, plain.swiglu_grad(x.detach(), d))
