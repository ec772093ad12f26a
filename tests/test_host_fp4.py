"""The 4-bit operators and the balance loss of include/tuna_moe.h without a GPU: what is refused before anything is enqueued, sizes of workspaces, the
definitions that the GPU tests compare with."""
import pytest
import torch

import fp4_plain as plain
import paper_2411_02581_amd as tuna
from test_host_moe import A, ARG, LARGE, OK, SMALL, refused

U8, F4 = torch.uint8, torch.float4_e2m1fn_x2


def test_quantise_refusals():
    c = ("tuna_fp4_quantize", dict(x=A, type=1, ldx=256, rows=4, cols=256, act=0, slots=None, copies=1, out=4, q=A, ldq=128, s=A, lds=8))
    for ch in (dict(x=None), dict(x=A + 1), dict(type=2), dict(type=4), dict(ldx=255), dict(rows=-1), dict(cols=-1), dict(act=2), dict(act=1), dict(copies=0),
               dict(copies=2), dict(out=3), dict(out=-1), dict(slots=A + 2), dict(slots=A, copies=17), dict(q=None), dict(ldq=127), dict(s=None), dict(lds=7),
               dict(cols=257, ldx=257, lds=9), dict(cols=257, ldx=257, ldq=129)):
        refused(c, ARG, **ch)
    refused(c, LARGE, rows=1 << 31, out=1 << 31)
    refused(c, LARGE, rows=1 << 28, out=1 << 28)
    for ch in (dict(rows=0), dict(cols=0), dict(slots=A, out=0, q=None, s=None)):
        refused(c, OK, **ch)
    t = ("tuna_fp4_quantize_columns", dict(x=A, type=0, ldx=100, rows=300, cols=100, g=A, groups=3, q=A, ldq=320, s=A, lds=20))
    for ch in (dict(x=None), dict(ldx=99), dict(groups=0), dict(groups=1025), dict(g=None), dict(g=A + 2), dict(ldq=319), dict(lds=19), dict(type=3), dict(q=None),
               dict(rows=-1), dict(cols=-1)):
        refused(t, ARG, **ch)
    refused(t, LARGE, cols=1 << 30, ldx=1 << 30)
    refused(t, OK, rows=0)
    d = ("tuna_fp4_dequantize", dict(q=A, ldq=128, s=A, lds=8, rows=4, cols=256, x=A, type=1, ldx=256))
    for ch in (dict(q=None), dict(ldq=127), dict(s=None), dict(lds=7), dict(x=None), dict(x=A + 1), dict(ldx=255), dict(type=2), dict(type=4), dict(rows=-1), dict(cols=-1)):
        refused(d, ARG, **ch)
    refused(d, LARGE, rows=1 << 30)
    refused(d, OK, rows=0, q=None)


def test_product_refusals():
    c = ("tuna_fp4_matmul", dict(x=A, ldx=128, xs=A, lxs=8, w=A, ldw=128, wg=100 * 128, ws=A, lws=8, wsg=800, g=A, groups=4, y=A, yt=1, ldy=100, m=10, n=100, k=256))
    for ch in (dict(x=None), dict(ldx=127), dict(xs=None), dict(lxs=7), dict(w=None), dict(ldw=127), dict(ws=None), dict(lws=7), dict(g=None), dict(groups=0),
               dict(groups=2000), dict(g=A + 1), dict(y=None), dict(yt=2), dict(yt=4), dict(ldy=99), dict(m=-1), dict(n=-1), dict(k=-1), dict(wg=-1), dict(wsg=-1),
               dict(y=A + 1), dict(k=257, lxs=9, lws=9), dict(k=257, ldx=129, ldw=129)):
        refused(c, ARG, **ch)
    refused(c, LARGE, m=1 << 31)
    refused(c, LARGE, n=1 << 30, ldy=1 << 30)
    refused(c, OK, m=0)
    refused(c, OK, n=0)
    w = ("tuna_fp4_matmul_grad_w", dict(a=A, la=320, sa=A, lsa=20, b=A, lb=320, sb=A, lsb=20, g=A, groups=3, dw=A, dt=0, ld=50, dg=2000, m=300, n=40, k=50))
    for ch in (dict(a=None), dict(la=319), dict(lsa=19), dict(b=None), dict(lb=319), dict(lsb=19), dict(dw=None), dict(dw=A + 2), dict(dt=2), dict(ld=49), dict(dg=1999),
               dict(g=None), dict(groups=0), dict(m=-1), dict(n=-1), dict(k=-1)):
        refused(w, ARG, **ch)
    refused(w, LARGE, n=1 << 31, dg=1 << 50)
    refused(w, OK, n=0)


def test_few_refusals_in_4_bits():
    rc, size = tuna.tuna_moe_few_workspace(4, 64, 48, 8, 2)
    c = ("tuna_moe_few", dict(x=A, ldx=64, n=4, h=64, l=A, lt=0, ldl=8, e=8, k=2, flags=1, w1=A, s1=A, w2=A, s2=A, f=48, wt=tuna.TUNA_F4, kind=1, out=A, ot=1, ldo=64,
                              ws=A, size=size))
    for ch in (dict(kind=0), dict(kind=2), dict(s1=None), dict(s2=None), dict(w1=None), dict(w2=None), dict(wt=3), dict(wt=5)):
        refused(c, ARG, **ch)
    refused(c, SMALL, size=size - 1)
    refused(c, OK, n=0)


def test_balance_refusals():
    rc, size = tuna.tuna_moe_balance_workspace(40, 8, 3)
    assert rc == OK and size > 0
    c = ("tuna_moe_balance", dict(l=A, type=0, ld=8, n=40, e=8, ex=A, k=2, g=A, groups=3, c=A, t=A, s=A, loss=A, ws=A, size=size))
    for ch in (dict(l=None), dict(l=A + 2), dict(type=2), dict(ld=7), dict(n=-1), dict(e=0), dict(e=1025, ld=1025), dict(ex=None), dict(ex=A + 1), dict(k=0), dict(k=17),
               dict(g=None), dict(g=A + 2), dict(groups=0), dict(groups=1025), dict(c=None), dict(t=None), dict(s=None), dict(loss=None), dict(c=A + 1), dict(t=A + 2),
               dict(s=A + 2), dict(loss=A + 2), dict(ws=None), dict(ws=A + 8)):
        refused(c, ARG, **ch)
    refused(c, SMALL, size=size - 1)
    refused(c, LARGE, n=(1 << 28) + 1)
    refused(c, LARGE, n=1 << 28, k=8)
    g = ("tuna_moe_balance_grad", dict(l=A, type=1, ld=8, n=40, e=8, g=A, groups=3, c=A, t=A, dl=A, flags=1, out=A, ldo=8))
    for ch in (dict(l=None), dict(l=A + 1), dict(type=2), dict(ld=7), dict(n=-1), dict(e=0), dict(g=None), dict(groups=0), dict(c=None), dict(t=A + 1), dict(dl=None),
               dict(flags=2), dict(out=None), dict(out=A + 1), dict(ldo=7)):
        refused(g, ARG, **ch)
    refused(g, LARGE, n=(1 << 28) + 1)
    refused(g, OK, n=0)
    assert tuna.tuna_moe_balance_workspace(-1, 8, 3)[0] == ARG and tuna.tuna_moe_balance_workspace(1 << 29, 8, 3)[0] == LARGE


@pytest.mark.parametrize("experts,groups", [(8, 1), (256, 7), (1024, 1024)])
def test_balance_workspace_never_falls(experts, groups):
    last = 0
    for n in list(range(0, 1300, 7)) + [65535, 65536, 65537, 1 << 20, 1 << 28]:
        rc, size = tuna.tuna_moe_balance_workspace(n, experts, groups)
        assert rc == OK and size >= last
        last = size


class Tensor:
    is_cuda, shape = True, (4, 256)

    def __init__(self, dtype):
        self.dtype = dtype

    def stride(self):
        return (256, 1)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return A


def test_tensors_have_the_types_that_the_call_names():
    one = lambda t: tuna.tuna_fp4_dequantize(t, 128, A, 8, 0, 256, A, 0, 256, stream=0)  # noqa: E731
    assert one(Tensor(U8)) == OK and one(Tensor(F4)) == OK
    two = lambda t: tuna.tuna_fp4_dequantize(A, 128, t, 8, 0, 256, A, 0, 256, stream=0)  # noqa: E731
    assert two(Tensor(U8)) == OK and two(Tensor(torch.float8_e8m0fnu)) == OK
    for call in (one, two):
        for t in (torch.float8_e4m3fn, torch.float32, torch.int8, torch.bfloat16):
            with pytest.raises(TypeError):
                call(Tensor(t))
    with pytest.raises(TypeError):
        tuna.tuna_moe_balance_grad(A, 0, 8, 0, 8, None, 1, Tensor(torch.int64), A, A, 0, A, 8, stream=0)
    with pytest.raises(TypeError):
        tuna.tuna_fp4_quantize(torch.zeros(4, 32), 0, 32, 4, 32, 0, None, 1, 4, A, 16, A, 1, stream=0)


# ------------------------------------------------------------------------------------------------ the definitions


def test_plain_values_are_nearest():
    v = plain.VALUES
    x = torch.linspace(-6, 6, 9601, dtype=torch.float64)
    got = plain.from_codes(plain.to_codes(x))
    best = (x[:, None].abs() - v).abs().amin(1)
    assert torch.equal((got.abs() - x.abs()).abs(), best)
    ties = (v[1:] + v[:-1]) / 2
    assert bool((plain.to_codes(ties) % 2 == 0).all())


def test_plain_scale_is_the_smallest_that_holds_the_block():
    x = torch.exp2(torch.rand(20000, generator=torch.Generator().manual_seed(0)) * 240 - 120).double()
    x = torch.cat([x, 6 * torch.exp2(torch.arange(-100.0, 100.0)).double()])
    p = plain.power(plain.scale_bytes(x))
    assert bool((x <= 6 * p).all()) and bool((x > 3 * p).all())


def test_plain_balance_gradient_is_the_derivative():
    x = torch.randn(9, 7, generator=torch.Generator().manual_seed(1)).double().requires_grad_()
    ex = torch.randint(0, 7, (9, 2), generator=torch.Generator().manual_seed(2), dtype=torch.int32)
    d, rows = torch.tensor([0.5, -2.0]), [0, 4, 9]
    counts, tokens, shares, loss = plain.balance(x.detach(), ex, rows)
    total = 0
    for s in range(2):
        f = counts[s].double() / counts[s].sum()
        one = 7 * (f * torch.softmax(x[rows[s]:rows[s + 1]], 1).mean(0)).sum()
        assert torch.allclose(one.detach(), loss[s])
        total = total + d[s] * one
    total.backward()
    assert torch.allclose(x.grad, plain.balance_grad(x.detach(), counts, tokens, rows, d))
