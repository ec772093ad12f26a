"""Every form that a rule on sizes can choose for the operators of include/tuna_moe.h, where test_gpu_moe.py's sizes choose others."""
import math

import pytest
import torch

import moe_plain as plain
import paper_2411_02581_amd as tuna
from test_gpu_moe import CODE, DEV, EPS, TYPES, few, gen, gpu_route, ok, product, rounding, strided

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ the layer, a wave for 16 columns of its own


def crowded(t, e, seed):
    """Logits that send most tokens to the first experts: more than 32 of 64 to one of them, none to others."""
    return torch.randn(t, e, generator=gen(seed)) + torch.linspace(4, -4, e)


# at least 1024 pairs times 64 columns: 16 tokens at a time with up to 8 pairs an expert on average, else 32
@pytest.mark.parametrize("t,h,f,e,k", [(40, 256, 384, 40, 8), (64, 256, 272, 128, 6), (33, 272, 520, 60, 8), (64, 256, 384, 8, 4), (64, 528, 80, 10, 8), (50, 144, 1040, 6, 2)])
@pytest.mark.parametrize("weights,kind", [("f8", "f32"), ("f8", "e8"), ("bf16", "f32")])
@pytest.mark.parametrize("logits", ["even", "crowded"])
def test_few_with_many_pairs(t, h, f, e, k, weights, kind, logits):
    assert t * k * -(-f // 64) >= 1024
    few(t, h, f, e, k, weights, kind, renorm=k % 4 == 0, logits=crowded(t, e, 5) if logits == "crowded" else None)


@pytest.mark.parametrize("dtype,lt", [("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("weights,kind,shift", [("f8", "e8", 0), ("bf16", "f32", 1)])
def test_few_with_many_pairs_off_alignment(weights, kind, shift, dtype, lt):
    few(41, 201, 403, 12, 4, weights, kind, dtype=dtype, lt=lt, shift=shift, logits=crowded(41, 12, 6))
    few(64, 200, 392, 7, 3, weights, kind, dtype=dtype, lt=lt, shift=shift)


def test_few_with_many_pairs_and_masks():
    l = crowded(64, 24, 7)
    l[::5] = -math.inf
    l[1::5] = math.nan
    l[2::5, 1:] = -math.inf
    l[3, 4], l[8, 9] = math.inf, math.inf
    few(64, 256, 384, 24, 4, "f8", "e8", True, logits=l)
    few(64, 256, 384, 24, 4, "f8", "f32", False, logits=l)


# ------------------------------------------------------------------------------------------------ the router's gradient, four and eight logits a lane


@pytest.mark.parametrize("e,k", [(4, 2), (64, 4), (200, 8), (256, 8), (260, 5), (512, 8), (1000, 16), (1024, 16)])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_route_grad_with_rows_on_sixteen_bytes(e, k, renorm, dtype):
    t = 22
    x = torch.randn(t, e, generator=gen(e)) * 2
    x[::4, :e // 2] = -math.inf
    x[1::4, e // 3] = math.nan
    x[2] = -math.inf
    x[3, :e - 1] = -math.inf
    x[5] = torch.finfo(torch.bfloat16).min
    x[6, [1, e - 1]] = math.inf
    x[7] = math.nan
    x = x.to(TYPES[dtype])
    flags = tuna.TUNA_ROUTE_RENORM if renorm else 0
    p, names, w = plain.route(x, k, renorm)
    g = torch.randn(t, k, generator=gen(9))
    exact = plain.route_grad(p, names, w, g.double(), renorm)
    # p (g - s): every factor within 64 half ulps of what is added, then the output's rounding
    room = 64 * EPS * (p if not renorm else 1.0) * (g.abs().sum(1, keepdim=True) + 1) + rounding(dtype) * exact.abs() + 1e-37
    for more in (0, 8, 1):                                       # the last one is off 16 bytes
        d, experts, weights, *_ = gpu_route(x, k, renorm, False, ld=e + more, dtype=dtype)
        assert torch.equal(experts.cpu().long(), names)
        dl = torch.full((t, e + more), 5.0, dtype=TYPES[dtype], device=DEV)
        ok(tuna.tuna_moe_route_grad(d, CODE[dtype], e + more, t, e, k, flags, experts, weights, g.to(DEV), dl, e + more))
        torch.cuda.synchronize()
        assert bool(((dl[:, :e].cpu().double() - exact).abs() <= room).all()) and bool((dl[:, e:] == 5.0).all())


# ------------------------------------------------------------------------------------------------ products of 17 to 64 rows of one group


@pytest.mark.parametrize("m,n,k", [(17, 40, 208), (20, 144, 208), (32, 100, 1168), (32, 4112, 128), (33, 24, 208), (48, 300, 2064)])
@pytest.mark.parametrize("kind", ["f32", "e8"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_matmul_of_some_rows(m, n, k, kind, dtype):
    product(m, n, k, [0, m], kind, dtype)
    product(m, n, k, [0, m], kind, dtype, pad=16)


def test_strided_helper_keeps_sixteen_bytes():
    """What the tests above rest on: rows of a tensor from `strided` start on 16 bytes where the distance says so."""
    for dtype, more in ((torch.float32, 8), (torch.bfloat16, 8), (torch.uint8, 16)):
        v = strided(torch.zeros(3, 64).to(dtype), 64 + more)
        assert v.data_ptr() % 16 == 0 and v.stride(0) * v.element_size() % 16 == 0
