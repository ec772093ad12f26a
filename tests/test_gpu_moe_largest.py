"""The operators of include/tuna_moe.h at the largest sizes that they take, and where rows pass from one axis of the grid to the next."""
import pytest
import torch

import moe_plain as plain
import paper_2411_02581_amd as tuna
from test_gpu_moe import CODE, DEV, EPS, TYPES, gen, ok, rounding

pytestmark = pytest.mark.gpu
B = (1 << 24) - 1                                                # workgroups of 256 threads in a launch


def pattern(n, period):
    """n whole numbers 0 .. period - 1 in turn, as bytes."""
    return torch.arange(period, dtype=torch.uint8, device=DEV).repeat(-(-n // period))[:n]


def test_router_and_its_gradient():
    t, e = 4 * B, 2
    which = pattern(t, 3).clamp_max(1)                           # the expert of a token: 0, 1, 1, 0, ...
    logits = torch.zeros(t, e, dtype=torch.bfloat16, device=DEV)
    logits[:, 0], logits[:, 1] = 1 - which, which
    rc, size = tuna.tuna_moe_route_workspace(t, e, 1, False)
    ok(rc)
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    experts, slots = (torch.full((t, 1), 77, dtype=torch.int32, device=DEV) for _ in range(2))
    weights, rows = torch.full((t, 1), 77.0, device=DEV), torch.zeros(e + 1, dtype=torch.int32, device=DEV)
    ok(tuna.tuna_moe_route(logits, tuna.TUNA_BF16, e, t, e, 1, 0, experts, weights, slots, rows, 1, None, None, None, None, ws, size))
    assert bool((experts[:, 0] == which).all())
    zeros = -(-t // 3)
    assert rows.tolist() == [0, zeros, t]
    at = torch.arange(t, dtype=torch.int32, device=DEV)
    third = at // 3
    want = torch.where(which == 0, third, zeros + at - third - 1)
    assert bool((slots[:, 0] == want).all())
    del want, third, at
    share = float(1 / (1 + torch.exp(torch.tensor(-1.0, dtype=torch.float64))))
    assert bool(((weights - share).abs() <= 16 * EPS).all())
    g, dl = torch.full((t, 1), 0.5, device=DEV), torch.full((t, e), 7.0, dtype=torch.bfloat16, device=DEV)
    ok(tuna.tuna_moe_route_grad(logits, tuna.TUNA_BF16, e, t, e, 1, 0, experts, weights, g, dl, e))
    slope = 0.5 * share * (1 - share)
    sign = torch.where(logits > 0, 1.0, -1.0)
    assert bool(((dl.float() * sign - slope).abs() <= (rounding("bf16") + 64 * EPS) * slope).all())


def test_rows_in_eight_bits():
    rows = 32 * B
    x = (pattern(rows, 251).bfloat16() - 125).view(rows, 1)
    q, s = torch.full((rows, 1), 0xA5, dtype=torch.uint8, device=DEV), torch.zeros(rows, 1, device=DEV)
    ok(tuna.tuna_fp8_quantize(x, tuna.TUNA_BF16, 1, rows, 1, tuna.TUNA_ACT_NONE, None, 1, rows, q, 1, s, 1, tuna.TUNA_SCALE_F32))
    table = torch.arange(251).float() - 125
    want, ws = plain.quantise(table[:, None], "f32")
    which = pattern(rows, 251)
    assert bool((q[:, 0] == want[:, 0].to(DEV)[which.int()]).all()) and bool((s[:, 0] == ws[:, 0].to(DEV)[which.int()]).all())


def test_columns_in_eight_bits():
    rows = 128 * B
    x = torch.ones(rows, 1, dtype=torch.bfloat16, device=DEV)
    x[::128] = 448                                               # the first of every block sets a scale of one
    x[-1], x[rows // 2 + 1] = -3, 5
    q, s = torch.full((1, rows), 0xA5, dtype=torch.uint8, device=DEV), torch.zeros(1, B, dtype=torch.uint8, device=DEV)
    ok(tuna.tuna_fp8_quantize_columns(x, tuna.TUNA_BF16, 1, rows, 1, None, 1, q, rows, s, B, tuna.TUNA_SCALE_E8))
    assert bool((s == 127).all())
    for at in range(0, rows, 1 << 28):
        assert bool((q[0, at:at + (1 << 28)].view(torch.float8_e4m3fn).to(torch.bfloat16) == x[at:at + (1 << 28), 0]).all())


def test_products_of_rows_off_sixteen_bytes():
    m = 64 * B
    x = pattern(m, 127).view(m, 1)                               # every e4m3 value that is not negative, in turn
    xs = torch.full((m, 1), 127, dtype=torch.uint8, device=DEV)
    w, ws = torch.full((1, 1), 0x40, dtype=torch.uint8, device=DEV), torch.full((1, 1), 126, dtype=torch.uint8, device=DEV)      # 2, and a half
    y = torch.full((m, 1), 9.0, dtype=torch.bfloat16, device=DEV)
    ok(tuna.tuna_fp8_matmul(x, 1, xs, 1, w, 1, 0, ws, 1, 0, tuna.TUNA_SCALE_E8, None, 1, y, tuna.TUNA_BF16, 1, m, 1, 1))
    table = plain.from_e4m3(torch.arange(127, dtype=torch.uint8)).bfloat16().to(DEV)
    for at in range(0, m, 1 << 28):
        assert bool((y[at:at + (1 << 28), 0] == table[x[at:at + (1 << 28), 0].int()]).all())


def test_the_sum_s_gradient():
    t, cols = B, 8
    y = torch.randn(1000, cols, generator=gen(1)).to(DEV)
    y = y.repeat(-(-t // 1000), 1)[:t].contiguous()
    slots = torch.arange(t - 1, -1, -1, dtype=torch.int32, device=DEV).view(t, 1)
    w, dout = torch.full((t, 1), 0.25, device=DEV), torch.ones(t, cols, device=DEV)
    dout[:, 0] = pattern(t, 7).float()
    dy, dw = torch.full((t, cols), 9.0, device=DEV), torch.full((t, 1), 9.0, device=DEV)
    ok(tuna.tuna_moe_combine_grad(dout, tuna.TUNA_F32, cols, y, tuna.TUNA_F32, cols, t, slots, w, t, 1, cols, dy, cols, dw))
    assert bool((dy == 0.25 * dout.flip(0)).all())
    exact = (dout.double() * y.flip(0).double()).sum(1)
    assert bool(((dw[:, 0].double() - exact).abs() <= 16 * EPS * (dout.double() * y.flip(0).double().abs()).sum(1)).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_beyond_one_axis_of_the_grid(dtype):
    """The sum and the gate's gradient have 32768 rows on one axis and the rest on the next."""
    t, cols = 2 * 32768 + 5, 24
    y = torch.randn(777, cols, generator=gen(1)).to(TYPES[dtype]).to(DEV)
    slots = torch.randint(-1, 777, (t, 2), generator=gen(2)).int().to(DEV)
    w = torch.rand(t, 2, generator=gen(3)).to(DEV)
    out = torch.full((t, cols), 9.0, dtype=TYPES[dtype], device=DEV)
    ok(tuna.tuna_moe_combine(y, CODE[dtype], cols, 777, slots, w, t, 2, cols, out, CODE[dtype], cols))
    v = torch.where((slots >= 0)[..., None], y[slots.clamp_min(0).long()].double() * w.double()[..., None], 0.0)
    exact = v.sum(1)
    assert bool(((out.double() - exact).abs() <= 4 * EPS * v.abs().sum(1) + rounding(dtype) * exact.abs()).all())
    x, dh = (torch.randn(t, c, generator=gen(4 + c)).to(TYPES[dtype]).to(DEV) for c in (2 * cols, cols))
    dx = torch.full((t, 2 * cols), 9.0, dtype=TYPES[dtype], device=DEV)
    ok(tuna.tuna_moe_swiglu_grad(x, CODE[dtype], 2 * cols, dh, cols, t, cols, dx, 2 * cols))
    exact = plain.swiglu_grad(x, dh)
    gate, up = x.double().chunk(2, -1)
    room = 32 * EPS * torch.cat([dh.double().abs() * up.abs() * (1 + gate.abs()), dh.double().abs() * gate.abs()], -1)
    assert bool(((dx.double() - exact).abs() <= room + rounding(dtype) * exact.abs() + 1e-37).all())
