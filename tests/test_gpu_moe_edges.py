"""The operators of include/tuna_moe.h on the GPU at the ends of their ranges, against their definitions in 64 bits (moe_plain.py)."""
import pytest
import torch

import moe_plain as plain
import paper_2411_02581_amd as tuna
from test_gpu_moe import CODE, DEV, EPS, KIND, STORED, TYPES, check_product, codes, gen, ok, rounding, some_scales

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ gates far below zero

GATES = [-80.0, -86.5, -87.0, -87.25, -87.5, -88.0, -88.75, -90.0, -95.0, -100.0, -103.5, -104.0, -110.0, -1e4, -1e30, -1e36, -3e38]


def far_gates(dtype, cols):
    """A row for each gate, so that no other one sets its blocks' scales; the last row's are the type's lowest value."""
    gate = torch.tensor(GATES + [torch.finfo(TYPES[dtype]).min], dtype=torch.float32)[:, None].expand(-1, cols)
    up = torch.randn(gate.shape[0], cols, generator=gen(1)) * 4
    return torch.cat([gate, up], 1).to(TYPES[dtype])


@pytest.mark.parametrize("cols", [128, 203])
@pytest.mark.parametrize("kind", ["f32", "e8"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gates_far_below_zero(cols, kind, dtype):
    x = far_gates(dtype, cols)
    rows = x.shape[0]
    dh = torch.randn(rows, cols, generator=gen(2)).to(TYPES[dtype])
    q = torch.zeros(rows, cols, dtype=torch.uint8, device=DEV)
    s = torch.zeros(rows, plain.blocks(cols), dtype=STORED[kind], device=DEV)
    g = torch.zeros(rows, 2 * cols, dtype=TYPES[dtype], device=DEV)
    ok(tuna.tuna_fp8_quantize(x.to(DEV), CODE[dtype], 2 * cols, rows, cols, tuna.TUNA_ACT_SWIGLU, None, 1, rows, q, cols, s, s.shape[1], KIND[kind]))
    ok(tuna.tuna_moe_swiglu_grad(x.to(DEV), CODE[dtype], 2 * cols, dh.to(DEV), cols, rows, cols, g, 2 * cols))
    torch.cuda.synchronize()
    gate, up = x.double().chunk(2, -1)
    # the sigmoid is a 32-bit value that may be below the smallest normal one: half a step of 2^-149, nothing where it is far below that; the
    # products with the gate and with up may end there too
    low = 2.0 ** -149 * ((gate > -110) * gate.abs() + 2) * (1 + up.abs())
    h = plain.swiglu(x)
    v = plain.wide(q.cpu(), s.cpu(), kind)
    sc = plain.scale_values(s.cpu(), kind).repeat_interleave(128, -1)[:, :cols]
    # half a step of e4m3: 1/16 of the value, or half the smallest step
    assert bool(((v - h).abs() <= torch.maximum(h.abs() / 16, sc * 2.0 ** -10) * (1 + 64 * EPS) + low).all())
    peak = torch.nn.functional.pad(h.abs(), (0, -cols % 128)).unflatten(-1, (-1, 128)).amax(-1)
    assert bool((sc[:, ::128] <= torch.where(peak < 2.0 ** -140, 1.0, (peak / 224).clamp_min(2.0 ** -126) * (1 + 64 * EPS))).all())
    exact = plain.swiglu_grad(x, dh)
    d = dh.double().abs()
    # every factor within a few half ulps of itself, for 1 + gate (1 - sigmoid) does not cancel down here
    room = 32 * EPS * exact.abs() + torch.cat([low * (1 + d), 2.0 ** -149 * ((gate > -110) * gate.abs() + 2) * (1 + d)], -1)
    step = 2.0 ** -133 if dtype == "bf16" else 2.0 ** -149       # the output's smallest
    assert bool(((g.cpu().double() - exact).abs() <= room + rounding(dtype) * exact.abs() + step).all())


@pytest.mark.parametrize("tokens", [1, 3])
def test_few_with_gates_far_below_zero(tokens):
    """The gate is -1e36 and below in every column, so nothing is left of the layer."""
    h, f, e, k = 128, 32, 4, 2
    x = torch.zeros(tokens, h, dtype=torch.bfloat16)
    x[:, 0], x[:, 1] = -1e30, 1.0
    w1, w2 = torch.zeros(e, 2 * f, h, dtype=torch.bfloat16), torch.ones(e, h, f, dtype=torch.bfloat16)
    w1[:, :f, 0] = torch.logspace(6, 8, f).bfloat16()
    w1[:, f:, 1] = 1.0
    logits = torch.randn(tokens, e, generator=gen(3))
    rc, size = tuna.tuna_moe_few_workspace(tokens, h, f, e, k)
    ok(rc)
    out, ws = torch.full((tokens, h), 9.0, device=DEV), torch.zeros(size, dtype=torch.uint8, device=DEV)
    ok(tuna.tuna_moe_few(x.to(DEV), h, tokens, h, logits.to(DEV), tuna.TUNA_F32, e, e, k, 1, w1.to(DEV), None, w2.to(DEV), None, f, tuna.TUNA_BF16, 0, out,
                         tuna.TUNA_F32, h, ws, size))
    exact, _ = plain.few(x, logits, k, True, w1.double(), w2.double())
    assert bool((exact == 0).all()) and bool((out.cpu() == 0).all())


# ------------------------------------------------------------------------------------------------ group bounds in any order


def ascending(bounds, m):
    """What bounds in any order stand for: each the largest of all up to it, inside [0, m]."""
    out, low = [], 0
    for b in bounds:
        low = max(low, min(max(b, 0), m))
        out.append(low)
    return out


def mixed(groups, m, seed):
    """Bounds that rise and fall, some of them outside [0, m]."""
    rise = torch.linspace(-20, m + 20, groups + 1)
    return (rise + torch.randn(groups + 1, generator=gen(seed)) * m / 8).int().tolist()


FALLING = [([0, 1280, 0, 1280, 0, 1280, 0, 1280, 0], 1280), ([0, 300, 100, 500, -7, 650, 2000000000, 40], 700), ([50, 20, 400], 600), ([-5, 1000, 10, 2000000000], 40),
           ([700, 0, 300], 700), ([0, 129] * 33 + [0, 128, 257, 300], 400), (mixed(70, 900, 1), 900), (mixed(130, 1500, 2), 1500)]


@pytest.mark.parametrize("bounds,m", FALLING)
@pytest.mark.parametrize("kind,cols", [("f32", 130), ("e8", 256)])
def test_columns_of_groups_in_any_order(bounds, m, kind, cols):
    groups, up = len(bounds) - 1, ascending(bounds, m)
    nb = plain.blocks(m) + groups - 1
    x = torch.randn(m, cols, generator=gen(4)).bfloat16()
    want, ws, used = plain.quantise_columns(x, up, kind, nb * 128)
    assert used <= nb
    q = torch.full((cols + 1, nb * 128), 0xA5, dtype=torch.uint8, device=DEV)
    s = torch.full((cols + 1, nb), 7, dtype=STORED[kind], device=DEV)
    ok(tuna.tuna_fp8_quantize_columns(x.to(DEV), tuna.TUNA_BF16, cols, m, cols, torch.tensor(bounds, dtype=torch.int32, device=DEV), groups, q, nb * 128, s, nb,
                                      KIND[kind]))
    torch.cuda.synchronize()
    assert torch.equal(s[:cols, :used].cpu(), ws[:, :used]) and torch.equal(q[:cols, :used * 128].cpu(), want[:, :used * 128])
    assert bool((q[:, used * 128:] == 0xA5).all()) and bool((q[cols] == 0xA5).all())
    assert bool((s[:, used:] == 7).all()) and bool((s[cols] == 7).all())


# the simple form, tiles of 128 x 128, few rows a group, tiles of 256 x 256
@pytest.mark.parametrize("bounds,m,n,k", [(b, m, 40, 100) for b, m in FALLING] + [(b, m, 144, 272) for b, m in FALLING] +
                         [(mixed(70, 100, 3), 100, 48, 272), (mixed(8, 2560, 5), 2560, 8200, 128)])
@pytest.mark.parametrize("kind,dtype", [("f32", "f32"), ("e8", "bf16")])
def test_matmul_of_groups_in_any_order(bounds, m, n, k, kind, dtype):
    groups, up, nk, nn = len(bounds) - 1, ascending(bounds, m), plain.blocks(k), plain.blocks(n)
    x, xs = codes(m, k, 1), some_scales((m, nk), kind, 2)
    w, ws = codes(groups * n, k, 3), some_scales((groups * nn, nk), kind, 4)
    y = torch.full((m + 1, n), 9.0, dtype=TYPES[dtype], device=DEV)
    ok(tuna.tuna_fp8_matmul(x.to(DEV), k, xs.to(DEV), nk, w.to(DEV), k, n * k, ws.to(DEV), nk, nn * nk, KIND[kind],
                            torch.tensor(bounds, dtype=torch.int32, device=DEV), groups, y, CODE[dtype], n, m, n, k))
    torch.cuda.synchronize()
    a, b = plain.wide(x, xs, kind), plain.wide(w.view(groups, n, k), ws.view(groups, nn, nk), kind, 128)
    for g in range(groups):
        check_product(y[up[g]:up[g + 1]], a[up[g]:up[g + 1]], b[g], dtype, k)
    assert bool((y[:up[0]] == 9.0).all()) and bool((y[up[-1]:] == 9.0).all())


@pytest.mark.parametrize("bounds,m", FALLING)
@pytest.mark.parametrize("n,k", [(70, 33), (130, 144)])
@pytest.mark.parametrize("kind,dtype", [("f32", "f32"), ("e8", "bf16")])
def test_grad_w_of_groups_in_any_order(bounds, m, n, k, kind, dtype):
    groups, up = len(bounds) - 1, ascending(bounds, m)
    nb = plain.blocks(m) + groups - 1
    (q, s, used), (p, t, _) = (plain.quantise_columns(torch.randn(m, c, generator=gen(c)), up, kind, nb * 128) for c in (n, k))
    for v in (q, p):
        v[:, used * 128:] = 0x7F                                 # what lies behind the groups' blocks is not read
    dw = torch.full((groups, n, k + 2), 9.0, dtype=TYPES[dtype], device=DEV)
    ok(tuna.tuna_fp8_matmul_grad_w(q.to(DEV), nb * 128, s.to(DEV), nb, p.to(DEV), nb * 128, t.to(DEV), nb, KIND[kind],
                                   torch.tensor(bounds, dtype=torch.int32, device=DEV), groups, dw, CODE[dtype], k + 2, n * (k + 2), m, n, k))
    torch.cuda.synchronize()
    at = 0
    for g in range(groups):
        c = plain.blocks(up[g + 1] - up[g])
        part = slice(at * 128, (at + c) * 128)
        a, b = (plain.wide(v[:, part], z[:, at:at + c], kind) if c else torch.zeros(v.shape[0], 0).double() for v, z in ((q, s), (p, t)))
        check_product(dw[g, :, :k], a, b, dtype, max(c, 1) * 128)
        at += c
    assert bool((dw[:, :, k:] == 9.0).all())


# ------------------------------------------------------------------------------------------------ activations between the two kernels of the layer for few tokens


def few_plain(x, w1, w2, e, k=1, logits=None, out_type="f32"):
    """The layer with bf16 weights; every token's experts by `logits` (the first one)."""
    t, h, f = x.shape[0], x.shape[1], w2.shape[2]
    logits = torch.zeros(t, e) if logits is None else logits
    rc, size = tuna.tuna_moe_few_workspace(t, h, f, e, k)
    ok(rc)
    out, ws = torch.full((t, h), 9.0, dtype=TYPES[out_type], device=DEV), torch.zeros(size, dtype=torch.uint8, device=DEV)
    ok(tuna.tuna_moe_few(x.to(DEV), h, t, h, logits.to(DEV), tuna.TUNA_F32, e, e, k, 1, w1.to(DEV), None, w2.to(DEV), None, f, tuna.TUNA_BF16, 0, out,
                         CODE[out_type], h, ws, size))
    torch.cuda.synchronize()
    return out.cpu()


@pytest.mark.parametrize("tokens", [1, 5])
def test_few_with_activations_beyond_bf16(tokens):
    """Finite activations above bf16's largest value: a first part that is rounded to nearest would be infinite."""
    h, f, e = 128, 16, 2
    x = torch.zeros(tokens, h, dtype=torch.bfloat16)
    w1, w2 = torch.zeros(e, 2 * f, h, dtype=torch.bfloat16), torch.zeros(e, h, f, dtype=torch.bfloat16)
    x[:, 0], x[:, 1], x[:, 2] = torch.finfo(torch.bfloat16).max, 1.5 * 2.0 ** 119, 1.0
    w1[:, :f, :2] = 1.0                                          # gate: 2^128 - 2^118, which is nearer to 2^128 than to bf16's largest
    w1[:, f:, 2] = 1.0                                           # up: one, or minus one
    w1[:, f + 1::2, 2] = -1.0
    w2[:] = (torch.eye(f).repeat(h // f, 1) * 2.0 ** -100).bfloat16()
    got = few_plain(x, w1, w2, e).double()
    exact, _ = plain.few(x, torch.zeros(tokens, e), 1, True, w1.double(), w2.double())
    assert bool((plain.swiglu(w1[0].double() @ x[0].double()).abs() > float(torch.finfo(torch.bfloat16).max) + 2.0 ** 119).any())
    assert bool((plain.swiglu(w1[0].double() @ x[0].double()).abs() < float(torch.finfo(torch.float32).max)).all())
    # two sums of two terms, a product, then 2^-16 of the activation at most
    assert bool(((got - exact).abs() <= 2.0 ** -15 * exact.abs()).all())


@pytest.mark.parametrize("tokens,f", [(1, 48), (5, 48), (30, 2304)])
def test_few_keeps_sixteen_bits_of_an_activation(tokens, f):
    """The second product passes single activations through: two parts of eight bits each, 2^-16 of the activation, and what its own sum needs."""
    h, e = 256, 2
    x = torch.randn(tokens, h, generator=gen(1)).bfloat16()
    w1 = (torch.randn(e, 2 * f, h, generator=gen(2)) * 0.1).bfloat16()
    w2 = torch.zeros(e, h, f, dtype=torch.bfloat16)
    at = torch.randint(0, f, (h,), generator=gen(3))
    w2[:, torch.arange(h), at] = 1.0
    got = few_plain(x, w1, w2, e).double()
    exact, _ = plain.few(x, torch.zeros(tokens, e), 1, True, w1.double(), w2.double())
    gate, up = (x.double() @ w1[0].double().t()).chunk(2, -1)
    size_g, size_u = (x.double().abs() @ w1[0].double().abs().t()).chunk(2, -1)
    # a product's sum of 256 terms: 128 half ulps of the magnitudes (blocks of 128 in 32 bits); silu has a slope of at most 1.1
    room = 2.0 ** -16 * exact.abs() + (130 * EPS * (1.1 * size_g * up.abs() + size_u * gate.abs()))[:, at] + 8 * EPS * exact.abs()
    assert bool(((got - exact).abs() <= room).all())


# ------------------------------------------------------------------------------------------------ products that cancel


@pytest.mark.parametrize("m,n,k", [(20, 48, 256), (130, 144, 384), (70, 33, 200)])
@pytest.mark.parametrize("kind", ["f32", "e8"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_matmul_of_large_terms_that_cancel(m, n, k, kind, dtype):
    """In every eight neighbours two products of 2^17 cancel beside six of about one.  In 32 bits the sum is exact (whole numbers below 2^24); in bf16 it is
    held to the magnitudes, which is all that is said of it: the small terms of such a sum are lost."""
    x = torch.randint(-1, 2, (m, k), generator=gen(1)).double()
    w = torch.randint(-1, 2, (n, k), generator=gen(2)).double()
    x[:, 0:k - 4:8], w[:, 0:k - 4:8] = 384.0, 352.0
    x[:, 3:k - 4:8], w[:, 3:k - 4:8] = -384.0, 352.0
    one = (lambda *s: torch.ones(*s, device=DEV)) if kind == "f32" else (lambda *s: torch.full(s, 127, dtype=torch.uint8, device=DEV))
    nk = plain.blocks(k)
    y = torch.full((m, n), 9.0, dtype=TYPES[dtype], device=DEV)
    ok(tuna.tuna_fp8_matmul(plain.to_e4m3(x).to(DEV), k, one(m, nk), nk, plain.to_e4m3(w).to(DEV), k, 0, one(plain.blocks(n), nk), nk, 0, KIND[kind], None, 1, y,
                            CODE[dtype], n, m, n, k))
    torch.cuda.synchronize()
    exact = x @ w.t()
    assert float(exact.abs().max()) < 2 ** 8
    if dtype == "f32":
        assert torch.equal(y.cpu().double(), exact)
    check_product(y, x, w, dtype, k)
    # what the header says: 2^-10 of the magnitudes, and the output's rounding
    assert bool(((y.cpu().double() - exact).abs() <= 2.0 ** -10 * (x.abs() @ w.abs().t()) + rounding(dtype) * exact.abs()).all())


# ------------------------------------------------------------------------------------------------ not a number, in every form of the product


# few rows, the simple form, tiles of 128 x 128 and of 256 x 256
@pytest.mark.parametrize("m,n,k", [(20, 144, 256), (70, 130, 200), (70, 130, 256), (300, 272, 272), (4100, 4100, 128)])
@pytest.mark.parametrize("kind", ["f32", "e8"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_not_a_number_stays_in_its_row_and_column(m, n, k, kind, dtype):
    x, w = codes(m, k, 3), codes(n, k, 4)
    x[5, 17], w[9, k - 3], x[m - 1, k - 1] = 0x7F, 0xFF, 0x7F
    nk = plain.blocks(k)
    one = (lambda *s: torch.ones(*s, device=DEV)) if kind == "f32" else (lambda *s: torch.full(s, 127, dtype=torch.uint8, device=DEV))
    y = torch.zeros(m, n, dtype=TYPES[dtype], device=DEV)
    ok(tuna.tuna_fp8_matmul(x.to(DEV), k, one(m, nk), nk, w.to(DEV), k, 0, one(plain.blocks(n), nk), nk, 0, KIND[kind], None, 1, y, CODE[dtype], n, m, n, k))
    nan = y.cpu().isnan()
    assert bool(nan[5].all()) and bool(nan[m - 1].all()) and bool(nan[:, 9].all()) and int(nan.sum()) == m + 2 * n - 2
