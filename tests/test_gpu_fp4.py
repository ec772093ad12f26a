"""The 4-bit operators of include/tuna_moe.h on the GPU against their definitions in 64 bits (fp4_plain.py)."""
import math

import pytest
import torch

import fp4_plain as plain
import moe_plain
import paper_2411_02581_amd as tuna

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CODE = {"f32": tuna.TUNA_F32, "bf16": tuna.TUNA_BF16}
EPS = 2.0 ** -24                                                 # half a unit in the last place of a 32-bit value
U8 = torch.uint8


def gen(seed):
    return torch.Generator().manual_seed(seed)


def ok(rc):
    assert rc == tuna.TUNA_OK, tuna.tuna_strerror(rc)


def strided(x, ld=None, shift=0, fill=0):
    """A copy of the CPU matrix `x` on the GPU whose rows lie `ld` apart, `shift` elements behind the start of its memory; `fill` between them."""
    rows, cols = x.shape
    ld = ld or cols
    mem = torch.full((shift + rows * ld + 64,), fill, dtype=x.dtype, device=DEV)
    v = mem[shift:shift + rows * ld].view(rows, ld)[:, :cols]
    v.copy_(x)
    return v


def rounding(dtype):
    return 2.0 ** -8 if dtype == "bf16" else EPS                 # of one value, once


# ------------------------------------------------------------------------------------------------ rows and columns in 4 bits


def wild(rows, cols, seed):
    """Values over many powers of two, ties, and blocks of zeros, of subnormal and of the largest values; infinities and NaN in some rows."""
    g = gen(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp2(torch.randint(-30, 30, (rows, 1), generator=g).float())
    ties = torch.randint(-24, 25, (rows, cols), generator=g).float() / 4
    x = torch.where(torch.rand(rows, cols, generator=g) < 0.3, ties, x)
    x[::5, :40] = 0.0
    x[::5, 1:40:3] = -0.0
    x[1::7] *= 2.0 ** -126
    x[2::7] = torch.sign(x[2::7]) * 3.0e38
    x[3::11, cols // 2] = math.nan
    x[4::11, cols // 3] = math.inf
    x[6::11, -1] = -math.inf
    x[7::9] = ties[7::9]
    return x


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (3, 33), (9, 31), (7, 1000), (20, 256), (5, 4099), (130, 72)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantise_and_read_back(rows, cols, dtype):
    x = wild(rows, cols, rows + cols).to(TYPES[dtype])
    want, ws = plain.quantise(x)
    want = plain.packed(want)
    half, nb = plain.blocks(cols, 2), plain.blocks(cols)
    for ld, lq, ls, shift in ((cols, half, nb, 0), (cols + 3, half + 1, nb + 2, 1), (plain.blocks(cols, 16) * 16, plain.blocks(half, 16) * 16, plain.blocks(nb, 4) * 4, 0)):
        d = strided(x, ld, shift)
        mem = torch.full((shift + rows * lq + 16,), 0x5A, dtype=U8, device=DEV)
        q, s = mem[shift:shift + rows * lq].view(rows, lq), torch.full((rows, ls), 0x5A, dtype=U8, device=DEV)
        ok(tuna.tuna_fp4_quantize(d, CODE[dtype], ld, rows, cols, 0, None, 1, rows, q, lq, s, ls))
        torch.cuda.synchronize()
        assert torch.equal(q[:, :half].cpu(), want) and torch.equal(s[:, :nb].cpu(), ws)
        assert bool((q[:, half:] == 0x5A).all()) and bool((s[:, nb:] == 0x5A).all()) and bool((mem[shift + rows * lq:] == 0x5A).all())
        if cols % 2:
            q[:, half - 1] |= 0xF0                               # not read
        for out in ("f32", "bf16"):
            back = torch.full((rows, ld + 8), 9.0, dtype=TYPES[out], device=DEV)
            ok(tuna.tuna_fp4_dequantize(q, lq, s, ls, rows, cols, back, CODE[out], ld + 8))
            exact = plain.wide(plain.unpacked(want, cols), ws).to(TYPES[out])      # 3.53 * 2^126 is held as 2^128, which neither type has: infinity
            assert torch.equal(back[:, :cols].cpu().float().nan_to_num(nan=7e7), exact.float().nan_to_num(nan=7e7))
            assert bool((back[:, cols:] == 9.0).all())


def test_read_back_of_every_code_and_scale():
    q = torch.arange(256, dtype=U8).repeat(256, 1)
    s = torch.arange(256, dtype=U8)[:, None].repeat(1, 16)
    exact = plain.wide(plain.unpacked(q, 512), s)
    for out in ("f32", "bf16"):
        back = torch.empty(256, 512, dtype=TYPES[out], device=DEV)
        ok(tuna.tuna_fp4_dequantize(q.to(DEV), 256, s.to(DEV), 16, 256, 512, back, CODE[out], 512))
        want = exact.to(TYPES[out])                              # only what is above the largest value is not held exactly: infinity
        assert torch.equal(back.cpu().float().nan_to_num(nan=7e7), want.float().nan_to_num(nan=7e7))


def test_every_border_of_a_scale_and_of_a_value():
    """Largest values on both sides of 6 times a power of two, and values on both sides of every tie, over the whole range of exponents."""
    x = []
    for e in range(-126, 126, 3):
        for v in (6.0, 3.0, 4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0):
            t = torch.tensor(v * 2.0 ** e if e > -124 or v > 1 else v * 2.0 ** -120)
            row = torch.zeros(3, 32)
            for i in range(3):
                row[i, 0] = [t, torch.nextafter(t, torch.tensor(math.inf)), torch.nextafter(t, torch.tensor(0.0))][i]
                row[i, 1] = 6.0 * 2.0 ** e if v < 6 else 0.0
                row[i, 2] = -row[i, 0]
            x.append(row)
    x = torch.cat(x)
    q, s = torch.empty(x.shape[0], 16, dtype=U8, device=DEV), torch.empty(x.shape[0], 1, dtype=U8, device=DEV)
    ok(tuna.tuna_fp4_quantize(x.to(DEV), tuna.TUNA_F32, 32, x.shape[0], 32, 0, None, 1, x.shape[0], q, 16, s, 1))
    want, ws = plain.quantise(x)
    assert torch.equal(q.cpu(), plain.packed(want)) and torch.equal(s.cpu(), ws)


def test_quantise_to_slots():
    rows, cols, k, out = 30, 200, 4, 100
    x = torch.randn(rows, cols, generator=gen(1)).bfloat16()
    slots = torch.randperm(rows * k, generator=gen(2)).int().view(rows, k)
    slots[slots >= out] = -1
    slots[3, 1], slots[4, 2] = -5, 1 << 30
    rec = torch.full((out, 112), 0x5A, dtype=U8, device=DEV)
    ok(tuna.tuna_fp4_quantize(x.to(DEV), tuna.TUNA_BF16, cols, rows, cols, 0, slots.to(DEV), k, out, rec, 112, rec[:, 100:], 112))
    want, ws = plain.quantise(x)
    exact = torch.full((out, 112), 0x5A, dtype=U8)
    for r in range(rows):
        for to in slots[r].tolist():
            if 0 <= to < out:
                exact[to, :100], exact[to, 100:107] = plain.packed(want[r]), ws[r]
    assert torch.equal(rec.cpu(), exact)


@pytest.mark.parametrize("rows,cols", [(1, 8), (33, 200), (9, 1031), (100, 384)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_swiglu_quantised(rows, cols, dtype):
    x = (torch.randn(rows, 2 * cols, generator=gen(rows)) * 3).to(TYPES[dtype])
    x[0, 0], x[-1, cols - 1] = -100.0, -89.0
    half, nb = plain.blocks(cols, 2), plain.blocks(cols)
    act = plain.swiglu(x)
    for ld in (2 * cols, 2 * cols + 5):
        q, s = torch.empty(rows, half, dtype=U8, device=DEV), torch.empty(rows, nb, dtype=U8, device=DEV)
        ok(tuna.tuna_fp4_quantize(strided(x, ld), CODE[dtype], ld, rows, cols, tuna.TUNA_ACT_SWIGLU, None, 1, rows, q, half, s, nb))
        s, codes = s.cpu(), plain.unpacked(q.cpu(), cols)
        # silu(gate) up in 32 bits: an exponential of 2 units, a sum, a quotient of 1, two products: 8 units are 2^-20; the scale is one of those that
        # such values have, and the value is the nearest to one of them
        peak = torch.nn.functional.pad(act.abs(), (0, -cols % 32)).unflatten(-1, (-1, 32)).amax(-1)
        near = [plain.scale_bytes((peak * (1 + d)).float().double()) for d in (-2.0 ** -19, 2.0 ** -19)]
        assert bool(((s == near[0]) | (s == near[1])).all())
        p = plain.power(s).repeat_interleave(32, -1)[:, :cols]
        got, scaled = plain.from_codes(codes), act / p
        best = plain.from_codes(plain.to_codes(scaled.clamp(-6, 6)))
        assert bool(((got - scaled).abs() <= (best - scaled).abs() + 2.0 ** -19 * (scaled.abs() + 1e-30)).all())


ROWS = [[0, 1], [0, 128], [0, 300], [0, 5, 5, 133, 400], [0, 0, 0, 7], [3, 70, 290], [0, 256, 512]]


@pytest.mark.parametrize("bounds", ROWS)
@pytest.mark.parametrize("cols", [1, 130, 256])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantise_columns(bounds, cols, dtype):
    rows, groups = bounds[-1] + 2, len(bounds) - 1
    if groups == 1:
        rows = bounds[-1]
    x = wild(rows, cols, rows).to(TYPES[dtype])
    x[rows // 2:] *= 0.5
    nb = plain.blocks(rows, 128) + groups - 1
    want, ws, n = plain.quantise_columns(x, bounds, nb)
    want = plain.packed(want)
    for ld, lq, ls, shift in ((cols, 64 * nb, 4 * nb, 0), (cols + 3, 64 * nb + 5, 4 * nb + 1, 1), (plain.blocks(cols, 8) * 8, 64 * nb + 16, 4 * nb + 4, 0)):
        mem = torch.full((cols * lq + 80,), 0x5A, dtype=U8, device=DEV)
        q, s = mem[shift:shift + cols * lq].view(cols, lq), torch.full((cols, ls), 0x5A, dtype=U8, device=DEV)
        ok(tuna.tuna_fp4_quantize_columns(strided(x, ld), CODE[dtype], ld, rows, cols, torch.tensor(bounds, dtype=torch.int32, device=DEV) if groups > 1 else None,
                                          groups, q, lq, s, ls))
        torch.cuda.synchronize()
        assert torch.equal(q[:, :64 * n].cpu(), want[:, :64 * n]) and torch.equal(s[:, :4 * n].cpu(), ws[:, :4 * n])
        assert bool((q[:, 64 * n:] == 0x5A).all()) and bool((s[:, 4 * n:] == 0x5A).all())


# ------------------------------------------------------------------------------------------------ products


def codes(rows, cols, seed):
    return torch.randint(0, 16, (rows, cols), generator=gen(seed), dtype=U8)


def some_scales(shape, seed, spread=8):
    return torch.randint(127 - spread, 127 + spread, shape, generator=gen(seed), dtype=U8)


def check_product(got, a, b, dtype):
    """The products are exact; a step of 128 of them and the sum so far are added to within 2^-23 of their magnitudes: 2^-23 of all magnitudes for each step."""
    size = a.abs() @ b.abs().t()
    exact = a @ b.t()
    room = (plain.blocks(a.shape[1], 128) + 16) * 2 * EPS * size + rounding(dtype) * exact.abs()      # (up to 16 partial sums are added at the end)
    assert bool(((got.cpu().double() - exact).abs() <= room + 1e-37).all())


def dirty(q, n):
    """Packed rows whose high half behind an odd row's end holds something."""
    if n % 2:
        q = q.clone()
        q[:, -1] |= 0xF0
    return q


def product(m, n, k, bounds, dtype, pad=0, shift=0, spread=8):
    groups, half, nb = len(bounds) - 1, plain.blocks(k, 2), plain.blocks(k)
    x, xs = codes(m, k, m + k), some_scales((m, nb), 1, spread)
    w, ws = codes(groups * n, k, n + k), some_scales((groups * n, nb), 2, spread)
    ld, ls = half + pad, nb + (pad + 3) // 4 if pad else nb
    if pad == 16:                                                # rows on 16 bytes, scales on 4
        ld, ls = plain.blocks(half, 16) * 16, plain.blocks(nb, 4) * 4
    dx, dw = strided(dirty(plain.packed(x), k), ld, shift, 0x77), strided(dirty(plain.packed(w), k), ld, shift, 0x77)
    dxs, dws = strided(xs, ls, 4 * shift, 0xFF), strided(ws, ls, 4 * shift, 0xFF)          # NaN between the rows
    y = torch.full((m, n + pad), 9.0, dtype=TYPES[dtype], device=DEV)
    rows = torch.tensor(bounds, dtype=torch.int32, device=DEV) if groups > 1 else None
    ok(tuna.tuna_fp4_matmul(dx, ld, dxs, ls, dw, ld, n * ld, dws, ls, n * ls, rows, groups, y, CODE[dtype], n + pad, m, n, k))
    torch.cuda.synchronize()
    a, b = plain.wide(x, xs), plain.wide(w, ws).view(groups, n, k)
    for g in range(groups):
        i, j = bounds[g], bounds[g + 1]
        check_product(y[i:j, :n], a[i:j], b[g], dtype)
    assert bool((y[:, n:] == 9.0).all())
    assert bool((y[bounds[-1]:] == 9.0).all()) and bool((y[:bounds[0]] == 9.0).all())


SHAPES = [(1, 1, 1), (1, 16, 128), (3, 130, 129), (16, 64, 256), (17, 33, 100), (64, 256, 512), (65, 257, 640), (130, 144, 1040), (200, 384, 304), (300, 520, 2048),
          (513, 300, 272), (40, 2064, 384), (640, 640, 128), (5, 70, 2880)]


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("pad", [0, 16])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_matmul(m, n, k, pad, dtype):
    product(m, n, k, [0, m], dtype, pad)


@pytest.mark.parametrize("m,n,k,pad,shift", [(33, 70, 200, 3, 1), (33, 70, 208, 16, 0), (33, 64, 208, 0, 8), (150, 131, 257, 0, 0), (270, 260, 384, 32, 16),
                                             (270, 260, 385, 16, 16)])
def test_matmul_strides_and_alignment(m, n, k, pad, shift):
    product(m, n, k, [0, m], "f32", pad, shift)


@pytest.mark.parametrize("k", list(range(225, 290)) + [511, 513, 767])
def test_matmul_of_every_length(k):
    """Rows that end inside a block, a step and a stage."""
    product(70, 80, k, [0, 70], "f32", 16)
    product(3, 20, k, [0, 3], "f32", 16)


@pytest.mark.parametrize("m,n,k", [(40, 48, 640), (300, 270, 640)])
def test_matmul_of_widely_spread_scales(m, n, k):
    product(m, n, k, [0, m], "f32", 16, spread=60)


@pytest.mark.parametrize("bounds", [[0, 0, 5, 5, 140, 300, 300], [0, 1, 2, 3, 4], [3, 70, 290], [0, 256, 512, 770], [0, 0, 0, 900]] +
                         [[min(g * 37, 2500) for g in range(70)]])
@pytest.mark.parametrize("n,k,pad", [(144, 272, 0), (300, 128, 0), (300, 400, 16)])
def test_matmul_of_groups(bounds, n, k, pad):
    product(bounds[-1] + (2 if bounds[0] else 0), n, k, bounds, "bf16", pad)


def test_matmul_group_bounds_are_held_inside():
    """Bounds outside [0, m] and falling ones: a bound counts as the largest of all up to it."""
    m, n, k, bounds = 90, 70, 256, [-5, 40, 20, 60, 1000]
    x, w = codes(m, k, 1), codes(4 * n, k, 2)
    one = lambda r: torch.full((r, 8), 127, dtype=U8, device=DEV)  # noqa: E731
    y = torch.full((m, n), 9.0, device=DEV)
    ok(tuna.tuna_fp4_matmul(plain.packed(x).to(DEV), 128, one(m), 8, plain.packed(w).to(DEV), 128, n * 128, one(4 * n), 8, n * 8,
                            torch.tensor(bounds, dtype=torch.int32, device=DEV), 4, y, tuna.TUNA_F32, n, m, n, k))
    a, b = plain.from_codes(x), plain.from_codes(w).view(4, n, k)
    for g, (i, j) in enumerate([(0, 40), (40, 40), (40, 60), (60, 90)]):
        check_product(y[i:j], a[i:j], b[g], "f32")


def test_matmul_of_nothing():
    y = torch.full((5, 6), 9.0, device=DEV)
    ok(tuna.tuna_fp4_matmul(None, 8, None, 8, None, 8, 0, None, 8, 0, None, 1, y, 0, 6, 5, 6, 0))
    assert bool((y == 0).all())
    ok(tuna.tuna_fp4_matmul(None, 8, None, 8, None, 8, 0, None, 8, 0, None, 1, None, 0, 6, 0, 6, 8))


@pytest.mark.parametrize("m,n,k", [(9, 40, 320), (80, 200, 320), (600, 300, 320)])
def test_matmul_not_a_number_stays_in_its_row(m, n, k):
    x, w = codes(m, k, 1), codes(n, k, 2)
    xs, ws = some_scales((m, 12), 3), some_scales((n, 12), 4)
    xs[:, 10:], ws[:, 10:] = 255, 255                            # behind the rows' ends: not read
    xs[m // 2, 3] = 255
    ws[n - 1, 9] = 255
    y = torch.empty(m, n, device=DEV)
    ok(tuna.tuna_fp4_matmul(plain.packed(x).to(DEV), k // 2, xs.to(DEV), 12, plain.packed(w).to(DEV), k // 2, 0, ws.to(DEV), 12, 0, None, 1, y, 0, n, m, n, k))
    bad = y.isnan().cpu()
    want = torch.zeros(m, n, dtype=torch.bool)
    want[m // 2], want[:, n - 1] = True, True
    assert torch.equal(bad, want)


@pytest.mark.parametrize("bounds", ROWS + [[0, 700], [0, 500, 500, 513]])
@pytest.mark.parametrize("n,k", [(1, 1), (70, 130), (128, 264), (272, 300)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_grad_w(bounds, n, k, dtype):
    rows, groups = bounds[-1], len(bounds) - 1
    dy, x = torch.randn(rows, n, generator=gen(1)).bfloat16(), torch.randn(rows, k, generator=gen(2))
    nb = plain.blocks(rows, 128) + groups - 1
    d = torch.tensor(bounds, dtype=torch.int32, device=DEV) if groups > 1 else None
    for pad in (0, 16, 5):
        lq, ls, side = 64 * nb + pad, 4 * nb + (pad and 4 + pad % 2), []
        for v, c, name in ((dy, n, "bf16"), (x, k, "f32")):
            q, s = torch.full((c, lq), 0x77, dtype=U8, device=DEV), torch.full((c, ls), 255, dtype=U8, device=DEV)
            ok(tuna.tuna_fp4_quantize_columns(v.to(DEV), CODE[name], c, rows, c, d, groups, q, lq, s, ls))
            side += [q, lq, s, ls]
        dw = torch.full((groups, n, k + 2), 9.0, dtype=TYPES[dtype], device=DEV)
        ok(tuna.tuna_fp4_matmul_grad_w(*side, d, groups, dw, CODE[dtype], k + 2, n * (k + 2), rows, n, k))
        torch.cuda.synchronize()
        assert bool((dw[..., k:] == 9.0).all())
        for g in range(groups):
            a, b = bounds[g], bounds[g + 1]
            if a == b:
                assert bool((dw[g, :, :k] == 0).all())
                continue
            check_product(dw[g, :, :k], plain.held(dy[a:b].t()), plain.held(x[a:b].t()), dtype)


def test_products_are_each_others_gradients():
    """A linear layer in 4 bits: y, dx and dw against the derivatives of sum(y * g) by differences, every operand being what 4 bits hold of it."""
    m, n, k = 48, 96, 64
    g = gen(5)
    x, w, dy = (plain.held(torch.randn(*s, generator=g)).float() for s in ((m, k), (n, k), (m, n)))
    def side(v, columns):
        r, c = v.shape
        if columns:
            q, s = torch.empty(c, 64 * plain.blocks(r, 128), dtype=U8, device=DEV), torch.empty(c, 4 * plain.blocks(r, 128), dtype=U8, device=DEV)
            ok(tuna.tuna_fp4_quantize_columns(v.to(DEV), 0, c, r, c, None, 1, q, q.shape[1], s, s.shape[1]))
        else:
            q, s = torch.empty(r, c // 2, dtype=U8, device=DEV), torch.empty(r, c // 32, dtype=U8, device=DEV)
            ok(tuna.tuna_fp4_quantize(v.to(DEV), 0, c, r, c, 0, None, 1, r, q, c // 2, s, c // 32))
        return q, q.shape[1], s, s.shape[1]

    def matmul(a, b, m, n, k):
        out = torch.empty(m, n, device=DEV)
        q, ld, s, ls = side(b, False) if not isinstance(b, tuple) else b
        ok(tuna.tuna_fp4_matmul(*side(a, False), q, ld, 0, s, ls, 0, None, 1, out, 0, n, m, n, k))
        return out.cpu().double()

    dx = matmul(dy, side(w, True), m, k, n)
    wt = plain.held(w.t())                                       # what the other axis' blocks hold of w
    dw = torch.empty(n, k, device=DEV)
    ok(tuna.tuna_fp4_matmul_grad_w(*side(dy, True), *side(x, True), None, 1, dw, 0, k, n * k, m, n, k))
    dyt, xt = plain.held(dy.t()), plain.held(x.t())
    h, base = 0.5, lambda a, b, c: float((a.double() @ b.double().t() * c.double()).sum())  # noqa: E731
    for i, j in ((0, 0), (3, 5), (m - 1, k - 1), (17, 33)):
        e = torch.zeros(m, k, dtype=torch.float64)
        e[i, j] = h
        slope = (base(x + e, wt.t(), dy) - base(x - e, wt.t(), dy)) / (2 * h)
        assert abs(float(dx[i, j]) - slope) <= 2.0 ** -20 * float((dy[i].double().abs() * wt[j].abs()).sum()) + 1e-9
    for i, j in ((0, 0), (3, 5), (n - 1, k - 1), (17, 33)):
        e = torch.zeros(n, k, dtype=torch.float64)
        e[i, j] = h
        slope = (base(xt.t(), w + e, dyt.t()) - base(xt.t(), w - e, dyt.t())) / (2 * h)
        assert abs(float(dw[i, j]) - slope) <= 2.0 ** -20 * float((dyt[i].abs() * xt[j].abs()).sum()) + 1e-9
    y = matmul(x, w, m, n, k)
    check_product(y, x.double(), w.double(), "f32")


def test_weights_by_columns_are_the_other_product_s():
    """w [groups n, k] by columns, with the bounds 0, n, 2 n: w transposed of every group, at the distances that the header names."""
    groups, n, k, m = 3, 150, 70, 40
    w, dy = torch.randn(groups * n, k, generator=gen(1)), torch.randn(m, n, generator=gen(2)).bfloat16()
    per = plain.blocks(n, 128)
    nb = plain.blocks(groups * n, 128) + groups - 1
    q, s = torch.full((k, 64 * nb), 0x77, dtype=U8, device=DEV), torch.full((k, 4 * nb), 255, dtype=U8, device=DEV)
    at = torch.arange(groups + 1, dtype=torch.int32, device=DEV) * n
    ok(tuna.tuna_fp4_quantize_columns(w.to(DEV), 0, k, groups * n, k, at, groups, q, 64 * nb, s, 4 * nb))
    dq, ds = torch.empty(m, n // 2, dtype=U8, device=DEV), torch.empty(m, plain.blocks(n), dtype=U8, device=DEV)
    ok(tuna.tuna_fp4_quantize(dy.to(DEV), 1, n, m, n, 0, None, 1, m, dq, n // 2, ds, plain.blocks(n)))
    bounds = [0, 7, 7, m]
    dx = torch.empty(m, k, device=DEV)
    ok(tuna.tuna_fp4_matmul(dq, n // 2, ds, plain.blocks(n), q, 64 * nb, 64 * per, s, 4 * nb, 4 * per, torch.tensor(bounds, dtype=torch.int32, device=DEV), groups,
                            dx, 0, k, m, k, n))
    for g in range(groups):
        a, b = bounds[g], bounds[g + 1]
        check_product(dx[a:b], plain.held(dy[a:b]), plain.held(w[g * n:(g + 1) * n].t()), "f32")


# ------------------------------------------------------------------------------------------------ the layer for a few tokens


def few(t, h, f, e, k, renorm=True, dtype="bf16", logits=None, lt="f32", shift=0):
    x = torch.randn(t, h, generator=gen(1)).bfloat16()
    logits = (torch.randn(t, e, generator=gen(2)) * 2 if logits is None else logits).to(TYPES[lt])
    dev, vals = [], []
    for i, (r, c) in enumerate(((2 * f, h), (h, f))):
        q, s = codes(e * r, c, 3 + i), torch.randint(118, 124, (e * r, plain.blocks(c)), generator=gen(5 + i), dtype=U8)
        vals.append(plain.wide(q, s).view(e, r, c))
        dev += [strided(dirty(plain.packed(q), c), None, shift, 0x77), strided(s, None, shift, 0xFF)]
    rc, size = tuna.tuna_moe_few_workspace(t, h, f, e, k)
    ok(rc)
    ws = torch.full((size + 16,), 0xFF, dtype=U8, device=DEV)    # NaN where nothing is written
    out = torch.full((t, h + 1), 9.0, dtype=TYPES[dtype], device=DEV)
    dx, dl = strided(x, h + (8 if h % 8 == 0 else 1)), strided(logits, e + 2)
    for _ in range(2):
        ok(tuna.tuna_moe_few(dx, dx.stride(0), t, h, dl, CODE[lt], e + 2, e, k, tuna.TUNA_ROUTE_RENORM if renorm else 0, *dev, f, tuna.TUNA_F4,
                             tuna.TUNA_SCALE_E8, out, CODE[dtype], h + 1, ws, size))
    torch.cuda.synchronize()
    assert bool((ws[size:] == 0xFF).all()) and bool((out[:, h:] == 9.0).all())
    exact, size = moe_plain.few(x, logits, k, renorm, *vals)
    # an activation: sums of `h` terms twice, relative to the magnitudes added, which are at most some sqrt(h) times the sum; kept in two bf16 parts
    # (2^-16); then sums of f terms: an error of 2^-13 of the magnitudes that the second product adds is far above all of them
    assert bool(((out[:, :h].cpu().double() - exact).abs() <= 2.0 ** -13 * size + rounding(dtype) * exact.abs() + 1e-30).all())


@pytest.mark.parametrize("t,h,f,e,k", [(1, 128, 64, 8, 2), (1, 256, 100, 60, 4), (2, 300, 48, 5, 5), (7, 384, 144, 16, 1), (17, 520, 72, 12, 4), (64, 256, 128, 8, 3),
                                       (33, 136, 40, 100, 8), (64, 128, 32, 3, 2), (5, 1040, 1040, 4, 2), (3, 160, 224, 6, 2), (9, 2880, 352, 4, 1), (1, 1, 1, 1, 1),
                                       (1, 2048, 1024, 16, 4), (40, 1024, 512, 32, 4), (6, 640, 416, 8, 3), (50, 768, 384, 16, 4), (30, 896, 640, 20, 4),
                                       (1, 1152, 928, 7, 3)])
def test_few(t, h, f, e, k):
    few(t, h, f, e, k, renorm=t % 2 == 0)


def test_few_types_and_alignment():
    few(9, 200, 88, 10, 3, dtype="f32", lt="bf16")
    few(9, 256, 96, 10, 3, dtype="f32", shift=1)
    few(9, 201, 83, 10, 3)
    few(1, 31, 63, 10, 3)                                        # whole sixteens of bytes, whose last half is behind the end


@pytest.mark.parametrize("renorm", [False, True])
def test_few_masks(renorm):
    l = torch.randn(20, 12, generator=gen(8))
    l[0] = -math.inf
    l[1] = math.nan
    l[2, 1:] = -math.inf
    l[3, ::2] = -math.inf
    l[4, 3] = math.inf
    l[5] = 1.0
    few(20, 160, 64, 12, 4, renorm, logits=l)
    few(20, 160, 64, 12, 4, renorm, logits=torch.full((20, 12), -math.inf))
