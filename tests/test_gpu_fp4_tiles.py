"""Products in 4 bits in the large forms, in tiles of 256 x 256 and 128 x 256: rows of values and of scales start on 16 bytes, there is more than a round of small tiles.
The reference is computed on the GPU in 64 bits from the definition."""
import pytest
import torch

import paper_2411_02581_amd as tuna

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CODE = {"f32": tuna.TUNA_F32, "bf16": tuna.TUNA_BF16}
EPS = 2.0 ** -24
U8 = torch.uint8


@pytest.fixture(scope="module", autouse=True)
def memory_is_given_back():
    yield
    torch.cuda.empty_cache()


def ok(rc):
    assert rc == tuna.TUNA_OK, tuna.tuna_strerror(rc)


def up(n, to):
    return -(-n // to) * to


def wide(q, s, n):
    """Packed rows of n values (and what is behind them) times their scales, in 64 bits."""
    c = torch.stack([q & 15, q >> 4], -1).flatten(-2)[..., :n].long()
    v = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=DEV)
    v = torch.cat([v, -v])[c]
    p = torch.where(s == 255, torch.nan, torch.exp2(s.double() - 127))
    return v * p.repeat_interleave(32, -1)[..., :n]


def operand(rows, k, seed, spread=8, more=0):
    """Rows of k random values on 16 bytes; behind a row's end there are values, and scales that are NaN."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    nb, ld = -(-k // 32), up(-(-k // 2), 16) + more
    q = torch.randint(0, 256, (rows, ld), generator=g, device=DEV, dtype=U8)
    s = torch.full((rows, up(nb, 16) + more), 255, dtype=U8, device=DEV)
    s[:, :nb] = torch.randint(127 - spread, 127 + spread, (rows, nb), generator=g, device=DEV, dtype=U8)
    return q, s


def check(got, a, b, dtype):
    """A step of 64 products and the sum so far are added to within 2^-23 of their magnitudes (and the result is rounded once)."""
    exact, size = a @ b.t(), a.abs() @ b.abs().t()
    room = (-(-a.shape[1] // 64) + 4) * 2 * EPS * size + (2.0 ** -8 if dtype == "bf16" else EPS) * exact.abs() + 1e-37
    assert bool(((got.double() - exact).abs() <= room).all())


def product(m, n, k, bounds, dtype, spread=8, more=0, shift=0):
    groups = len(bounds) - 1
    x, xs = operand(m, k, 1, spread, more)
    w, ws = operand(groups * n, k, 2, spread, more)
    y = torch.full((m, n + shift), 9.0, dtype=TYPES[dtype], device=DEV)
    rows = torch.tensor(bounds, dtype=torch.int32, device=DEV) if groups > 1 else None
    ld, ls = x.shape[1], xs.shape[1]
    ok(tuna.tuna_fp4_matmul(x, ld, xs, ls, w, ld, n * ld, ws, ls, n * ls, rows, groups, y, CODE[dtype], n + shift, m, n, k))
    a = wide(x, xs, k)
    for g in range(groups):
        i, j = bounds[g], bounds[g + 1]
        check(y[i:j, :n], a[i:j], wide(w[g * n:(g + 1) * n], ws[g * n:(g + 1) * n], k), dtype)
    assert bool((y[:, n:] == 9.0).all()) and bool((y[bounds[-1]:] == 9.0).all()) and bool((y[:bounds[0]] == 9.0).all())


LENGTHS = [128, 129, 130, 143, 159, 160, 161, 191, 200, 255, 256, 257, 272, 300, 383, 384, 400, 511, 512, 513, 545, 640, 767, 768, 1000, 1023, 1024, 1040, 1500, 2049, 2880]


@pytest.mark.parametrize("k", LENGTHS)
def test_tiles_of_256_of_every_length(k):
    """Rows that end inside a sixteen of bytes, a block, a stage and a run of four stages."""
    product(4100, 4110, k, [0, 4100], "f32" if k % 2 else "bf16")


@pytest.mark.parametrize("k", LENGTHS)
def test_tiles_of_128_of_every_length(k):
    product(1100, 1030, k, [0, 1100], "bf16" if k % 2 else "f32")


@pytest.mark.parametrize("m,n", [(1100, 1030), (4100, 4110)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("more,shift", [(0, 0), (16, 3), (48, 8), (16, 1)])
def test_strides_and_results_of_any_alignment(m, n, dtype, more, shift):
    product(m, n, 352, [0, m], dtype, 60, more, shift)
    product(m + 1, n + 1, 352, [0, m + 1], dtype, 8, more, shift)


@pytest.mark.parametrize("bounds", [[0, 4100, 4100], [0, 5, 5, 1140, 3300, 4100], [3, 300, 2900, 4095], [0] + [600 + 37 * g for g in range(12)] + [4100],
                                    [0, 0, 0, 4100], [0, 256, 512, 768, 1024, 4096, 4100]])
@pytest.mark.parametrize("n,k", [(4110, 400), (2100, 1111)])
def test_ragged_groups_in_tiles_of_256(bounds, n, k):
    product(bounds[-1] + (2 if bounds[0] else 0), n, k, bounds, "bf16")


@pytest.mark.parametrize("groups", [20, 65, 130])
def test_many_ragged_groups(groups):
    bounds = [0]
    for g in range(groups):
        bounds.append(bounds[-1] + (g * 53) % 97)
    product(bounds[-1], 300, 700, bounds, "bf16")
    product(bounds[-1], 1030, 260, bounds, "f32")


@pytest.mark.parametrize("m,n", [(1100, 1030), (4100, 4110)])
def test_not_a_number_stays_in_its_row(m, n):
    k = 1200
    x, xs = operand(m, k, 3)
    w, ws = operand(n, k, 4)
    xs[m // 2, 3], ws[n - 1, 37] = 255, 255
    y = torch.empty(m, n, device=DEV)
    ok(tuna.tuna_fp4_matmul(x, x.shape[1], xs, xs.shape[1], w, x.shape[1], 0, ws, xs.shape[1], 0, None, 1, y, 0, n, m, n, k))
    want = torch.zeros(m, n, dtype=torch.bool, device=DEV)
    want[m // 2], want[:, n - 1] = True, True
    assert torch.equal(y.isnan(), want)


def test_group_bounds_are_held_inside():
    """Bounds outside [0, m] and falling ones in the large form: a bound counts as the largest of all up to it."""
    m, n, k, bounds = 4000, 4110, 256, [-5, 1000, 20, 2500, 100000]
    x, xs = operand(m, k, 5)
    w, ws = operand(4 * n, k, 6)
    y = torch.full((m, n), 9.0, device=DEV)
    ld, ls = x.shape[1], xs.shape[1]
    ok(tuna.tuna_fp4_matmul(x, ld, xs, ls, w, ld, n * ld, ws, ls, n * ls, torch.tensor(bounds, dtype=torch.int32, device=DEV), 4, y, 0, n, m, n, k))
    a = wide(x, xs, k)
    for g, (i, j) in enumerate([(0, 1000), (1000, 1000), (1000, 2500), (2500, 4000)]):
        check(y[i:j], a[i:j], wide(w[g * n:(g + 1) * n], ws[g * n:(g + 1) * n], k), "f32")


# groups that start at every remainder of four blocks of 128, empty ones, of one row, of one block, longer than a run of stages
SPLITS = [[0, 1, 130, 131, 600, 600, 2000], [0, 129, 300, 600, 1200, 2500], [0, 128, 256, 384, 512, 1024, 1700], [0, 2000], [0, 50, 100, 150, 200, 1000],
          [7, 140, 900, 1800]]


def by_columns(x, rows, groups, bounds, dtype, code):
    c = x.shape[1]
    nb = up(x.shape[0], 128) // 128 + groups - 1
    q, s = torch.full((c, 64 * nb), 0x77, dtype=U8, device=DEV), torch.full((c, up(4 * nb, 16)), 255, dtype=U8, device=DEV)
    ok(tuna.tuna_fp4_quantize_columns(x, code, c, x.shape[0], c, bounds, groups, q, 64 * nb, s, s.shape[1]))
    return q, s


@pytest.mark.parametrize("split", SPLITS)
@pytest.mark.parametrize("n,k", [(2100, 2050), (520, 700)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_weights_gradient(split, n, k, dtype):
    rows, groups = split[-1], len(split) - 1
    g = torch.Generator(device=DEV).manual_seed(rows)
    dy, x = torch.randn(rows, n, generator=g, device=DEV).bfloat16(), torch.randn(rows, k, generator=g, device=DEV)
    bounds = torch.tensor(split, dtype=torch.int32, device=DEV) if groups > 1 else None
    (a, sa), (b, sb) = by_columns(dy, rows, groups, bounds, "bf16", 1), by_columns(x, rows, groups, bounds, "f32", 0)
    dw = torch.full((groups, n, k + 2), 9.0, dtype=TYPES[dtype], device=DEV)
    ok(tuna.tuna_fp4_matmul_grad_w(a, a.shape[1], sa, sa.shape[1], b, b.shape[1], sb, sb.shape[1], bounds, groups, dw, CODE[dtype], k + 2, n * (k + 2), rows, n, k))
    assert bool((dw[..., k:] == 9.0).all())
    at = 0
    for i in range(groups):
        n_blocks = up(split[i + 1] - split[i], 128) // 128
        if n_blocks == 0:
            assert bool((dw[i, :, :k] == 0).all())
            continue
        part = slice(at * 64, (at + n_blocks) * 64), slice(at * 4, (at + n_blocks) * 4)
        check(dw[i, :, :k], wide(a[:, part[0]], sa[:, part[1]], n_blocks * 128), wide(b[:, part[0]], sb[:, part[1]], n_blocks * 128), dtype)
        at += n_blocks


@pytest.mark.parametrize("m", [1, 15, 16, 17, 33, 48, 49, 64, 65, 128, 129, 200, 256, 257, 520])
@pytest.mark.parametrize("n,k", [(1040, 640), (2050, 1111)])
def test_rows_from_few_to_many(m, n, k):
    """On both sides of every limit between the forms."""
    product(m, n, k, [0, m], "bf16")
    product(m, n, k, [0, m], "f32")


@pytest.mark.parametrize("each", [1, 5, 15, 16, 17, 40])
def test_few_rows_of_many_groups(each):
    groups = 24
    bounds = [0]
    for g in range(groups):
        bounds.append(bounds[-1] + (each * 2 * (g % 7)) // 6)
    product(bounds[-1], 200, 900, bounds, "bf16")


# ------------------------------------------------------------------------------------------------ offsets beyond 32 bits


def test_weights_beyond_32_bits():
    groups, n, k, m = 70, 8192, 16384, 600                       # 64 MB of values a group: 4.7 GB
    w = torch.zeros(groups, n, k // 2, dtype=U8, device=DEV)
    ws = torch.full((groups, n, k // 32), 120, dtype=U8, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    w[-1] = torch.randint(0, 256, (n, k // 2), generator=g, device=DEV, dtype=U8)
    x, xs = operand(m, k, 7)
    b = wide(w[-1], ws[-1], k)
    for rows in (m, 40):                                         # tiles; few rows
        y = torch.zeros(rows, n, device=DEV)
        bounds = torch.tensor([0] * groups + [rows], dtype=torch.int32, device=DEV)
        ok(tuna.tuna_fp4_matmul(x, k // 2, xs, k // 32, w, k // 2, n * k // 2, ws, k // 32, n * k // 32, bounds, groups, y, 0, n, rows, n, k))
        check(y, wide(x, xs, k)[:rows], b, "f32")


def test_rows_beyond_32_bits():
    """Records whose offsets pass 2^32 bytes, packed and read back, and multiplied."""
    cols, rows, size = 4096, 1200000, 4096
    x = torch.randn(6, cols, generator=torch.Generator().manual_seed(1)).bfloat16().to(DEV)
    rec = torch.zeros(rows, size, dtype=U8, device=DEV)
    slots = torch.tensor([0, 5, 524287, 1048576, 1048577, rows - 1], dtype=torch.int32, device=DEV)
    ok(tuna.tuna_fp4_quantize(x, 1, cols, 6, cols, 0, slots, 1, rows, rec, size, rec[:, 2048:], size))
    q, s = torch.empty(6, 2048, dtype=U8, device=DEV), torch.empty(6, 128, dtype=U8, device=DEV)
    ok(tuna.tuna_fp4_quantize(x, 1, cols, 6, cols, 0, None, 1, 6, q, 2048, s, 128))
    assert torch.equal(rec[slots.long(), :2048], q) and torch.equal(rec[slots.long(), 2048:2176], s)
    assert int((rec[:, 2048:2176] != 0).any(1).sum()) == 6
    last = rec[rows - 1024:]
    back = torch.empty(1024, cols, device=DEV)
    ok(tuna.tuna_fp4_dequantize(last, size, last[:, 2048:], size, 1024, cols, back, 0, cols))
    assert torch.equal(back[-1].double(), wide(q, s, cols)[5])
    y = torch.full((rows, 32), 9.0, device=DEV)
    w, ws = operand(32, cols, 9)
    ok(tuna.tuna_fp4_matmul(rec, size, rec[:, 2048:], size, w, cols // 2, 0, ws, 128, 0, None, 1, y, 0, 32, rows, 32, cols))
    check(y[slots.long()], wide(q, s, cols), wide(w, ws, cols), "f32")
    assert int((y != 0).any(1).sum()) == 6
