"""Every form of the products in 4 bits at sizes that it is known to run (fp4_forms.py; test_host_fp4_forms.py holds them to that), against 64 bits on the GPU."""
import pytest
import torch

import fp4_forms as forms
import paper_2411_02581_amd as tuna
from test_gpu_fp4_tiles import CODE, DEV, TYPES, U8, by_columns, check, ok, operand, product, up, wide

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def memory_is_given_back():
    yield
    torch.cuda.empty_cache()


def even(m, groups):
    return [m * g // groups for g in range(groups + 1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("form", list(forms.SIZES))
def test_the_form(form, dtype):
    s = forms.SIZES[form]
    product(s["m"], s["n"], s["k"], even(s["m"], s["groups"]), dtype)


@pytest.mark.parametrize("k", forms.LENGTHS)
@pytest.mark.parametrize("form", forms.LARGE[:2])
def test_every_length(form, k):
    s = forms.SIZES[form]
    product(s["m"], s["n"], k, [0, s["m"]], "f32" if k % 2 else "bf16")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("more,shift", [(0, 0), (16, 3), (48, 8), (16, 1)])
@pytest.mark.parametrize("form", forms.LARGE[:2])
def test_strides_and_results_of_any_alignment(form, more, shift, dtype):
    s = forms.SIZES[form]
    product(s["m"], s["n"], 1376, [0, s["m"]], dtype, 60, more, shift)
    product(s["m"] + 1, s["n"] + 1, 1376, [0, s["m"] + 1], dtype, 8, more, shift)


@pytest.mark.parametrize("form,bounds", forms.RAGGED)
def test_ragged_groups(form, bounds):
    product(bounds[-1] + (2 if bounds[0] else 0), forms.SIZES[form]["n"], 1111, bounds, "bf16")


@pytest.mark.parametrize("form", list(forms.BOUNDS))
def test_group_bounds_are_held_inside(form):
    m, bounds, count_as = forms.BOUNDS[form]
    n, k = forms.SIZES[form]["n"], 1100
    x, xs = operand(m, k, 5)
    w, ws = operand(4 * n, k, 6)
    y = torch.full((m, n), 9.0, dtype=torch.bfloat16, device=DEV)
    ld, ls = x.shape[1], xs.shape[1]
    ok(tuna.tuna_fp4_matmul(x, ld, xs, ls, w, ld, n * ld, ws, ls, n * ls, torch.tensor(bounds, dtype=torch.int32, device=DEV), 4, y, 1, n, m, n, k))
    a = wide(x, xs, k)
    for g, (i, j) in enumerate(count_as):
        check(y[i:j], a[i:j], wide(w[g * n:(g + 1) * n], ws[g * n:(g + 1) * n], k), "bf16")


@pytest.mark.parametrize("form", list(forms.SIZES))
def test_not_a_number_stays_in_its_row(form):
    s = forms.SIZES[form]
    m, n, k, groups = s["m"], s["n"], s["k"], s["groups"]
    x, xs = operand(m, k, 3)
    w, ws = operand(groups * n, k, 4)
    xs[m // 2, 3], ws[groups * n - 1, 37] = 255, 255             # the last row of the last group's weights
    bounds = even(m, groups)
    y = torch.empty(m, n, device=DEV)
    rows = torch.tensor(bounds, dtype=torch.int32, device=DEV) if groups > 1 else None
    ok(tuna.tuna_fp4_matmul(x, x.shape[1], xs, xs.shape[1], w, x.shape[1], n * x.shape[1], ws, xs.shape[1], n * xs.shape[1], rows, groups, y, 0, n, m, n, k))
    want = torch.zeros(m, n, dtype=torch.bool, device=DEV)
    want[m // 2], want[bounds[-2]:, n - 1] = True, True
    assert torch.equal(y.isnan(), want)


@pytest.mark.parametrize("form", list(forms.SIZES))
def test_scales_at_the_ends_of_their_range(form):
    """Powers of two from 2^-127 to 2^127 on one side, and such on the other that their products stay in the range of 32 bits."""
    s = forms.SIZES[form]
    m, n, k, groups = s["m"], s["n"], s["k"], s["groups"]
    x, xs = operand(m, k, 3)
    w, ws = operand(groups * n, k, 4)
    nb = -(-k // 32)
    g = torch.Generator(device=DEV).manual_seed(5)
    # block by block: x's scale is 2^(e - 127) and w's 2^(127 - e), give or take four
    e = torch.randint(4, 250, (nb,), generator=g, device=DEV)
    e[0], e[-1], e[nb // 2] = 0, 254, 1
    near = lambda r: torch.randint(-2, 3, (r, nb), generator=g, device=DEV)  # noqa: E731
    xs[:, :nb] = (e + near(m)).clamp(0, 254).to(U8)
    ws[:, :nb] = (254 - e + near(groups * n)).clamp(0, 254).to(U8)
    bounds = even(m, groups)
    y = torch.empty(m, n, device=DEV)
    rows = torch.tensor(bounds, dtype=torch.int32, device=DEV) if groups > 1 else None
    ok(tuna.tuna_fp4_matmul(x, x.shape[1], xs, xs.shape[1], w, x.shape[1], n * x.shape[1], ws, xs.shape[1], n * xs.shape[1], rows, groups, y, 0, n, m, n, k))
    a = wide(x, xs, k)
    for i in range(groups):
        check(y[bounds[i]:bounds[i + 1]], a[bounds[i]:bounds[i + 1]], wide(w[i * n:(i + 1) * n], ws[i * n:(i + 1) * n], k), "f32")


# ------------------------------------------------------------------------------------------------ the weights' gradient, and that of x, by columns


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("form,n,k,split", forms.GRADIENT)
def test_weights_gradient(form, n, k, split, dtype):
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
        count = up(split[i + 1] - split[i], 128) // 128
        if count == 0:
            assert bool((dw[i, :, :k] == 0).all())
            continue
        part = slice(at * 64, (at + count) * 64), slice(at * 4, (at + count) * 4)
        check(dw[i, :, :k], wide(a[:, part[0]], sa[:, part[1]], count * 128), wide(b[:, part[0]], sb[:, part[1]], count * 128), dtype)
        at += count


@pytest.mark.parametrize("m,n,k,groups", [(4100, 2048, 4110, 3), (2050, 1536, 2100, 2), (2050, 1408, 2100, 2), (4100, 1100, 2100, 3), (1040, 512, 1030, 3), (60, 1408, 1030, 4)])
def test_gradient_of_rows_with_weights_by_columns(m, n, k, groups):
    """dx = dy w, with w as tuna_fp4_quantize_columns leaves [groups * n, k] with the bounds 0, n, 2 n, ...: n of whole 512, whose groups' scales start on 16 bytes, and
    others."""
    g = torch.Generator(device=DEV).manual_seed(m)
    w, at = torch.randn(groups * n, k, generator=g, device=DEV), torch.arange(groups + 1, dtype=torch.int32, device=DEV) * n
    wt, st = by_columns(w, groups * n, groups, at, "f32", 0)
    dy, ds = operand(m, n, 9)
    per, bounds = up(n, 128), even(m, groups)
    dx = torch.full((m, k), 9.0, device=DEV)
    ok(tuna.tuna_fp4_matmul(dy, dy.shape[1], ds, ds.shape[1], wt, wt.shape[1], per // 2, st, st.shape[1], per // 32, torch.tensor(bounds, dtype=torch.int32, device=DEV), groups,
                            dx, 0, k, m, k, n))
    a = wide(dy, ds, n)
    for i in range(groups):
        q, s = wt[:, i * per // 2:(i + 1) * per // 2], st[:, i * per // 32:(i + 1) * per // 32]
        b = wide(q, s, per)[:, :n]
        # the values are those of w: off by half a step of e2m1, which is at most 2 times the scale
        assert bool(((b - w[i * n:(i + 1) * n].t().double()).abs() <= torch.exp2(s.double() - 127).repeat_interleave(32, 1)[:, :n]).all())
        check(dx[bounds[i]:bounds[i + 1]], a[bounds[i]:bounds[i + 1]], b, "f32")


# ------------------------------------------------------------------------------------------------ offsets beyond 32 bits


@pytest.mark.parametrize("form", list(forms.FAR_WEIGHTS))
def test_weights_beyond_32_bits(form):
    s = forms.FAR_WEIGHTS[form]
    m, n, k, groups = s["m"], s["n"], s["k"], s["groups"]
    w = torch.zeros(groups, n, k // 2, dtype=U8, device=DEV)
    ws = torch.full((groups, n, k // 32), 120, dtype=U8, device=DEV)
    assert (groups - 1) * n * k // 2 > 1 << 32
    w[-1] = torch.randint(0, 256, (n, k // 2), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV, dtype=U8)
    x, xs = operand(m, k, 7)
    y = torch.zeros(m, n, dtype=torch.bfloat16, device=DEV)
    bounds = torch.tensor([0] * groups + [m], dtype=torch.int32, device=DEV)
    ok(tuna.tuna_fp4_matmul(x, k // 2, xs, k // 32, w, k // 2, n * k // 2, ws, k // 32, n * k // 32, bounds, groups, y, 1, n, m, n, k))
    b = wide(w[-1], ws[-1], k)
    for rows in (slice(0, 300), slice(m - 300, m)):
        check(y[rows], wide(x[rows], xs[rows], k), b, "bf16")


@pytest.mark.parametrize("form", list(forms.FAR_ROWS))
def test_rows_beyond_32_bits(form):
    s, ld = forms.SIZES[form], forms.FAR_ROWS[form]
    m, n, k = s["m"], s["n"], s["k"]
    assert (m - 1) * ld > 1 << 32
    x, xs = operand(m, k, 7)
    w, ws = operand(n, k, 8)
    far = torch.empty(m * ld, dtype=U8, device=DEV)
    q, sc = far.view(m, ld)[:, :x.shape[1]], far.view(m, ld)[:, 4096:4096 + xs.shape[1]]
    q.copy_(x)
    sc.copy_(xs)                                                 # in the same records
    y = torch.full((m, n), 9.0, device=DEV)
    ok(tuna.tuna_fp4_matmul(q, ld, sc, ld, w, w.shape[1], 0, ws, ws.shape[1], 0, None, 1, y, 0, n, m, n, k))
    check(y, wide(x, xs, k), wide(w, ws, k), "f32")
