"""Products in 4 bits of more than eight stages of 128 and more than a round of small tiles: the forms of 256 x 256 and 128 x 256.  References and tolerances are those of the
other forms' tests."""
import pytest
import torch

import paper_2411_02581_amd as tuna
from test_gpu_fp4_tiles import CODE, DEV, TYPES, by_columns, check, memory_is_given_back, ok, product, wide  # noqa: F401

pytestmark = pytest.mark.gpu

LENGTHS = [1024, 1025, 1026, 1039, 1055, 1056, 1057, 1087, 1096, 1151, 1152, 1153, 1168, 1196, 1279, 1280, 1281, 1296, 1408, 1409, 1441, 1536, 1663, 1664, 1919, 2047, 2048]


@pytest.mark.parametrize("k", LENGTHS)
def test_tiles_of_256_of_every_length(k):
    product(4100, 4110, k, [0, 4100], "f32" if k % 2 else "bf16")


@pytest.mark.parametrize("k", LENGTHS)
def test_tiles_of_128_by_256_of_every_length(k):
    product(2100, 2200, k, [0, 2100], "bf16" if k % 2 else "f32")


@pytest.mark.parametrize("k", LENGTHS)
def test_tiles_of_128_of_every_length(k):
    """Few of them, and long."""
    product(1100, 1030, k, [0, 1100], "bf16" if k % 3 else "f32")


@pytest.mark.parametrize("m,n", [(2100, 2200), (4100, 4110)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("more,shift", [(0, 0), (16, 3), (48, 8), (16, 1)])
def test_strides_and_results_of_any_alignment(m, n, dtype, more, shift):
    product(m + 1, n + 1, 1120, [0, m + 1], dtype, 60, more, shift)


@pytest.mark.parametrize("bounds", [[0, 5, 5, 1140, 3300, 4100], [3, 300, 2900, 4095], [0] + [600 + 37 * g for g in range(12)] + [4100], [0, 0, 0, 4100]])
@pytest.mark.parametrize("n", [4110, 1300])
def test_ragged_groups(bounds, n):
    product(bounds[-1] + (2 if bounds[0] else 0), n, 1200, bounds, "bf16")


@pytest.mark.parametrize("split", [[0, 1500], [0, 1, 2700], [5, 1300, 3900, 3900, 6000], [0, 129, 2600, 5000, 5130], [0, 2000, 2128, 4400]])
@pytest.mark.parametrize("n,k", [(2100, 2200), (4110, 4100)])
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
        blocks = -(-(split[i + 1] - split[i]) // 128)
        if blocks == 0:
            assert bool((dw[i, :, :k] == 0).all())
            continue
        part = slice(at * 64, (at + blocks) * 64), slice(at * 4, (at + blocks) * 4)
        check(dw[i, :, :k], wide(a[:, part[0]], sa[:, part[1]], blocks * 128), wide(b[:, part[0]], sb[:, part[1]], blocks * 128), dtype)
        at += blocks
