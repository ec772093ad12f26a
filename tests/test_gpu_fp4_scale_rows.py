"""Rows of scales in 4 bits that start on 16 bytes, as the tiles of the products want them: the example's, and those of weights by columns for the gradient of x."""
import os
import sys

import pytest
import torch

import fp4_plain as plain
import moe_plain
import paper_2411_02581_amd as tuna
from test_gpu_fp4_tiles import DEV, U8, check, ok, operand, up, wide

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module", autouse=True)
def memory_is_given_back():
    yield
    torch.cuda.empty_cache()


def starts(t):
    """Whether every row of a tensor starts on 16 bytes."""
    return t.data_ptr() % 16 == 0 and all(s % 16 == 0 for s in t.stride()[:-1])


@pytest.mark.parametrize("tokens,hidden,inner,experts,k", [(700, 2880, 1408, 4, 2), (900, 2048, 1792, 4, 3), (40, 1312, 352, 4, 2)])
def test_the_layers_rows_of_scales_start_on_16_bytes(tokens, hidden, inner, experts, k):
    import expert_parallel
    layer, x, logits, out, step = expert_parallel.main(tokens, hidden, inner, experts, k, 2, 4)
    for s, p, c in ((layer.s1, layer.p1, hidden), (layer.s2, layer.p2, inner)):
        assert s.is_contiguous() and s.shape[2] == plain.blocks(c) and torch.equal(p[..., :s.shape[2]], s) and starts(p)
    assert starts(layer.qs) and starts(layer.recv[:, layer.h_bytes:])
    _, names, weights = moe_plain.route(logits.cpu(), k, True)
    names, weights = names.to(DEV), weights.to(DEV)
    w1, w2 = wide(layer.w1, layer.s1, hidden), wide(layer.w2, layer.s2, inner)
    held = lambda v: plain.held(v.cpu()).to(DEV)  # noqa: E731
    xq, want = held(x), torch.zeros(tokens, hidden, dtype=torch.float64, device=DEV)
    for e in range(experts):
        t, j = (names == e).nonzero(as_tuple=True)
        g, u = (xq[t] @ w1[e].t()).bfloat16().double().chunk(2, -1)
        y = (held(g * torch.sigmoid(g) * u) @ w2[e].t()).bfloat16().double()
        want.index_add_(0, t, weights[t, j][:, None] * y)
    # as in test_gpu_fp4_layer.py: values at a rounding's edge, and the last roundings
    assert (out.double() - want).norm() <= 0.02 * want.norm()


@pytest.mark.parametrize("m,n,k,groups", [(4100, 2816, 4110, 3), (2050, 1100, 2100, 2), (1040, 1408, 1030, 3)])
def test_weights_by_columns_a_group_at_a_time(m, n, k, groups):
    """Each group's values and scales at a distance of the caller's choice, for tuna_fp4_matmul: the same values as one call leaves."""
    g = torch.Generator(device=DEV).manual_seed(m)
    w, blocks = torch.randn(groups * n, k, generator=g, device=DEV), up(n, 128) // 128
    at = torch.arange(groups + 1, dtype=torch.int32, device=DEV) * n
    nb = up(groups * n, 128) // 128 + groups - 1
    one, one_s = torch.zeros(k, 64 * nb, dtype=U8, device=DEV), torch.zeros(k, 4 * nb, dtype=U8, device=DEV)
    ok(tuna.tuna_fp4_quantize_columns(w, 0, k, groups * n, k, at, groups, one, 64 * nb, one_s, 4 * nb))
    per, per_s = 64 * blocks, up(4 * blocks, 16)
    q, s = torch.zeros(k, groups * per, dtype=U8, device=DEV), torch.zeros(k, groups * per_s, dtype=U8, device=DEV)
    for i in range(groups):
        ok(tuna.tuna_fp4_quantize_columns(w[i * n:(i + 1) * n], 0, k, n, k, None, 1, q[:, i * per:], q.stride(0), s[:, i * per_s:], s.stride(0)))
        assert torch.equal(q[:, i * per:(i + 1) * per], one[:, i * per:(i + 1) * per])
        assert torch.equal(s[:, i * per_s:i * per_s + 4 * blocks], one_s[:, 4 * i * blocks:4 * (i + 1) * blocks])
    dy, ds = operand(m, n, 9)
    bounds, dx = [m * i // groups for i in range(groups + 1)], torch.full((m, k), 9.0, device=DEV)
    rows = torch.tensor(bounds, dtype=torch.int32, device=DEV)
    ok(tuna.tuna_fp4_matmul(dy, dy.shape[1], ds, ds.shape[1], q, q.stride(0), per, s, s.stride(0), per_s, rows, groups, dx, 0, k, m, k, n))
    a = wide(dy, ds, n)
    for i in range(groups):
        check(dx[bounds[i]:bounds[i + 1]], a[bounds[i]:bounds[i + 1]], wide(q[:, i * per:(i + 1) * per], s[:, i * per_s:i * per_s + 4 * blocks], 128 * blocks)[:, :n], "f32")
