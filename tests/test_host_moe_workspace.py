"""Workspaces of include/tuna_moe.h: what is enough for a batch is enough for every smaller one."""
import pytest

import paper_2411_02581_amd as tuna

A = 0x7000000000                                                 # an address that is never used


def size_of(n, e, k, plan):
    rc, size = tuna.tuna_moe_route_workspace(n, e, k, plan)
    assert rc == tuna.TUNA_OK
    return size


@pytest.mark.parametrize("e,k", [(1, 1), (8, 2), (256, 8), (1024, 16)])
@pytest.mark.parametrize("plan", [False, True])
def test_the_router_s_never_falls_as_tokens_grow(e, k, plan):
    ends = [64 << i for i in range(0, 20)] + [65536 * i for i in range(1, 40)]
    counts = sorted({max(0, n + d) for n in ends for d in (-65, -64, -1, 0, 1, 63, 64)})
    sizes = [size_of(n, e, k, plan) for n in counts]
    for a, b, n in zip(sizes, sizes[1:], counts):
        assert a <= b, n


def test_a_batch_runs_in_a_larger_one_s_workspace():
    """65536 tokens in what 65537 need."""
    size = size_of(65537, 256, 8, False)
    args = [A, tuna.TUNA_F32, 256, 65536, 256, 8, 0, A, A, A, A, 1, None, None, None, None]
    assert tuna.tuna_moe_route(*args, A, size_of(65536, 256, 8, False) - 1, stream=0) == tuna.TUNA_ERR_WORKSPACE_TOO_SMALL
    assert size >= size_of(65536, 256, 8, False)


@pytest.mark.parametrize("h,f,e,k", [(128, 64, 8, 2), (4096, 1536, 128, 8), (100, 1, 1, 1)])
def test_the_layer_s_never_falls_as_tokens_grow(h, f, e, k):
    sizes = [tuna.tuna_moe_few_workspace(n, h, f, e, k)[1] for n in range(tuna.TUNA_MOE_FEW_TOKENS + 1)]
    assert sizes == sorted(sizes)
