"""examples/expert_parallel.py without a GPU: what it refuses before it calls anything that writes."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import expert_parallel  # noqa: E402

E, H, F, K, MOST = 6, 160, 48, 2, 10


@pytest.fixture(scope="module")
def layer():
    g = torch.Generator().manual_seed(0)
    return expert_parallel.ExpertParallel(torch.randn(E, 2 * F, H, generator=g), torch.randn(E, H, F, generator=g), K, MOST)


def inputs(tokens, hidden=H, experts=E, dtype=torch.bfloat16):
    return torch.zeros(tokens, hidden, dtype=dtype), torch.zeros(tokens, experts)


@pytest.mark.parametrize("bad", [inputs(MOST + 1), inputs(4000), inputs(4, H - 1), inputs(4, experts=E + 1), inputs(4, dtype=torch.float32),
                                 (inputs(4)[0], inputs(5)[1]), (inputs(4)[0], inputs(4)[1].bfloat16()), (inputs(8)[0][::2], inputs(4)[1]),
                                 (inputs(4, 2 * H)[0][:, :H], inputs(4)[1]), (inputs(4)[0], inputs(4, experts=2 * E)[1][:, :E])])
@pytest.mark.parametrize("way", ["__call__", "step"])
def test_inputs_that_do_not_fit_its_buffers_are_refused(layer, bad, way):
    """Its buffers' sizes and the distances of rows that it names hold for dense inputs of up to max_tokens tokens."""
    with pytest.raises(ValueError):
        getattr(layer, way)(*bad)


def test_the_step_has_its_own_most():
    g = torch.Generator().manual_seed(0)
    big = expert_parallel.ExpertParallel(torch.randn(E, 2 * F, H, generator=g), torch.randn(E, H, F, generator=g), K, 200)
    with pytest.raises(ValueError):
        big.step(*inputs(65))
