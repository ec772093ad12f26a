"""The types of tensors where torch has no type of two 4-bit values.  Tensors are stand-ins; every call has nothing to do."""
import pytest
import torch

import paper_2411_02581_amd as tuna
from paper_2411_02581_amd import binding
from test_host_moe_binding import A, BF16, F32, U8, Tensor


@pytest.fixture
def torch_without_4_bits(monkeypatch):
    monkeypatch.delattr(torch, "float4_e2m1fn_x2", raising=False)
    kept = [dict(t) for t in (binding._value_types, binding._scale_types)]
    for t in (binding._value_types, binding._scale_types):
        t.clear()
    yield
    for t, k in zip((binding._value_types, binding._scale_types), kept):
        t.clear()
        t.update(k)


def test_calls_need_no_type_of_4_bits(torch_without_4_bits):
    assert tuna.tuna_moe_swiglu_grad(Tensor(F32), tuna.TUNA_F32, 256, Tensor(F32), 128, 0, 128, Tensor(F32), 256, stream=0) == tuna.TUNA_OK
    assert tuna.tuna_fp8_quantize(Tensor(BF16), tuna.TUNA_BF16, 256, 0, 256, 0, None, 1, 0, Tensor(U8), 256, Tensor(U8), 2, tuna.TUNA_SCALE_E8, stream=0) == tuna.TUNA_OK
    assert tuna.tuna_fp4_quantize(Tensor(BF16), tuna.TUNA_BF16, 256, 0, 256, 0, None, 1, 0, Tensor(U8), 128, Tensor(U8), 8, stream=0) == tuna.TUNA_OK
    with pytest.raises(TypeError):
        tuna.tuna_fp4_quantize(A, tuna.TUNA_BF16, 256, 0, 256, 0, None, 1, 0, Tensor(BF16), 128, A, 8, stream=0)
