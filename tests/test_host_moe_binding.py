"""Which tensors the functions of tuna_moe.h take from Python: their types have to be those that the call names.  Tensors are stand-ins; every call that
passes the check is refused by the library or has nothing to do."""
import pytest
import torch

import paper_2411_02581_amd as tuna

A = 0x7000000000                                                 # an address that is never used


class Tensor:
    is_cuda = True
    shape = (4, 256)

    def __init__(self, dtype):
        self.dtype = dtype

    def element_size(self):
        return torch.empty(0, dtype=self.dtype).element_size()

    def stride(self):
        return (256, 1)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return A


F32, BF16, F8, E8, U8 = torch.float32, torch.bfloat16, torch.float8_e4m3fn, torch.float8_e8m0fnu, torch.uint8
VALUES = {tuna.TUNA_F32: [F32], tuna.TUNA_BF16: [BF16], tuna.TUNA_F8: [F8, U8]}
SCALES = {tuna.TUNA_SCALE_F32: [F32], tuna.TUNA_SCALE_E8: [U8, E8]}
ALL = [F32, BF16, F8, E8, U8, torch.float16, torch.int32, torch.int16, torch.int8, torch.bool, torch.float64, torch.float8_e5m2, torch.float8_e4m3fnuz]

# calls with nothing to do; which arguments are of which type: (position, names of the position of the type's code)
ROUTE = ("tuna_moe_route_grad", [A, 1, 8, 0, 8, 2, 0, A, A, A, A, 8], {0: 1, 10: 1}, {})
QUANTISE = ("tuna_fp8_quantize", [A, 1, 256, 0, 256, 0, None, 1, 0, A, 256, A, 2, 0], {0: 1, 9: tuna.TUNA_F8 + 100}, {11: 13})
COLUMNS = ("tuna_fp8_quantize_columns", [A, 1, 256, 0, 256, None, 1, A, 256, A, 2, 0], {0: 1, 7: tuna.TUNA_F8 + 100}, {9: 11})
SWIGLU = ("tuna_moe_swiglu_grad", [A, 1, 256, A, 128, 0, 128, A, 256], {0: 1, 3: 1, 7: 1}, {})
MATMUL = ("tuna_fp8_matmul", [A, 256, A, 2, A, 256, 0, A, 2, 0, 0, None, 1, A, 1, 256, 0, 256, 256], {0: 102, 4: 102, 13: 14}, {2: 10, 7: 10})
GRAD_W = ("tuna_fp8_matmul_grad_w", [A, 256, A, 2, A, 256, A, 2, 0, None, 1, A, 1, 256, 0, 0, 0, 256], {0: 102, 4: 102, 11: 12}, {2: 8, 6: 8})
COMBINE = ("tuna_moe_combine", [A, 1, 256, 4, A, A, 0, 2, 256, A, 0, 256], {0: 1, 9: 10}, {})
COMBINE_GRAD = ("tuna_moe_combine_grad", [A, 1, 256, A, 0, 256, 4, A, A, 0, 2, 256, A, 256, A], {0: 1, 3: 4, 12: 4}, {})
FEW = ("tuna_moe_few", [A, 256, 0, 256, A, 1, 8, 8, 2, 0, A, A, A, A, 256, 2, 0, A, 1, 256, A, 1 << 30], {0: 101, 4: 5, 10: 15, 12: 15, 17: 18}, {11: 16, 13: 16})


@pytest.mark.parametrize("name,args,values,scales", [ROUTE, QUANTISE, COLUMNS, SWIGLU, MATMUL, GRAD_W, COMBINE, COMBINE_GRAD, FEW], ids=lambda v: v if isinstance(v, str) else "")
def test_tensors_have_the_types_that_the_call_names(name, args, values, scales):
    call = lambda a: getattr(tuna, name)(*a, stream=0)  # noqa: E731
    assert call(args) == tuna.TUNA_OK
    for where, table in ((values, VALUES), (scales, SCALES)):
        for at, code in where.items():
            fixed = code >= 100                                  # the type is the argument's own
            for kind in ([code - 100] if fixed else [c for c in table if (name, at) != ("tuna_moe_few", 4) or c != tuna.TUNA_F8]):
                if not fixed and table is VALUES and name != "tuna_moe_few" and kind == tuna.TUNA_F8:
                    continue                                     # not a type of these arguments
                for dtype in ALL:
                    a = list(args)
                    a[at] = Tensor(dtype)
                    if not fixed:
                        a[code] = kind
                    if dtype in table[kind]:
                        call(a)
                    else:
                        with pytest.raises(TypeError):
                            call(a)


def test_an_unknown_type_is_the_library_s_to_refuse():
    for code in (-1, 3, 7):
        assert tuna.tuna_moe_swiglu_grad(Tensor(F32), code, 256, Tensor(F32), 128, 4, 128, Tensor(F32), 256, stream=0) == tuna.TUNA_ERR_ARG
        assert tuna.tuna_fp8_quantize(Tensor(F32), tuna.TUNA_F32, 256, 4, 256, 0, None, 1, 4, Tensor(U8), 256, Tensor(F32), 2, code, stream=0) == tuna.TUNA_ERR_ARG


def test_index_and_weight_arrays():
    for at, good in ((7, torch.int32), (8, F32), (9, F32)):
        for dtype in ALL:
            a = list(ROUTE[1])
            a[at] = Tensor(dtype)
            if dtype == good:
                tuna.tuna_moe_route_grad(*a, stream=0)
            else:
                with pytest.raises(TypeError):
                    tuna.tuna_moe_route_grad(*a, stream=0)


def test_the_last_axis_is_dense_and_the_rows_may_lie_apart():
    def with_steps(shape, steps):
        v = Tensor(BF16)
        v.shape, v.stride, v.is_contiguous = shape, lambda: steps, lambda: False
        return v

    call = lambda v: tuna.tuna_moe_swiglu_grad(v, 1, 300, A, 128, 0, 128, A, 256, stream=0)  # noqa: E731
    assert call(with_steps((4, 256), (300, 1))) == tuna.TUNA_OK
    assert call(with_steps((4, 1), (300, 7))) == tuna.TUNA_OK
    assert call(with_steps((2, 4, 256), (9000, 300, 1))) == tuna.TUNA_OK
    with pytest.raises(TypeError):
        call(with_steps((4, 256), (1, 4)))
