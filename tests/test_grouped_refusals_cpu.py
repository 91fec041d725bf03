"""Calls of the grouped products and the 4-bit experts that are refused before anything is launched, and which kernel takes which form.
Nothing here reaches a GPU: addresses are never dereferenced, tensors lie on the host."""
import ctypes as C

import pytest
import torch

import paper_2508_17624_amd as ew

ONE = C.c_void_p(256)   # never dereferenced
INVALID, UNSUPPORTED = -1, -6


def rows_on_host():
    """(x, dy, counts, offsets) of two tokens, one row each, on the host: any call that gets past the checks of types and sizes ends at the
    check of devices."""
    x = torch.zeros(2, 64, dtype=torch.bfloat16)
    return x, x.clone(), torch.zeros(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)


@pytest.mark.parametrize("dtype", [torch.float16, torch.int16, torch.uint8, torch.float64, torch.int32])
def test_weight_gradients_of_other_types_are_refused(dtype):
    """The kernels write float32 or bfloat16: into 2-byte tensors of another type they would put wrong numbers, and past the end of 1-byte ones."""
    x, dy, c, off = rows_on_host()
    with pytest.raises(TypeError, match="unsupported dtype"):
        ew.moe_grouped_ffn_backward(x, dy, 1, 32, 3, c, off, None, 0, 0, dw_dtype=dtype)
    out = torch.zeros(3, 64, 64, dtype=dtype)
    with pytest.raises(TypeError, match="unsupported dtype"):
        ew.moe_grouped_gemm_wgrad(dy, x, 1, 3, c, off, None, dtype=dtype, out=out)
