"""The types that kge_matmul_quantized takes for its output: fp32, bf16, and bf16 with fp32 sums (host only: no rows, or refused)."""
import ctypes as C

import pytest

import paper_2211_12281_amd.binding as b


@pytest.mark.parametrize("dtype,want", [(0, 0), (1, 0), (b.KGE_FP32_SUMS | 1, 0), (b.KGE_FP32_SUMS, -1), (b.KGE_FP32_SUMS | 2, -1), (2, -1), (-1, -1), (2 * b.KGE_FP32_SUMS | 1, -1)])
def test_output_types(dtype, want):
    q = b.KgeQuantizedT(0, 0, 0, 300, None, 384, None, 4)
    assert b.load().kge_matmul_quantized(C.byref(q), None, 0, C.byref(q), 0, None, dtype, 0, None, 0, None) == want
