"""Ends of the ranges that the paged cache's entry points check before any GPU
work, on the CPU: sizes whose products pass 64 bits, empty batches, heads of no
elements."""
import ctypes
import os

import pytest
import torch

from paper_2607_01065_amd import gsrq as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libgsrq.so not built")


@pytest.mark.parametrize("T", [1 << 28, 1 << 30, 1 << 61, 1 << 62, (1 << 62) + 1, (1 << 63) - 1])
def test_attention_refuses_rows_whose_queries_pass_any_size(T):
    """Four query heads per key head: T * 4 wraps to 0 at T = 2^62."""
    S3 = ctypes.c_int64 * 3
    strides = S3(16 * 8 * 128, 8 * 128, 128)
    pages = B.Pages(1 << 20, 1 << 20, strides, strides, 1 << 20, 4, 10, 16, 4, 2, 8, 128, B.GSRQ_F16)
    n = ctypes.c_size_t(7)
    s = B.PagedAttn(T, 32, 0, 0.1, 0)
    status = B.load_library().gsrq_attn_paged_workspace_bytes(ctypes.byref(s), ctypes.byref(pages), ctypes.byref(n))
    assert (status, n.value) == (B.GSRQ_E_UNSUPPORTED, 7)


@pytest.mark.parametrize("B_,cap", [(0, 5), (2, 0), (0, 0)])
def test_restore_of_nothing_returns(B_, cap):
    """No sequences or no code rows: nothing runs, as for appending and attention without rows."""
    kp = torch.zeros((4, 8, 2, 64), dtype=torch.float16)
    codes = torch.zeros((B_, cap, 4), dtype=torch.int32)
    gain, shape = torch.zeros((1, 16, 256)), torch.zeros((1, 16, 256, 8))
    assert B.paged_restore(codes, codes, torch.zeros(B_, dtype=torch.int32), gain, shape, gain, shape, kp, kp,
                           torch.zeros((B_, 2), dtype=torch.int32)) is None


def test_attention_refuses_heads_of_no_elements():
    """They have no default scale; refused as any other head size is."""
    kp = torch.zeros((4, 8, 2, 0), dtype=torch.float16)
    with pytest.raises(ValueError):
        B.attn_paged(torch.zeros((3, 4, 0), dtype=torch.float16), kp, kp, torch.zeros((2, 2), dtype=torch.int32),
                     torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
