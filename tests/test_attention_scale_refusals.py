"""Scales that the attention refuses (no GPU needed: see test_paged_refusals)."""
import ctypes as C
import math

import pytest

from paper_2608_25431_b200 import binding, build as B
from test_paged_refusals import attention, attn, batch, pool


@pytest.mark.parametrize("scale,code", [(math.nan, binding.E_INVAL), (math.inf, binding.E_INVAL), (-math.inf, binding.E_INVAL),
                                        (3e38, binding.E_RANGE), (-3e38, binding.E_RANGE)])
def test_scales(scale, code):
    B.build_lib()
    lib, ctx = binding.lib(), C.create_string_buffer(1 << 16)
    for rows in (1, 4):                            # few rows per K/V head, and (with 32 heads to one) many
        assert attention(lib, ctx, batch(), pool(), attn(n_rows=rows, scale=scale)) == code
        assert attention(lib, ctx, batch(n_req=1), pool(n_heads=1), attn(n_rows=rows, n_heads=32, scale=scale)) == code
