"""Outputs of the layer's operators that are another operand: refused before anything is enqueued (no GPU needed)."""
import ctypes
import os

import pytest

from paper_2602_06161_amd import cover

pytestmark = pytest.mark.skipif(not os.path.exists(cover.LIB), reason="libcover.so not built")

FAKE = 0x100000  # 16-byte aligned, never dereferenced: every case below is refused


@pytest.mark.parametrize("q,k,q_out,k_out", [(1, 2, 3, 3), (1, 2, 2, 4), (1, 2, 3, 1), (1, 2, 2, 1), (1, 1, 1, 1)])
def test_rotary_outputs_that_are_the_other_tensor(q, k, q_out, k_out):
    d = cover.RopeDesc(1, 8, 2, 2, 64, 64, 0, cover.COVER_BF16, 1.0, 8, *(1024, 512, 64) * 4)
    args = [ctypes.c_void_p(FAKE * i) for i in (q, k, 9, 10, q_out, k_out)]
    assert cover.lib().cover_rope(*args, ctypes.byref(d), None) == cover.COVER_ERR_INVALID


@pytest.mark.parametrize("out", [1, 2, 3])
def test_attention_outputs_that_are_an_input(out):
    d = cover.CachedDesc(1, 2, 2, 64, 16, 128, 0, 32, 1, 0.0, *(4096, 2048, 128) * 4, 16384, 8192, 128, 128, 64)
    args = [ctypes.c_void_p(FAKE * i) for i in range(1, 8)] + [None] * 4 + [ctypes.c_void_p(FAKE * out), None, None]
    assert cover.lib().cover_attn_cached(*args, ctypes.byref(d), None) == cover.COVER_ERR_INVALID
