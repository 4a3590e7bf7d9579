"""cover_attn_cached_plan: what it answers and what it refuses (no GPU needed)."""
import ctypes
import os

import pytest

from paper_2602_06161_amd import cover

pytestmark = pytest.mark.skipif(not os.path.exists(cover.LIB), reason="libcover.so not built")

GOOD = dict(B=1, Hq=4, Hkv=2, L=8192, Lq=4, d=128, n_split=64)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size", [(1, 1, 1, 1, 1), (1, 32, 8, 8192, 1), (1, 28, 4, 65536, 32), (8, 32, 32, 2048, 256),
                                  (1, 2, 1, 4096, 2048), (64, 40, 8, 999, 17)])
def test_plans_are_within_what_the_call_takes(size, d):
    for most in (1, 2, 7, 64, 256, None):
        ranges, rows = cover.attn_cached_plan(*size, d, most)
        assert 1 <= ranges <= (most or 256) and rows in (32, 64, 128)
        assert rows < 128 or (d == 128 and ranges == 1)
    # the ranges asked for by the rule itself are the ones taken
    assert cover.attn_cached_plan(*size, d)[0] == cover.attn_cached_splits(*size)


@pytest.mark.parametrize("kw,expect", [
    (dict(B=0), cover.COVER_ERR_INVALID), (dict(Hq=0), cover.COVER_ERR_INVALID), (dict(Hkv=3), cover.COVER_ERR_INVALID),
    (dict(Hkv=-1), cover.COVER_ERR_INVALID), (dict(L=0), cover.COVER_ERR_INVALID), (dict(Lq=0), cover.COVER_ERR_INVALID),
    (dict(d=0), cover.COVER_ERR_INVALID), (dict(n_split=0), cover.COVER_ERR_INVALID), (dict(n_split=257), cover.COVER_ERR_INVALID),
    (dict(d=96), cover.COVER_ERR_UNSUPPORTED), (dict(L=cover.COVER_MAX_L + 1), cover.COVER_ERR_UNSUPPORTED),
    (dict(Lq=cover.COVER_CACHED_MAX_LQ + 1), cover.COVER_ERR_UNSUPPORTED), (dict(B=2**20, Hq=64, Hkv=64), cover.COVER_ERR_UNSUPPORTED),
])
def test_refusals(kw, expect):
    with pytest.raises(cover.CoverError) as e:
        cover.attn_cached_plan(**{**GOOD, **kw})
    assert e.value.status == expect


def test_null_outputs():
    n = ctypes.c_int32(0)
    assert cover.lib().cover_attn_cached_plan(*GOOD.values(), None, ctypes.byref(n)) == cover.COVER_ERR_INVALID
    assert cover.lib().cover_attn_cached_plan(*GOOD.values(), ctypes.byref(n), None) == cover.COVER_ERR_INVALID


# ---- sizes whose products pass 64 bits -------------------------------------------------------
BIG = 2**31 - 1
FAKE = 0x100000  # 16-byte aligned, never dereferenced: every case below is refused


@pytest.mark.parametrize("size", [(2**30, 2**30, 2**30, 8192, 512), (BIG, BIG, BIG, 65536, 2048), (2**16, 2**16, 2**16, 64, 64),
                                  (BIG, BIG, 1, 4096, 4), (1, BIG, BIG, 64, 2048), (2**20, 64, 64, 8192, 1)])
def test_sizes_beyond_any_launch(size):
    assert cover.attn_cached_splits(*size) == 1
    with pytest.raises(cover.CoverError) as e:
        cover.attn_cached_plan(*size, 128, 256)
    assert e.value.status == cover.COVER_ERR_UNSUPPORTED


@pytest.mark.parametrize("name", ["cover_cache_store", "cover_cache_load"])
@pytest.mark.parametrize("B,H,N", [(2**30, 2**30, 2**28), (BIG, BIG, BIG), (2**24, 1, 1), (2**12, 2**12, 1), (1, 1, 2**28)])
def test_cache_calls_beyond_any_launch(name, B, H, N):
    d = cover.CacheDesc(B, H, N, BIG, 64, 0, cover.COVER_BF16, *[0] * 11)
    d.c_sl = 64
    args = [ctypes.c_void_p(i * FAKE) for i in range(1, 8)]
    assert getattr(cover.lib(), name)(*args, ctypes.byref(d), None) == cover.COVER_ERR_UNSUPPORTED


@pytest.mark.parametrize("B,L", [(BIG, BIG), (2**30, 2**30), (2**24, 2**10)])
def test_rotary_calls_beyond_any_launch(B, L):
    d = cover.RopeDesc(B, L, 64, 0, 64, 64, 0, cover.COVER_BF16, 1.0, *[0] * 13)
    args = [ctypes.c_void_p(i * FAKE) for i in range(1, 7)]
    assert cover.lib().cover_rope(*args, ctypes.byref(d), None) == cover.COVER_ERR_UNSUPPORTED
