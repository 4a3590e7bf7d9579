"""Host-side checks of the layer's operators (no GPU needed): descriptors and pointers that are
rejected before anything is enqueued, the frequency tables, and the binding's refusals."""
import ctypes
import math
import os

import pytest
import torch

from paper_2602_06161_amd import cover

pytestmark = pytest.mark.skipif(not os.path.exists(cover.LIB), reason="libcover.so not built")

INV, UNS, OK = cover.COVER_ERR_INVALID, cover.COVER_ERR_UNSUPPORTED, cover.COVER_OK
FAKE = 0x100000  # 16-byte aligned, never dereferenced: every case below fails validation or is empty


def _p(x):
    return None if x is None else ctypes.c_void_p(x)


def _call(fn, ptrs, desc):
    return fn(*(_p(x) for x in ptrs), None if desc is None else ctypes.byref(desc), None)


def _fill(cls, good, kw):
    d = cls()
    for k, v in {**good, **kw}.items():
        setattr(d, k, v)
    return d


NORM = dict(R=4, D=1000, dtype=cover.COVER_BF16, eps=1e-6, x_stride=1008, res_stride=1008, res_out_stride=1008,
            out_stride=1008)


@pytest.mark.parametrize("kw,ptrs,expect", [
    (dict(R=-1), {}, INV), (dict(D=0), {}, INV), (dict(dtype=5), {}, INV), (dict(eps=-1.0), {}, INV),
    (dict(eps=float("nan")), {}, INV), (dict(eps=float("inf")), {}, INV),
    (dict(D=32769, x_stride=32776, res_stride=32776, res_out_stride=32776, out_stride=32784), {}, UNS),
    (dict(x_stride=999), {}, INV), (dict(x_stride=1004), {}, INV), (dict(res_stride=8), {}, INV),
    (dict(res_out_stride=1001), {}, INV), (dict(out_stride=1001), {}, INV),
    (dict(out_stride=1000), {"scale": FAKE}, INV),               # codes: 1000 bytes, not a multiple of 16
    ({}, {"x": None}, INV), ({}, {"x": FAKE + 8}, INV), ({}, {"out": None}, INV), ({}, {"out": FAKE + 4}, INV),
    ({}, {"weight": FAKE + 2}, INV), ({}, {"residual": FAKE + 2}, INV),
    (dict(out_stride=1024), {"scale": FAKE + 2}, INV),
    (dict(res_out_stride=1016), {"residual_out": FAKE}, INV),   # x in place with another stride
    ({}, {"out": 2 * FAKE}, INV),                                # out and residual_out the same
    (dict(out_stride=1008), {"out": FAKE, "scale": FAKE}, INV),  # codes over x
    (dict(R=0), {"x": None, "out": None}, OK),
])
def test_norm_refusals(kw, ptrs, expect):
    a = {"x": FAKE, "residual": 3 * FAKE, "weight": FAKE, "residual_out": 2 * FAKE, "out": 4 * FAKE, "scale": None, **ptrs}
    assert _call(cover.lib().cover_rms_norm, a.values(), _fill(cover.NormDesc, NORM, kw)) == expect


ROPE = dict(B=2, L=8, Hq=4, Hkv=2, d=128, rot=128, interleaved=0, dtype=cover.COVER_BF16, attention_factor=1.0,
            pos_sb=8, **{f"{t}_{s}": v for t in ("q", "qo", "k", "ko")
                         for s, v in (("sb", 4096), ("sh", 1024), ("sl", 128))})


@pytest.mark.parametrize("kw,ptrs,expect", [
    (dict(B=-1), {}, INV), (dict(L=-1), {}, INV), (dict(Hq=-1), {}, INV), (dict(Hkv=-1), {}, INV),
    (dict(dtype=2), {}, INV), (dict(rot=0), {}, INV), (dict(rot=63), {}, INV), (dict(rot=130), {}, INV),
    (dict(interleaved=2), {}, INV), (dict(attention_factor=float("nan")), {}, INV),
    (dict(attention_factor=float("inf")), {}, INV), (dict(pos_sb=-8), {}, INV), (dict(d=96, rot=96), {}, UNS),
    (dict(q_sl=100), {}, INV), (dict(k_sh=-8), {}, INV), (dict(qo_sl=64), {}, INV), (dict(ko_sl=0), {}, INV),
    (dict(qo_sh=0), {}, INV), (dict(qo_sh=128), {}, INV), (dict(ko_sb=1024), {}, INV), (dict(qo_sb=0), {}, INV),
    (dict(Hq=60000, Hkv=6000), {}, UNS), (dict(B=2**20, L=2**20), {}, UNS),
    ({}, {"q": None}, INV), ({}, {"k": FAKE + 8}, INV), ({}, {"pos": None}, INV), ({}, {"pos": FAKE + 2}, INV),
    ({}, {"freq": None}, INV), ({}, {"freq": FAKE + 4}, INV), ({}, {"q_out": None}, INV),
    (dict(qo_sl=256), {"q_out": FAKE}, INV),                    # q in place with other strides
    (dict(ko_sb=8192), {"k_out": 2 * FAKE}, INV),
    (dict(B=0), {"q": None}, OK), (dict(L=0), {"q": None}, OK), (dict(Hq=0, Hkv=0), {"q": None, "k": None}, OK),
])
def test_rope_refusals(kw, ptrs, expect):
    a = {"q": FAKE, "k": 2 * FAKE, "pos": FAKE, "freq": FAKE, "q_out": 3 * FAKE, "k_out": 4 * FAKE, **ptrs}
    assert _call(cover.lib().cover_rope, a.values(), _fill(cover.RopeDesc, ROPE, kw)) == expect


def test_rope_frequencies():
    tau = 2 * math.pi
    plain = cover.rope_freq(128)
    assert plain.dtype == torch.float64 and plain.shape == (64,)
    for i in (0, 1, 63):
        assert plain[i].item() == pytest.approx(10000.0 ** (-2 * i / 128) / tau, rel=1e-14)
    assert torch.allclose(cover.rope_freq(128, scaling="linear", factor=4.0), plain / 4, rtol=1e-14, atol=0)
    base = cover.rope_freq(128, scaling="base", factor=4.0)
    assert base[0] == plain[0] and base[63].item() == pytest.approx(plain[63].item() / 4, rel=1e-12)
    parts = cover.rope_freq(128, 500000.0, "parts", 8.0, original_length=8192, low=1.0, high=4.0)
    f = cover.rope_freq(128, 500000.0)
    turns = 8192 * f
    assert torch.equal(parts[turns >= 4], f[turns >= 4])        # many turns: kept
    assert torch.allclose(parts[turns <= 1], f[turns <= 1] / 8, rtol=1e-14, atol=0)
    mid = (turns > 1) & (turns < 4)
    g = (turns[mid] - 1) / 3
    assert mid.any() and torch.allclose(parts[mid], f[mid] * g + f[mid] / 8 * (1 - g), rtol=1e-13, atol=0)
    assert cover.rope_freq(2).tolist() == [1 / tau]


@pytest.mark.parametrize("kw", [dict(rot=0), dict(rot=7), dict(rot=-2), dict(base=1.0), dict(base=float("inf")),
                                dict(scaling="linear", factor=0.5), dict(scaling="base", rot=2, factor=2.0),
                                dict(scaling="base", base=1e300, factor=1e300),
                                dict(scaling="parts", factor=2.0, original_length=0.0),
                                dict(scaling="parts", factor=2.0, original_length=10, low=3.0, high=3.0)])
def test_rope_frequency_refusals(kw):
    with pytest.raises(cover.CoverError) as e:
        cover.rope_freq(**{"rot": 64, **kw})
    assert e.value.status == INV
    with pytest.raises(ValueError):
        cover.rope_freq(64, scaling="other")


CACHE = dict(B=2, H=2, N=8, L=64, d=128, first=0, dtype=cover.COVER_BF16, k_sb=2048, k_sh=1024, k_sl=128, v_sb=2048,
             v_sh=1024, v_sl=128, c_sb=16384, c_sh=8192, c_sl=128, s_sb=128, s_sh=64)


@pytest.mark.parametrize("name", ["cover_cache_store", "cover_cache_load"])
@pytest.mark.parametrize("kw,ptrs,expect", [
    (dict(B=-1), {}, INV), (dict(H=-1), {}, INV), (dict(N=-1), {}, INV), (dict(L=0), {}, INV), (dict(dtype=9), {}, INV),
    (dict(d=0), {}, INV), (dict(d=80), {}, UNS), (dict(k_sl=100), {}, INV), (dict(v_sb=-8), {}, INV),
    (dict(c_sl=136), {}, INV), (dict(c_sl=64), {}, INV), (dict(s_sh=-1), {}, INV),
    (dict(first=-1), {"pos": None}, INV), (dict(first=57), {"pos": None}, INV),
    (dict(first=2**31 - 4), {"pos": None}, INV),
    ({}, {"k": None}, INV), ({}, {"v": FAKE + 8}, INV), ({}, {"pos": FAKE + 1}, INV), ({}, {"kc": None}, INV),
    ({}, {"vc": FAKE + 8}, INV), ({}, {"ks": None}, INV), ({}, {"vs": FAKE + 2}, INV),
    (dict(B=2**20, H=2**10), {}, UNS),
    (dict(N=0), {"k": None}, OK), (dict(B=0), {"k": None}, OK), (dict(H=0), {"k": None}, OK),
])
def test_cache_refusals(name, kw, ptrs, expect):
    a = {"k": FAKE, "v": 2 * FAKE, "pos": FAKE, "kc": 3 * FAKE, "vc": 4 * FAKE, "ks": 5 * FAKE, "vs": 6 * FAKE, **ptrs}
    assert _call(getattr(cover.lib(), name), a.values(), _fill(cover.CacheDesc, CACHE, kw)) == expect


def test_load_refuses_overlapping_rows():
    a = [i * FAKE for i in range(1, 8)]
    for kw in (dict(k_sl=64), dict(v_sl=0), dict(k_sh=0), dict(v_sb=1024), dict(k_sh=128, k_sb=256), dict(k_sl=136)):
        assert _call(cover.lib().cover_cache_load, a, _fill(cover.CacheDesc, CACHE, kw)) == INV, kw
    assert _call(cover.lib().cover_cache_load, [FAKE, FAKE, *a[2:]], _fill(cover.CacheDesc, CACHE, {})) == INV


def test_store_refuses_overlapping_caches():
    a = [i * FAKE for i in range(1, 8)]
    for kw in (dict(c_sh=0), dict(c_sb=8192), dict(s_sh=63), dict(s_sb=64), dict(c_sl=128, c_sh=128, c_sb=128),
               dict(c_sl=0)):
        assert _call(cover.lib().cover_cache_store, a, _fill(cover.CacheDesc, CACHE, kw)) == INV, kw
    for same in ((3, 4), (5, 6)):  # one tensor for the codes (the scales) of keys and values
        b = list(a)
        b[same[1]] = b[same[0]]
        assert _call(cover.lib().cover_cache_store, b, _fill(cover.CacheDesc, CACHE, {})) == INV


def test_more_rows_than_a_launch_takes():
    """Rows beyond 2^32 work-items: refused, not cut short."""
    wide = dict(R=2**22, D=32768, x_stride=32768, out_stride=32768)
    narrow = dict(R=2**26, D=8, x_stride=8, out_stride=8)
    for kw in (wide, narrow):
        a = [FAKE, None, None, None, 2 * FAKE, None]
        assert _call(cover.lib().cover_rms_norm, a, _fill(cover.NormDesc, NORM, kw)) == UNS


CACHED = dict(B=1, Hq=4, Hkv=2, L=64, Lq=16, d=128, max_seeds=4, q_off=32, n_split=1, scale=0.0, c_sb=16384, c_sh=8192,
              c_sl=128, s_sb=128, s_sh=64,
              **{f"{t}_{s}": v for t in "qokv" for s, v in (("sb", 8192), ("sh", 2048), ("sl", 128))})


@pytest.mark.parametrize("kw,ptrs,expect", [
    (dict(B=-1), {}, INV), (dict(Hq=0), {}, INV), (dict(Hkv=3), {}, INV), (dict(L=-1), {}, INV), (dict(Lq=-1), {}, INV),
    (dict(max_seeds=-1), {}, INV), (dict(scale=-1.0), {}, INV), (dict(scale=float("nan")), {}, INV),
    (dict(n_split=0), {}, INV), (dict(n_split=257), {}, INV), (dict(q_off=-1), {}, INV), (dict(q_off=49), {}, INV),
    (dict(d=96), {}, UNS), (dict(L=cover.COVER_MAX_L + 1), {}, UNS),
    (dict(L=4096, Lq=cover.COVER_CACHED_MAX_LQ + 1), {}, UNS),
    (dict(q_sl=100), {}, INV), (dict(o_sl=64), {}, INV), (dict(k_sh=-8), {}, INV), (dict(v_sl=0), {}, INV),
    (dict(c_sl=64), {}, INV), (dict(c_sh=8), {}, INV), (dict(s_sb=-1), {}, INV),
    ({}, {"q": None}, INV), ({}, {"out": FAKE + 8}, INV), ({}, {"kc": FAKE + 4}, INV), ({}, {"ks": None}, INV),
    ({}, {"off": FAKE + 2}, INV), ({}, {"len": FAKE + 1}, INV), ({}, {"idx": None}, INV), ({}, {"n": FAKE + 2}, INV),
    ({}, {"out": FAKE}, INV), (dict(o_sh=0), {}, INV), (dict(o_sh=128), {}, INV), (dict(B=2, o_sb=2048), {}, INV),
    (dict(o_sl=512, o_sh=64), {}, INV), ({}, {"lse": FAKE + 2}, INV), (dict(n_split=2), {"ws": None}, INV), (dict(n_split=2), {"ws": FAKE + 8}, INV),
    (dict(B=2**20, Hq=64, Hkv=64), {}, UNS),
    (dict(B=0), {"q": None}, OK), (dict(Lq=0, q_off=0), {"q": None}, OK), (dict(L=0, Lq=0, q_off=0), {"q": None}, OK),
])
def test_attn_cached_refusals(kw, ptrs, expect):
    a = {n: FAKE for n in ("q", "k", "v", "kc", "vc", "ks", "vs")}
    a.update({"off": None, "len": None, "idx": FAKE, "n": FAKE, "out": 2 * FAKE, "lse": None, "ws": None, **ptrs})
    assert _call(cover.lib().cover_attn_cached, a.values(), _fill(cover.CachedDesc, CACHED, kw)) == expect


def test_null_descriptors():
    lib = cover.lib()
    for name, n in (("cover_rms_norm", 6), ("cover_rope", 6), ("cover_cache_store", 7), ("cover_cache_load", 7),
                    ("cover_attn_cached", 14)):
        assert _call(getattr(lib, name), [FAKE] * n, None) == INV


def test_splits_are_within_what_the_call_takes():
    for size in ((1, 32, 8, 8192, 1), (1, 28, 4, 65536, 32), (8, 32, 32, 2048, 256), (1, 1, 1, 65536, 1), (1, 4, 2, 1, 1)):
        assert 1 <= cover.attn_cached_splits(*size) <= 256
    for bad in ((0, 4, 2, 8, 1), (1, 4, 3, 8, 1), (1, 4, 2, 0, 1), (1, 4, 2, 8, 0), (1, 4, 2, 70000, 1), (-1, 1, 1, 1, 1)):
        assert cover.attn_cached_splits(*bad) == 1
    assert cover.attn_cached_workspace(2, 4, 8, 128, 1) == 0
    assert cover.attn_cached_workspace(2, 4, 8, 128, 3) == 2 * 4 * 8 * 3 * 132


def test_binding_refuses_host_tensors():
    """Tensors that are not on the GPU never reach a kernel: the native forms hand them back, the
    Python forms raise."""
    h = cover.host()
    x = torch.zeros(4, 64)
    assert h.rms_norm(x, None, None, 1e-6, False, None, None, None, 0, -1) is None
    assert h.rms_norm() is None and h.attn_cached() is None
    with pytest.raises(ValueError):
        cover.cover_rms_norm(x)
    t = torch.zeros(1, 2, 4, 64)
    pos, freq = torch.zeros(1, 4, dtype=torch.int32), cover.rope_freq(64)
    with pytest.raises(ValueError):
        cover.cover_rope(t, t, pos, freq)
    codes, s = torch.zeros(1, 2, 8, 64).to(torch.float8_e4m3fn), torch.zeros(1, 2, 8)
    with pytest.raises(ValueError):
        cover.cover_cache_store(t, t, 0, codes, codes, s, s)
    with pytest.raises(ValueError):
        cover.cover_cache_load(codes, codes, s, s, 0, n=4)
    with pytest.raises(ValueError):
        cover.cover_attn_cached(t.bfloat16(), t.bfloat16(), t.bfloat16(), codes, codes, s, s, 0)
    with pytest.raises(ValueError):
        h.bind_layer(1)
