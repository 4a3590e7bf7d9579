"""The layer's operators around the attention (norm, rotary positions, the 8-bit cache and the
attention over it) against plain implementations in 64 bits.

Tolerances, derived: a rounding to bf16 is off by at most 2^-8 of the value, to e4m3 by 2^-4 (or half
the smallest step, 2^-10 of the scale), an fp32 operation by 2^-24.
  norm   mean of D squares in fp32: at most (D / 64 + 12) roundings in a row in the sum, half of that
         relative in its root, and 5 more operations: 2^-24 (D / 128 + 12) relative
  rope   the turn is rounded once to fp32 (2^-24 of half a turn is 2^-24 pi radians), sine and cosine
         are good to 2^-22, then 4 roundings: 2^-21 of |x| + |y|, times the factor
  attn   weights rounded to bf16: 2^-8 of sum p |v|, the output 2^-8; a score sums d products in fp32,
         (d + 8) 2^-24 of scale sum |q| |k| at most, twice as much relative in a weight
"""
import math

import pytest
import torch

from helpers import announce
from paper_2602_06161_amd import cover

pytestmark = pytest.mark.gpu

BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
STEP = {BF16: 2.0**-8, F32: 2.0**-24}


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return lambda *shape: torch.randn(*shape, generator=g, device="cuda")


def _within(got, want, tol, what):
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst by {((got.double() - want).abs() - tol).max()}"


def _same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


# ---- norm ------------------------------------------------------------------------------------
def _rows(r, R, D, dtype, scale=1.0):
    per = 16 // dtype.itemsize
    return (scale * r(R, -(-D // per) * per)).to(dtype)[:, :D]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("quantize", [False, True])
@pytest.mark.parametrize("R,D,residual,weight", [
    (1, 1, True, True), (3, 5, False, True), (1, 4096, True, True), (2, 513, True, False), (33, 1001, True, True),
    (5, 3584, False, False), (300, 768, True, True), (7, 8192, True, True), (4, 12288, True, True), (2, 32768, True, True),
    (2, 32761, False, True), (9, 64, True, True), (2100, 200, True, True),
])
def test_norm(dtype, quantize, R, D, residual, weight):
    announce(f"norm {dtype} q{quantize} R{R} D{D}")
    r = _gen(R * 7 + D)
    x, res = _rows(r, R, D, dtype), _rows(r, R, D, dtype, 2.0) if residual else None
    w = (1 + 0.2 * r(D)).to(dtype) if weight else None
    y, ro, s = cover.cover_rms_norm(x, w, res, 1e-5, quantize)
    torch.cuda.synchronize()
    h = x.double() + (res.double() if residual else 0)
    want = h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-5) * (w.double() if weight else 1.0)
    fp32 = 2.0**-24 * (D / 128 + 12)
    assert (ro is None) == (res is None) and (s is None) != quantize
    if residual:
        _within(ro, h, (STEP[dtype] + 2.0**-24) * h.abs(), "residual")
    if not quantize:
        _within(y, want, (STEP[dtype] + fp32) * want.abs(), "norm")
        return
    assert y.dtype == E4M3 and s.shape == (R,)
    top = want.abs().amax(1)
    _within(s, (top / 448).clamp_min(2.0**-126), (fp32 + 2.0**-23) * top / 448, "scale")
    back = y.double() * s.double()[:, None]
    half = torch.maximum(2.0**-4 * want.abs(), 2.0**-10 * s.double()[:, None])
    _within(back, want, half * (1 + 2.0**-12) + (fp32 + 2.0**-22) * want.abs(), "codes")


def test_norm_in_place_and_given_outputs():
    announce("norm in place")
    r = _gen(3)
    x, res, w = _rows(r, 40, 1000, BF16), _rows(r, 40, 1000, BF16), (1 + 0.1 * r(1000)).to(BF16)
    y, ro, _ = cover.cover_rms_norm(x, w, res)
    x2, res2 = x.clone(), res.clone()
    got = cover.cover_rms_norm(x2, w, res2, out=x2, residual_out=res2)
    assert got[0] is x2 and got[1] is res2 and _same(x2, y) and _same(res2, ro)
    x3 = x.clone()  # the sum over x, the norm apart
    y3, ro3, _ = cover.cover_rms_norm(x3, w, res, residual_out=x3)
    assert ro3 is x3 and _same(x3, ro) and _same(y3, y)
    # rows of a wider tensor: what lies between them is left alone
    wide = torch.full((40, 1024), 7.0, device="cuda", dtype=BF16)
    cover.cover_rms_norm(x, w, res, out=wide[:, :1000])
    assert _same(wide[:, :1000], y) and (wide[:, 1000:] == 7).all()
    assert _same(cover.cover_rms_norm(x[5:6], w, res[5:6])[0], y[5:6])


def test_norm_rows_of_zeros_infinities_and_nans():
    announce("norm special rows")
    x = torch.ones(5, 256, device="cuda", dtype=F32)
    x[0] = 0.0
    x[1, 7] = math.inf
    x[2, 9] = math.nan
    x[3] = 1e-30
    y, _, _ = cover.cover_rms_norm(x, eps=0.0)
    q, _, s = cover.cover_rms_norm(x, quantize=True)
    assert torch.isnan(y[1, 7]) and (y[1, :7] == 0).all() and torch.isnan(y[2]).all() and (y[4] == 1).all()
    assert (q[0].float() == 0).all() and s[0] == 2.0**-126
    back = q.float() * s[:, None]
    assert torch.isnan(back[1]).all() and torch.isnan(back[2]).all()
    assert (back[4] - 1).abs().max() <= 2.0**-20 and s[3] > 0


# ---- rotary positions ------------------------------------------------------------------------
def _turned(x, pos, freq, m, interleaved):
    rot = 2 * freq.shape[0]
    a = 2 * math.pi * ((pos.double()[:, None, :, None] * freq) % 1.0)
    c, s = m * a.cos(), m * a.sin()
    y = x.double().clone()
    i, j = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    p, q = x.double()[..., i], x.double()[..., j]
    y[..., i], y[..., j] = p * c - q * s, q * c + p * s
    size = torch.zeros_like(y)
    size[..., i] = size[..., j] = abs(m) * (p.abs() + q.abs())
    return y, size


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,Hq,Hkv,L,d,rot", [
    (1, 32, 32, 1, 128, 128), (2, 28, 4, 9, 128, 96), (1, 3, 1, 700, 64, 64), (3, 5, 5, 33, 64, 20), (2, 1, 0, 5, 128, 2),
    (1, 12, 12, 70, 128, 64), (1, 40, 8, 6, 64, 22), (2, 8, 2, 40, 128, 126), (1, 300, 20, 3, 64, 48),
])
def test_rope(dtype, interleaved, B, Hq, Hkv, L, d, rot):
    announce(f"rope {dtype} i{interleaved} B{B} H{Hq}/{Hkv} L{L} d{d} rot{rot}")
    r = _gen(L + rot)
    qkv = r(B, L, Hq + 2 * Hkv, d).to(dtype)  # views of a fused projection
    q, k = qkv[:, :, :Hq].transpose(1, 2), qkv[:, :, Hq:Hq + Hkv].transpose(1, 2) if Hkv else None
    m = 1.3 if rot % 4 == 0 else 1.0
    pos = torch.randint(-5, 100000, (B, L), device="cuda", dtype=torch.int32)
    pos[0, 0] = 2**31 - 1
    freq = cover.rope_freq(rot, 500000.0, device="cuda")
    before = qkv.clone()
    qo, ko = cover.cover_rope(q, k, pos, freq, interleaved, m)
    torch.cuda.synchronize()
    assert _same(qkv, before)
    for x, got in ((q, qo), (k, ko)):
        assert (x is None) == (got is None)
        if x is None:
            continue
        want, size = _turned(x, pos, freq, m, interleaved)
        _within(got, want, 2.0**-21 * size + STEP[dtype] * want.abs(), "rope")
        assert _same(got[..., rot:], x[..., rot:])
    # in place, in views of the projection; v's heads stay
    got = cover.cover_rope(q, k, pos, freq, interleaved, m, q_out=q, k_out=k)
    assert got[0] is q and _same(q, qo) and (k is None or _same(k, ko))
    assert _same(qkv[:, :, Hq + Hkv:], before[:, :, Hq + Hkv:])


def test_rope_shared_positions_and_layouts():
    announce("rope shared positions")
    r = _gen(1)
    q, k = r(2, 6, 50, 64).to(BF16), r(2, 2, 50, 64).to(BF16)
    pos = torch.arange(50, device="cuda", dtype=torch.int32)
    freq = cover.rope_freq(64, device="cuda")
    a, b = cover.cover_rope(q, k, pos, freq)
    c, e = cover.cover_rope(q, k, pos[None].repeat(2, 1), freq)
    assert _same(a, c) and _same(b, e)
    into = torch.zeros(2, 50, 6, 64, device="cuda", dtype=BF16).transpose(1, 2)  # token-major output
    got, none = cover.cover_rope(q, None, pos, freq, q_out=into)
    assert got is into and none is None and _same(into, a)
    assert cover.cover_rope(q[:, :, :0], k[:, :, :0], pos[:0], freq)[0].shape == (2, 6, 0, 64)


# ---- the 8-bit cache -------------------------------------------------------------------------
def _codes(x):
    """The e4m3 form in fp32 on the CPU, step by step as the header states it."""
    x = x.float().cpu()
    s = (x.abs().amax(-1) / 448).clamp_min(2.0**-126)
    return (x * (1 / s)[..., None]).to(E4M3), s


def _empty_cache(B, H, L, d, fill=0x55):
    code = lambda: torch.full((B, H, L, d), fill, device="cuda", dtype=torch.uint8).view(E4M3)  # noqa: E731
    return code(), code(), torch.full((B, H, L), 3.0, device="cuda"), torch.full((B, H, L), 5.0, device="cuda")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,H,N,L,d", [(1, 1, 1, 1, 64), (1, 32, 64, 256, 128), (2, 4, 17, 40, 128), (3, 2, 33, 33, 64),
                                       (1, 3, 300, 1001, 64), (2, 1, 5, 9, 128)])
def test_cache_store_and_load(dtype, B, H, N, L, d):
    announce(f"cache {dtype} B{B} H{H} N{N} L{L} d{d}")
    r = _gen(N + L)
    k = (r(B, N, H, d) * torch.exp(3 * r(B, N, H, 1))).to(dtype).transpose(1, 2)  # token-major
    v = r(B, H, N, d).to(dtype)
    pos = torch.rand(B, L, device="cuda").argsort(1)[:, :N].to(torch.int32).contiguous()  # any order
    if N > 4:
        pos[:, 1], pos[:, 3] = -1, L
        pos[0, 2] = -2**31
    cache = _empty_cache(B, H, L, d)
    before = [t.clone() for t in cache]
    got = cover.cover_cache_store(k, v, pos, *cache)
    torch.cuda.synchronize()
    assert all(a is b for a, b in zip(got, cache))
    want = [t.cpu() for t in before]
    for x, c, s in ((k, 0, 2), (v, 1, 3)):
        codes, scale = _codes(x)
        for b in range(B):
            for n, p in enumerate(pos[b].tolist()):
                if 0 <= p < L:
                    want[c].view(torch.uint8)[b, :, p] = codes.view(torch.uint8)[b, :, n]
                    want[s][b, :, p] = scale[b, :, n]
    for a, w in zip(cache, want):
        assert _same(a.cpu(), w)
    # back: listed rows (zeros where there is no such position), and a run of them
    for out_type in (BF16, F32):
        ko, vo = cover.cover_cache_load(*cache, pos, dtype=out_type)
        for codes, s, o in ((want[0], want[2], ko), (want[1], want[3], vo)):
            full = (codes.float() * s[..., None]).to(out_type)
            for b in range(B):
                for n, p in enumerate(pos[b].tolist()):
                    row = full[b, :, p] if 0 <= p < L else torch.zeros(H, d, dtype=out_type)
                    assert _same(o[b, :, n].cpu(), row)
        first, n = (L // 3, L - L // 3)
        ko, vo = cover.cover_cache_load(*cache, first, n=n, dtype=out_type)
        assert _same(ko.cpu(), (want[0].float() * want[2][..., None]).to(out_type)[:, :, first:])
        assert _same(vo.cpu(), (want[1].float() * want[3][..., None]).to(out_type)[:, :, first:])


def test_cache_run_of_positions_repeats_and_strides():
    announce("cache runs, repeats, strides")
    r = _gen(9)
    B, H, L, d = 2, 3, 50, 128
    k, v = r(B, H, 20, d).to(BF16), r(B, H, 20, d).to(BF16)
    big = _empty_cache(B, H, 2 * L, d)
    cache = tuple(t[:, :, L // 2:L // 2 + L] for t in big)  # a part of a larger cache
    cover.cover_cache_store(k, v, 30, *cache)
    plain = _empty_cache(B, H, L, d)
    cover.cover_cache_store(k, v, torch.arange(30, 50, device="cuda", dtype=torch.int32).repeat(B, 1), *plain)
    for a, b in zip(cache, plain):
        assert _same(a, b)
    assert all(_same(t[:, :, :L // 2 + 30], f[:, :, :L // 2 + 30]) for t, f in zip(big, _empty_cache(B, H, 2 * L, d)))
    twice = torch.tensor([[31, 31, 40], [0, 49, 49]], device="cuda", dtype=torch.int32)  # reading may repeat
    ko, _ = cover.cover_cache_load(*plain, twice)
    assert _same(ko[0, :, 0], ko[0, :, 1]) and _same(ko[1, :, 1], ko[1, :, 2])
    into = torch.zeros(B, 3, H, d, device="cuda", dtype=BF16).transpose(1, 2)
    back, _ = cover.cover_cache_load(*plain, twice, k=into)
    assert back is into and _same(into, ko)
    assert cover.cover_cache_load(*plain, 0, n=0)[0].shape == (B, H, 0, d)


def test_cache_special_rows_and_extremes():
    announce("cache special rows")
    x = torch.zeros(1, 1, 8, 64, device="cuda")
    x[0, 0, 1, 3] = math.inf
    x[0, 0, 2, 5] = math.nan
    x[0, 0, 3] = 1e-38
    x[0, 0, 4] = 3e38
    x[0, 0, 5, :32], x[0, 0, 5, 32:] = 448.0, 2.0**-12
    x[0, 0, 6] = torch.linspace(-1, 1, 64, device="cuda")
    cache = _empty_cache(1, 1, 8, 64)
    cover.cover_cache_store(x, -x, 0, *cache)
    k, v = cover.cover_cache_load(*cache, 0, n=8, dtype=F32)
    assert (k[0, 0, 0] == 0).all() and (k[0, 0, 7] == 0).all() and cache[2][0, 0, 0] == 2.0**-126
    assert torch.isnan(k[0, 0, 1]).all() and torch.isnan(v[0, 0, 1]).all() and torch.isnan(k[0, 0, 2]).all()
    for n in (3, 4, 6):
        s = cache[2][0, 0, n].double()
        tol = torch.maximum(2.0**-4 * x[0, 0, n].double().abs(), 2.0**-10 * s) * (1 + 2.0**-12)
        _within(k[0, 0, n], x[0, 0, n].double(), tol, f"row {n}")
        _within(v[0, 0, n], -x[0, 0, n].double(), tol, f"row {n}")
    assert (k[0, 0, 5, :32] == 448).all() and (k[0, 0, 5, 32:] == 0).all()


def test_offsets_beyond_32_bits():
    """Batch rows and heads of the cache more than 4 GiB apart."""
    announce("offsets beyond 32 bits")
    r = _gen(2)
    B, H, L, d, far = 2, 2, 64, 128, 2**31 + 4096
    pool = torch.empty(4 * far, device="cuda", dtype=torch.uint8)
    codes = [pool[i * 2 * L * d:].view(E4M3).as_strided((B, H, L, d), (2 * far - 8192, far - 4096, d, 1),
                                                        i * 2 * L * d) for i in (0, 1)]
    near = _empty_cache(B, H, L, d)
    k, v = r(B, H, L, d).to(BF16), r(B, H, L, d).to(BF16)
    s = (near[2], near[3])
    cover.cover_cache_store(k, v, 0, codes[0], codes[1], *s)
    cover.cover_cache_store(k, v, 0, near[0], near[1], *s)
    a, b = cover.cover_cache_load(*codes, *s, 0, n=L), cover.cover_cache_load(*near, 0, n=L)
    assert _same(a[0], b[0]) and _same(a[1], b[1])
    q = r(B, 4, 3, d).to(BF16)
    o1, l1 = cover.cover_attn_cached(q, k[:, :, :3], v[:, :, :3], *codes, *s, 20)
    o2, l2 = cover.cover_attn_cached(q, k[:, :, :3], v[:, :, :3], *near, 20)
    assert _same(o1, o2) and _same(l1, l2)


# ---- attention over the cache ----------------------------------------------------------------
def _problem(seed, B, Hq, Hkv, L, Lq, d, n_seeds, off, lens=None, spread=0.3):
    r = _gen(seed)
    t = {"q": r(B, Lq, Hq, d).to(BF16).transpose(1, 2), "k": r(B, Hkv, Lq, d).to(BF16),
         "v": r(B, Lq, Hkv, d).to(BF16).transpose(1, 2)}
    cache = _empty_cache(B, Hkv, L, d)
    cover.cover_cache_store((r(B, Hkv, L, d) * torch.exp(spread * r(B, Hkv, L, 1))).to(BF16),
                            (r(B, Hkv, L, d) * torch.exp(spread * r(B, Hkv, L, 1))).to(BF16), 0, *cache)
    t["cache"] = cache
    t["off"] = off if isinstance(off, int) else torch.tensor(off, device="cuda", dtype=torch.int32)
    t["len"] = None if lens is None else torch.tensor(lens, device="cuda", dtype=torch.int32)
    offs = [off] * B if isinstance(off, int) else off
    t["idx"] = t["n"] = None
    if n_seeds:
        g = torch.Generator().manual_seed(seed)
        idx = torch.stack([offs[b] + torch.randperm(Lq, generator=g)[:n_seeds] for b in range(B)])
        t["idx"] = idx.to(device="cuda", dtype=torch.int32)
        t["n"] = torch.tensor([n_seeds - (b % 2) * (n_seeds > 1) for b in range(B)], device="cuda", dtype=torch.int32)
    return t


def _call(t, **kw):
    return cover.cover_attn_cached(t["q"], t["k"], t["v"], *t["cache"], t["off"], t["idx"], t["n"], kv_len=t["len"], **kw)


def _reference(t, scale=None, weight=2.0**-8):
    """out, lse, and their tolerances, row by row from each row's own memory; NaN where no row exists.  weight: what
    a weight may be off by, relative."""
    q, k, v = (t[n].double().cpu() for n in "qkv")
    kc, vc = (t["cache"][i].cpu().double() * t["cache"][2 + i].cpu().double()[..., None] for i in (0, 1))
    B, Hq, Lq, d = q.shape
    Hkv, L = kc.shape[1:3]
    scale = scale or d**-0.5
    out, lse, tol, ltol = (torch.full(s, math.nan, dtype=torch.float64) for s in
                           ((B, Hq, Lq, d), (B, Hq, Lq), (B, Hq, Lq, d), (B, Hq, Lq)))
    for b in range(B):
        n = L if t["len"] is None else min(max(int(t["len"][b]), 0), L)
        o = t["off"] if isinstance(t["off"], int) else min(max(int(t["off"][b]), 0), n)
        rows = min(Lq, n - o)
        seeds = set() if t["idx"] is None else set(t["idx"][b, :int(t["n"][b])].tolist())
        K, V = kc[b, :, :n].clone(), vc[b, :, :n].clone()
        for r in range(rows):
            if o + r not in seeds:
                K[:, o + r], V[:, o + r] = k[b, :, r], v[b, :, r]
        for r in range(rows):
            Kr, Vr = K, V
            if o + r in seeds:
                Kr, Vr = K.clone(), V.clone()
                Kr[:, o + r], Vr[:, o + r] = k[b, :, r], v[b, :, r]
            G = Hq // Hkv
            x = q[b, :, r].view(Hkv, G, d)
            s = scale * (x @ Kr.transpose(1, 2))
            p = torch.softmax(s, -1)
            size = scale * (x.abs() @ Kr.abs().transpose(1, 2)).amax(-1)[..., None]
            err = (d + 8) * 2.0**-24 * size + 2.0**-20
            o_r = (p @ Vr)
            out[b, :, r] = o_r.reshape(Hq, d)
            tol[b, :, r] = ((weight + 2 * err + 2.0**-18) * (p @ Vr.abs()) + 2.0**-8 * o_r.abs()).reshape(Hq, d)
            lse[b, :, r] = torch.logsumexp(s, -1).reshape(Hq)
            ltol[b, :, r] = (err[..., 0] + 2.0**-20 * (1 + torch.logsumexp(s, -1).abs())).reshape(Hq)
    return out, lse, tol, ltol


def _check(got, ref, what=""):
    out, lse, tol, ltol = ref
    there = ~torch.isnan(lse)
    _within(got[0].cpu()[there], out[there], tol[there], f"{what} out")
    if got[1] is not None:
        _within(got[1].cpu()[there], lse[there], ltol[there], f"{what} lse")


@pytest.mark.parametrize("n_split", [1, 3, None])
@pytest.mark.parametrize("B,Hq,Hkv,L,Lq,off,seeds,d", [
    (1, 1, 1, 1, 1, 0, 0, 128), (1, 1, 1, 1, 1, 0, 1, 64), (1, 2, 1, 33, 1, 32, 0, 128), (2, 4, 4, 64, 64, 0, 20, 128),
    (1, 28, 4, 300, 1, 299, 1, 128), (1, 28, 4, 300, 5, 100, 2, 64), (2, 8, 2, 200, 37, 50, 9, 128),
    (1, 4, 4, 1024, 64, 832, 16, 128), (1, 4, 2, 513, 100, 413, 40, 64), (3, 2, 2, 95, 31, 31, 31, 128),
    (1, 3, 3, 2100, 7, 2000, 3, 128), (1, 2, 2, 700, 256, 200, 100, 128), (1, 12, 12, 64, 33, 0, 0, 64),
    (1, 5, 1, 130, 13, 117, 12, 128),
])
def test_attention(n_split, B, Hq, Hkv, L, Lq, off, seeds, d):
    announce(f"attn_cached split {n_split} B{B} H{Hq}/{Hkv} L{L} Lq{Lq} off{off} seeds{seeds} d{d}")
    t = _problem(L + Lq, B, Hq, Hkv, L, Lq, d, seeds, off)
    got = _call(t, n_split=n_split)
    torch.cuda.synchronize()
    _check(got, _reference(t))
    again = _call(t, n_split=n_split, want_lse=False)
    assert _same(again[0], got[0]) and again[1] is None


@pytest.mark.parametrize("n_split", [1, 4])
@pytest.mark.parametrize("d", [128, 64])
def test_rows_of_different_lengths(n_split, d):
    """A padded batch: lengths from 0 to the whole cache, blocks that stick out past the end, start at it
    or are cut by it; rows that do not exist are left as they were, keys past the end never read."""
    announce(f"attn_cached ragged split {n_split} d{d}")
    lens, offs = [400, 0, 1, 333, 333, 40, 400, 70, -3, 900], [300, 0, 0, 300, 333, 0, 0, 10, 0, 390]
    t = _problem(11, 10, 6, 2, 400, 40, d, 10, offs, lens)
    out = torch.full((10, 6, 40, d), 7.0, device="cuda", dtype=BF16)
    lse = torch.full((10, 6, 40), 9.0, device="cuda")
    got = _call(t, n_split=n_split, out=out, lse=lse)
    torch.cuda.synchronize()
    assert got[0] is out and got[1] is lse
    ref = _reference(t)
    _check(got, ref, "ragged")
    gone = torch.isnan(ref[1]).cuda()
    assert gone.any() and (out[gone] == 7).all() and (lse[gone] == 9).all()
    # poison everything that no row may read
    kc, vc, ks, vs = (x.clone() for x in t["cache"])
    for b, (n, o) in enumerate(zip(lens, offs)):
        n = min(max(n, 0), 400)
        o = min(o, n)
        seeds = set(t["idx"][b, :int(t["n"][b])].tolist())
        dead = [j for j in range(400) if j >= n or (o <= j < o + 40 and j not in seeds)]
        for c, s in ((kc, ks), (vc, vs)):
            c.view(torch.uint8)[b, :, dead] = 0x7F
            s[b, :, dead] = math.nan
        t["k"][b, :, max(0, n - o):] = math.nan
        t["v"][b, :, max(0, n - o):] = math.inf
    t["cache"] = (kc, vc, ks, vs)
    poisoned = _call(t, n_split=n_split)
    assert _same(poisoned[0][~gone], out[~gone]) and _same(poisoned[1][~gone], lse[~gone])


@pytest.mark.parametrize("n_split", [1, 2])
def test_masked_places_may_hold_anything(n_split):
    """A seed's own cached row is hidden from that row alone, its live row from all others."""
    announce(f"attn_cached poison split {n_split}")
    t = _problem(5, 1, 4, 2, 300, 40, 128, 6, 200)
    clean = _call(t, n_split=n_split)
    seed = int(t["idx"][0, 2]) - 200
    others = [r for r in range(40) if r != seed]
    kc, vc, ks, vs = (x.clone() for x in t["cache"])
    for c, s in ((kc, ks), (vc, vs)):
        c.view(torch.uint8)[0, :, 200 + seed] = 0x7F
        s[0, :, 200 + seed] = math.nan
    got = _call({**t, "cache": (kc, vc, ks, vs)}, n_split=n_split)
    assert _same(got[0][:, :, seed], clean[0][:, :, seed]) and _same(got[1][:, :, seed], clean[1][:, :, seed])
    assert torch.isnan(got[0][:, :, others]).all()
    only_v = _call({**t, "cache": (t["cache"][0], vc, t["cache"][2], vs)}, n_split=n_split)
    assert _same(only_v[0][:, :, seed], clean[0][:, :, seed]) and torch.isnan(only_v[0][:, :, others]).all()
    for bad in (math.nan, math.inf, -math.inf):
        k, v = t["k"].clone(), t["v"].clone()
        k[:, :, seed], v[:, :, seed] = bad, bad
        got = _call({**t, "k": k, "v": v}, n_split=n_split)
        assert _same(got[0][:, :, others], clean[0][:, :, others]) and _same(got[1][:, :, others], clean[1][:, :, others])


def test_seed_lists_as_sets():
    announce("attn_cached seed lists")
    t = _problem(8, 1, 4, 4, 200, 50, 64, 5, 100)
    want = _call(t)
    idx = t["idx"][0].tolist()
    odd = torch.tensor([[*reversed(idx), idx[0], idx[0], -1, 500, 3, 199, 99, 150]], device="cuda", dtype=torch.int32)
    got = _call({**t, "idx": odd, "n": torch.tensor([99], device="cuda", dtype=torch.int32)})
    assert _same(got[0], want[0])  # any order, repeats; outside the block or the cache: no effect
    none = _call({**t, "idx": None, "n": None})
    zero = _call({**t, "n": torch.tensor([-4], device="cuda", dtype=torch.int32)})
    assert _same(none[0], zero[0]) and not _same(none[0], want[0])


@pytest.mark.parametrize("grow", [1.0, 40.0])
def test_scores_that_grow_and_scales(grow):
    """Scores whose maximum keeps rising over the keys, large ones, and another score scale."""
    announce(f"attn_cached growing scores {grow}")
    t = _problem(4, 1, 2, 2, 600, 33, 128, 4, 500)
    r = _gen(44)
    k = r(1, 2, 600, 128) * torch.linspace(0.1, grow, 600, device="cuda")[:, None]
    cover.cover_cache_store(k, r(1, 2, 600, 128), 0, *t["cache"])
    for split in (1, 5):
        _check(_call(t, n_split=split), _reference(t), "default scale")
        _check(_call(t, n_split=split, scale=0.3), _reference(t, 0.3), "scale 0.3")


def test_rows_of_unlike_scale():
    """Cache rows whose scales span 2^24: the weights' rounding stays relative to each row."""
    announce("attn_cached scales")
    t = _problem(6, 1, 4, 2, 400, 20, 64, 3, 380, spread=4.0)
    _check(_call(t), _reference(t))


def test_agrees_with_block_attention_where_nothing_is_lost():
    """Keys and values that e4m3 holds exactly: cover_attn_rect on the same numbers in bf16."""
    announce("attn_cached against attn_rect")
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    B, Hq, Hkv, L, Lq, off = 2, 8, 4, 500, 45, 301
    def small():
        x = torch.randint(-7, 8, (B, Hkv, L, 128), generator=g, device="cuda").float() / 4
        x[..., 0] = 7.0 / 4  # every row's scale the same power of two times 1.75 / 448: codes exact
        return x.to(BF16)
    kl, vl, kc, vc = small(), small(), small(), small()
    q = torch.randn(B, Hq, Lq, 128, generator=g, device="cuda").to(BF16)
    idx = torch.tensor([[301, 310, 345], [320, 321, 340]], device="cuda", dtype=torch.int32)
    n = torch.tensor([3, 3], device="cuda", dtype=torch.int32)
    cache = _empty_cache(B, Hkv, L, 128)
    cover.cover_cache_store(kl, vl, 0, *cache)  # outside the block the live states are the prefix
    cover.cover_cache_store(kc[:, :, off:off + Lq], vc[:, :, off:off + Lq], off, *cache)
    back = cover.cover_cache_load(*cache, off, n=Lq)
    assert _same(back[0], kc[:, :, off:off + Lq]) and _same(back[1], vc[:, :, off:off + Lq])
    want, wl = cover.cover_attn_rect(q, kl, vl, kc, vc, off, idx, n)
    t = {"q": q, "k": kl[:, :, off:off + Lq], "v": vl[:, :, off:off + Lq], "cache": cache, "off": off, "idx": idx,
         "n": n, "len": None}
    got, gl = _call(t)
    ref = _reference(t)
    _check((got, gl), ref)
    _within(got.cpu(), want.double().cpu(), 2 * ref[2], "against attn_rect")


# ---- together --------------------------------------------------------------------------------
def _layer(r, B=2, L=96, Lq=32, Hq=8, Hkv=2, d=64, off=64):
    D = Hq * d
    return {"B": B, "L": L, "Lq": Lq, "Hq": Hq, "Hkv": Hkv, "d": d, "off": off,
            "x": r(B, L, D).to(BF16), "res": r(B, L, D).to(BF16), "w": (1 + 0.1 * r(D)).to(BF16),
            "wqkv": (r(D, (Hq + 2 * Hkv) * d) * D**-0.5).to(BF16),
            "freq": cover.rope_freq(d, device="cuda"), "cache": _empty_cache(B, Hkv, L, d),
            "idx": torch.tensor([[70, 80, 95], [64, 81, 82]], device="cuda", dtype=torch.int32)[:B],
            "n": torch.tensor([3, 2], device="cuda", dtype=torch.int32)[:B]}


def _project(p, x, res, pos, rope_args=()):
    """norm -> fused projection -> rotary positions: (q, k, v, residual)."""
    B, n = x.shape[:2]
    h, ro, _ = cover.cover_rms_norm(x.reshape(B * n, -1), p["w"], res.reshape(B * n, -1))
    qkv = (h @ p["wqkv"]).view(B, n, p["Hq"] + 2 * p["Hkv"], p["d"])
    q, k, v = (t.transpose(1, 2) for t in qkv.split([p["Hq"], p["Hkv"], p["Hkv"]], 2))
    q, k = cover.cover_rope(q, k, pos, p["freq"], *rope_args)
    return q, k, v, ro


def _decode(p):
    """The prefix into the cache, then one block against it, then the block into the cache."""
    at = torch.arange(p["L"], device="cuda", dtype=torch.int32)
    _, k, v, _ = _project(p, p["x"], p["res"], at)
    cover.cover_cache_store(k, v, 0, *p["cache"])
    s = slice(p["off"], p["off"] + p["Lq"])
    q, k, v, ro = _project(p, p["x"][:, s] * 0.5, p["res"][:, s], at[s])
    out, lse = cover.cover_attn_cached(q, k, v, *p["cache"], p["off"], p["idx"], p["n"])
    step = [t.clone() for t in p["cache"]]
    cover.cover_cache_store(k, v, p["off"], *p["cache"])
    return q, k, v, ro, out, lse, step


def test_a_layer_of_them():
    """The operators in a row as a decoding layer calls them, each held against its own inputs."""
    announce("layer of the operators")
    p = _layer(_gen(21))
    q, k, v, ro, out, lse, cache = _decode(p)
    torch.cuda.synchronize()
    _check((out, lse), _reference({"q": q, "k": k, "v": v, "cache": cache, "off": p["off"], "len": None, "idx": p["idx"],
                                   "n": p["n"]}), "layer")
    s = slice(p["off"], p["off"] + p["Lq"])
    h = (p["x"][:, s] * 0.5).double() + p["res"][:, s].double()
    _within(ro.view(h.shape), h, (2.0**-8 + 2.0**-24) * h.abs(), "residual")
    # the block's rows are in the cache now, the prefix is as it was
    back, _ = cover.cover_cache_load(*p["cache"], p["off"], n=p["Lq"])
    top = k.double().abs().amax(-1, keepdim=True)
    _within(back, k.double(), (2.0**-4 + 2.0**-7) * k.double().abs() + 2.0**-10 * top / 448, "stored block")
    for a, b in zip(p["cache"], cache):
        assert _same(a[:, :, :p["off"]], b[:, :, :p["off"]])


def test_layer_in_a_graph():
    """Captured and replayed with eager work between the replays; inputs changed in place."""
    announce("layer in a graph")
    p = _layer(_gen(22))
    want = [t.clone() for t in _decode(p)[3:6]]
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        _decode(p)
    stream.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        got = _decode(p)[3:6]
    x = p["x"].clone()
    for rep in range(4):
        for t in got:
            t.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(_same(a, b) for a, b in zip(got, want)), f"replay {rep}"
        p["x"].copy_(x + rep + 1)
        want = [t.clone() for t in _decode(p)[3:6]]
        torch.cuda.synchronize()
    assert not _same(got[1], want[1])


@pytest.mark.parametrize("pass_stream", [False, True])
def test_another_stream(pass_stream):
    announce(f"layer operators on another stream {pass_stream}")
    t = _problem(3, 1, 8, 2, 4096, 16, 128, 4, 4000)
    x, w = _rows(_gen(5), 64, 1000, BF16), torch.ones(1000, device="cuda", dtype=BF16)
    pos, freq = torch.arange(16, device="cuda", dtype=torch.int32), cover.rope_freq(128, device="cuda")

    def all_of(**kw):
        cache = tuple(c.clone() for c in t["cache"])
        if kw:
            kw["stream"].wait_stream(torch.cuda.current_stream())
        return (*cover.cover_rms_norm(x, w, x, quantize=True, **kw), *cover.cover_rope(t["q"], t["k"], pos, freq, **kw),
                *cover.cover_cache_store(t["k"], t["v"], 7, *cache, **kw), *cover.cover_cache_load(*cache, 0, n=40, **kw),
                *_call({**t, "cache": cache}, n_split=4, **kw))

    want = all_of()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    if pass_stream:
        got = all_of(stream=s)
    else:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got = all_of()
    s.synchronize()
    torch.cuda.synchronize()
    assert all(_same(a, b) for a, b in zip(got, want))


def test_two_calls_at_once():
    """Two streams, each with its own workspace and outputs, on shared inputs."""
    announce("two calls at once")
    t = _problem(3, 1, 8, 2, 8192, 16, 128, 4, 8000)
    want = _call(t, n_split=16)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(10):
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got.append(_call(t, n_split=16))
    torch.cuda.synchronize()
    assert all(_same(a, want[0]) and _same(b, want[1]) for a, b in got)


def test_workspaces():
    announce("attn_cached workspaces")
    t = _problem(9, 1, 4, 4, 8192, 8, 128, 2, 8000)
    n = cover.attn_cached_splits(1, 4, 4, 8192, 8)
    assert n > 2
    want = _reference(t)
    for floats in (cover.attn_cached_workspace(1, 4, 8, 128, n), cover.attn_cached_workspace(1, 4, 8, 128, 2), 5):
        _check(_call(t, workspace=torch.full((floats,), math.nan, device="cuda")), want)
    with pytest.raises(ValueError):
        _call(t, n_split=n, workspace=torch.empty(100, device="cuda"))


@pytest.mark.parametrize("python_form", [False, True])
def test_binding_errors_and_forms(python_form):
    announce(f"layer binding errors, python form {python_form}")
    t = _problem(2, 2, 4, 2, 64, 8, 64, 2, 8)
    q, k, v, c = t["q"], t["k"], t["v"], t["cache"]
    x = _rows(_gen(1), 4, 100, BF16)
    pos, freq = torch.zeros(2, 8, device="cuda", dtype=torch.int32), cover.rope_freq(64, device="cuda")
    CE = cover.CoverError
    bad = [
        (TypeError, lambda: cover.cover_rms_norm(x.half())), (ValueError, lambda: cover.cover_rms_norm(x[0])),
        (ValueError, lambda: cover.cover_rms_norm(x, x[:, 0])), (ValueError, lambda: cover.cover_rms_norm(x, None, x[:3])),
        (ValueError, lambda: cover.cover_rms_norm(x, None, x.float())), (CE, lambda: cover.cover_rms_norm(x, eps=-1.0)),
        (CE, lambda: cover.cover_rms_norm(x.contiguous()[:, 1:])), (ValueError, lambda: cover.cover_rms_norm(x, scale=x)),
        (ValueError, lambda: cover.cover_rms_norm(x, residual_out=x)), (ValueError, lambda: cover.cover_rms_norm(x.cpu())),
        (ValueError, lambda: cover.cover_rms_norm(x, quantize=True, out=x)),
        (TypeError, lambda: cover.cover_rope(q.half(), None, pos, freq)), (ValueError, lambda: cover.cover_rope(q, k[:1], pos, freq)),
        (ValueError, lambda: cover.cover_rope(q, k, pos.long(), freq)), (ValueError, lambda: cover.cover_rope(q, k, pos[:, :3], freq)),
        (ValueError, lambda: cover.cover_rope(q, k, pos, freq.float())), (ValueError, lambda: cover.cover_rope(q, k, pos, freq.cpu())),
        (CE, lambda: cover.cover_rope(q, k, pos, torch.cat((freq, freq)))), (ValueError, lambda: cover.cover_rope(q, None, pos, freq, k_out=k)),
        (CE, lambda: cover.cover_rope(q, k, pos, freq, attention_factor=math.inf)),
        (ValueError, lambda: cover.cover_cache_store(k, v[:1], 0, *c)), (ValueError, lambda: cover.cover_cache_store(k, v, pos[:1], *c)),
        (ValueError, lambda: cover.cover_cache_store(k, v, pos, c[0].view(torch.uint8), *c[1:])),
        (CE, lambda: cover.cover_cache_store(k, v, 60, *c)), (CE, lambda: cover.cover_cache_store(k, v, -1, *c)),
        (ValueError, lambda: cover.cover_cache_store(k, v, 0, *c[:3], c[3][:, :1])), (ValueError, lambda: cover.cover_cache_store(k, v.float(), 0, *c)),
        (ValueError, lambda: cover.cover_cache_load(*c, 0)), (ValueError, lambda: cover.cover_cache_load(*c, pos, n=3)),
        (CE, lambda: cover.cover_cache_load(*c, 60, n=5)), ((TypeError, ValueError), lambda: cover.cover_cache_load(*c, 0, n=5, dtype=torch.float16)),
        (ValueError, lambda: cover.cover_cache_load(*c, 0, n=5, k=k)),
        (TypeError, lambda: cover.cover_attn_cached(q.float(), k, v, *c, 8)), (ValueError, lambda: cover.cover_attn_cached(q, k, v[:, :1], *c, 8)),
        (CE, lambda: cover.cover_attn_cached(q, k, v, *c, 57)), (CE, lambda: cover.cover_attn_cached(q, k, v, *c, -1)),
        (CE, lambda: cover.cover_attn_cached(q[:, :3], k, v, *c, 8)), (CE, lambda: cover.cover_attn_cached(q, k, v, *c, 8, scale=-1.0)),
        (CE, lambda: cover.cover_attn_cached(q, k, v, *c, 8, n_split=0)), (ValueError, lambda: cover.cover_attn_cached(q, k, v, *c, 8, t["idx"])),
        (ValueError, lambda: cover.cover_attn_cached(q, k, v, *c, 8, t["idx"].long(), t["n"])),
        (ValueError, lambda: cover.cover_attn_cached(q, k, v, *c, 8, kv_len=t["n"].long())),
        (ValueError, lambda: cover.cover_attn_cached(q, k, v, *c, 8, out=q.float())),
        (ValueError, lambda: cover.cover_attn_cached(q, k, v, *(y.cpu() for y in c), 8)),
    ]
    for kind, call in bad:
        with pytest.raises(kind):
            if python_form:
                with torch.device("cuda"):
                    call()
            else:
                call()
    if python_form:  # the two forms of a call agree
        calls = [lambda: cover.cover_rms_norm(x, x[0].contiguous(), x, quantize=True), lambda: cover.cover_rms_norm(x),
                 lambda: cover.cover_rope(q, k, pos, freq), lambda: cover.cover_cache_store(k, v, 3, *c),
                 lambda: cover.cover_cache_load(*c, pos), lambda: cover.cover_cache_load(*c, 5, n=3, dtype=F32),
                 lambda: _call(t), lambda: _call({**t, "off": t["n"]}, n_split=3, want_lse=False)]
        for call in calls:
            a = call()
            with torch.device("cuda"):
                b = call()
            for y, z in zip(a, b):
                assert (y is None) == (z is None)
                if y is not None:
                    assert y.stride() == z.stride() and y.dtype == z.dtype and _same(y, z)


def test_debug_checks(monkeypatch):
    announce("layer debug checks")
    monkeypatch.setenv("COVER_DEBUG", "1")
    cover.debug_status(clear=True)
    t = _problem(2, 1, 4, 2, 64, 8, 64, 2, 8)
    _call(t)
    pos = torch.tensor([[5, -1, -1, 7, 99, 99, 3, 63]], device="cuda", dtype=torch.int32)
    cover.cover_cache_store(t["k"], t["v"], pos, *t["cache"])
    assert cover.debug_status() == 0
    pos[0, 6] = 7
    cover.cover_cache_store(t["k"], t["v"], pos, *t["cache"])
    assert cover.debug_status(clear=True) == cover.COVER_DEBUG_STORE_DUPLICATE
    _call({**t, "idx": torch.tensor([[9, 9]], device="cuda", dtype=torch.int32)})
    assert cover.debug_status(clear=True) == cover.COVER_DEBUG_SEED_DUPLICATE


def test_empty_calls():
    announce("layer empty calls")
    z = torch.empty(0, 64, device="cuda", dtype=BF16)
    assert cover.cover_rms_norm(z, quantize=True)[0].shape == (0, 64)
    t = _problem(2, 1, 4, 2, 64, 8, 64, 2, 8)
    out, lse = cover.cover_attn_cached(t["q"][:, :, :0], t["k"][:, :, :0], t["v"][:, :, :0], *t["cache"], 64)
    assert out.shape == (1, 4, 0, 64) and lse.shape == (1, 4, 0)
    cover.cover_cache_store(t["k"][:0], t["v"][:0], 0, *(c[:0] for c in t["cache"]))
    torch.cuda.synchronize()


@pytest.mark.parametrize("B,Hq,Hkv,L,Lq,off,seeds,d", [
    (5, 32, 32, 300, 256, 44, 200, 128), (3, 64, 64, 150, 130, 11, 3, 64), (40, 16, 4, 100, 70, 30, 0, 128),
    (2, 96, 96, 97, 33, 64, 33, 128), (2, 32, 32, 200, 200, 0, 70, 128),
])
def test_attention_many_rows(B, Hq, Hkv, L, Lq, off, seeds, d):
    """Enough tiles that a workgroup takes 64 query rows."""
    announce(f"attn_cached many rows B{B} H{Hq}/{Hkv} L{L} Lq{Lq} d{d}")
    t = _problem(L + Lq, B, Hq, Hkv, L, Lq, d, seeds, off)
    got = _call(t)
    torch.cuda.synchronize()
    for b in (0, B - 1):  # the reference is slow: the first and the last batch row
        part = {k: v if isinstance(v, int) or v is None else v[b:b + 1] for k, v in t.items() if k != "cache"}
        part["cache"] = tuple(c[b:b + 1] for c in t["cache"])
        _check((got[0][b:b + 1], got[1][b:b + 1]), _reference(part), f"row {b}")
    again = _call(t, want_lse=False)
    assert _same(again[0], got[0])


@pytest.mark.parametrize("d", [128, 64])
def test_many_rows_of_different_lengths(d):
    announce(f"attn_cached many ragged rows d{d}")
    B, Hq, Hkv, L, Lq = 24, 16, 8, 140, 100
    lens = [140 - 6 * b for b in range(B)]
    offs = [max(0, n - 60) if b % 3 else max(0, n - 100) for b, n in enumerate(lens)]
    t = _problem(12, B, Hq, Hkv, L, Lq, d, 9, offs, lens)
    out = torch.full((B, Hq, Lq, d), 7.0, device="cuda", dtype=BF16)
    lse = torch.full((B, Hq, Lq), 9.0, device="cuda")
    _call(t, out=out, lse=lse)
    torch.cuda.synchronize()
    ref = _reference(t)
    _check((out, lse), ref, "many ragged")
    gone = torch.isnan(ref[1]).cuda()
    assert (out[gone] == 7).all() and (lse[gone] == 9).all()
    kc, vc, ks, vs = (x.clone() for x in t["cache"])
    for b, (n, o) in enumerate(zip(lens, offs)):
        seeds = set(t["idx"][b, :int(t["n"][b])].tolist())
        dead = [j for j in range(L) if j >= n or (o <= j < o + Lq and j not in seeds)]
        for c, s in ((kc, ks), (vc, vs)):
            c.view(torch.uint8)[b, :, dead] = 0x7F
            s[b, :, dead] = math.nan
        t["k"][b, :, n - o:] = math.nan
        t["v"][b, :, n - o:] = math.inf
    poisoned = _call({**t, "cache": (kc, vc, ks, vs)})
    assert _same(poisoned[0][~gone], out[~gone]) and _same(poisoned[1][~gone], lse[~gone])


def test_many_rows_masked_places_may_hold_anything():
    announce("attn_cached many rows poison")
    t = _problem(5, 3, 64, 64, 300, 200, 128, 70, 90)
    clean = _call(t)
    seed = int(t["idx"][0, 2]) - 90
    others = [r for r in range(200) if r != seed]
    _, vc, _, vs = (x.clone() for x in t["cache"])
    vc.view(torch.uint8)[0, :, 90 + seed] = 0x7F
    vs[0, :, 90 + seed] = math.nan
    got = _call({**t, "cache": (t["cache"][0], vc, t["cache"][2], vs)})
    assert _same(got[0][0, :, seed], clean[0][0, :, seed]) and _same(got[0][1:], clean[0][1:])
    assert torch.isnan(got[0][0][:, others]).all()
    k, v = t["k"].clone(), t["v"].clone()
    k[0, :, seed], v[0, :, seed] = math.nan, math.inf
    got = _call({**t, "k": k, "v": v})
    assert _same(got[0][0][:, others], clean[0][0][:, others]) and _same(got[1][0][:, others], clean[1][0][:, others])
    assert _same(got[0][1:], clean[0][1:])


@pytest.mark.parametrize("B,Hq,Hkv,L,Lq,off,seeds", [
    (8, 32, 32, 300, 250, 44, 100), (16, 48, 16, 130, 83, 9, 0), (16, 64, 16, 97, 64, 33, 33), (8, 32, 32, 256, 256, 0, 256),
    (4, 64, 64, 700, 225, 450, 70), (9, 32, 32, 129, 129 + 96, 0, 1),
])
def test_attention_in_workgroups_of_128_rows(B, Hq, Hkv, L, Lq, off, seeds):
    """So many rows that each wave of a workgroup has 32 of its own."""
    announce(f"attn_cached 128 rows B{B} H{Hq}/{Hkv} L{L} Lq{Lq}")
    L = max(L, off + Lq)
    t = _problem(L + Lq, B, Hq, Hkv, L, Lq, 128, seeds, off)
    got = _call(t)
    torch.cuda.synchronize()
    for b in (0, B - 1):
        part = {k: v if isinstance(v, int) or v is None else v[b:b + 1] for k, v in t.items() if k != "cache"}
        part["cache"] = tuple(c[b:b + 1] for c in t["cache"])
        _check((got[0][b:b + 1], got[1][b:b + 1]), _reference(part), f"row {b}")
    again = _call(t, want_lse=False)
    assert _same(again[0], got[0])


def test_128_rows_ragged_and_masked():
    """Rows of different lengths, from whole blocks to none; what is not a row's own key may hold anything."""
    announce("attn_cached 128 rows ragged")
    B, Hq, Hkv, L, Lq, d = 16, 48, 16, 150, 83, 128
    lens = [150 - 10 * b if b < 15 else 0 for b in range(B)]
    offs = [max(0, n - (90, 60, 17)[b % 3]) for b, n in enumerate(lens)]
    t = _problem(12, B, Hq, Hkv, L, Lq, d, 9, offs, lens)
    out = torch.full((B, Hq, Lq, d), 7.0, device="cuda", dtype=BF16)
    lse = torch.full((B, Hq, Lq), 9.0, device="cuda")
    _call(t, out=out, lse=lse)
    torch.cuda.synchronize()
    ref = _reference(t)
    _check((out, lse), ref, "128 rows ragged")
    gone = torch.isnan(ref[1]).cuda()
    assert gone[15].all() and (out[gone] == 7).all() and (lse[gone] == 9).all()
    kc, vc, ks, vs = (x.clone() for x in t["cache"])
    for b, (n, o) in enumerate(zip(lens, offs)):
        seeds = set(t["idx"][b, :int(t["n"][b])].tolist())
        dead = [j for j in range(L) if j >= n or (o <= j < o + Lq and j not in seeds)]
        for c, s in ((kc, ks), (vc, vs)):
            c.view(torch.uint8)[b, :, dead] = 0x7F
            s[b, :, dead] = math.nan
        t["k"][b, :, n - o:] = math.nan
        t["v"][b, :, n - o:] = math.inf
    poisoned = _call({**t, "cache": (kc, vc, ks, vs)})
    assert _same(poisoned[0][~gone], out[~gone]) and _same(poisoned[1][~gone], lse[~gone])


def test_128_rows_seed_that_is_nan():
    """A seed whose cached value is NaN reaches every row but its own, one whose live value is reaches its own alone."""
    announce("attn_cached 128 rows poison")
    t = _problem(5, 4, 64, 64, 300, 225, 128, 70, 60)
    clean = _call(t)
    seed = int(t["idx"][0, 2]) - 60
    others = [r for r in range(225) if r != seed]
    _, vc, _, vs = (x.clone() for x in t["cache"])
    vc.view(torch.uint8)[0, :, 60 + seed] = 0x7F
    vs[0, :, 60 + seed] = math.nan
    got = _call({**t, "cache": (t["cache"][0], vc, t["cache"][2], vs)})
    assert _same(got[0][0, :, seed], clean[0][0, :, seed]) and _same(got[0][1:], clean[0][1:])
    assert torch.isnan(got[0][0][:, others]).all()
    k, v = t["k"].clone(), t["v"].clone()
    k[0, :, seed], v[0, :, seed] = math.nan, math.inf
    got = _call({**t, "k": k, "v": v})
    assert _same(got[0][0][:, others], clean[0][0][:, others]) and _same(got[1][0][:, others], clean[1][0][:, others])
    assert _same(got[0][1:], clean[0][1:])


def test_workspace_of_another_stream():
    """A call on a stream that is not the current one takes its workspace from that stream: what the current
    stream allocates right after does not share its memory."""
    announce("attn_cached workspace of another stream")
    t = _problem(3, 1, 32, 8, 8192, 1, 128, 0, 8191)
    want = _call(t)
    n = cover.attn_cached_splits(1, 32, 8, 8192, 1)
    assert n > 1
    floats = cover.attn_cached_workspace(1, 32, 1, 128, n)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (s, s.cuda_stream):
        for _ in range(20):
            got = _call(t, stream=stream)
            junk = torch.full((floats,), math.nan, device="cuda")
            s.synchronize()
            assert _same(got[0], want[0]) and _same(got[1], want[1])
            del junk


@pytest.mark.parametrize("B,Hq,Hkv,L,Lq,off,d", [
    (1, 8, 2, 4000, 8, 2000, 128), (2, 16, 16, 700, 64, 636, 64), (1, 4, 4, 200, 200, 0, 128), (8, 32, 32, 330, 250, 80, 128),
])
def test_weights_have_more_bits_than_bf16(B, Hq, Hkv, L, Lq, off, d):
    """Cached keys' weights are rounded to fp16 (half a step: 2^-11), live ones' to two parts of bf16 (2^-16), or
    both are below 2^-24 of the row's largest; then the output's own rounding, half a step of bf16."""
    announce(f"attn_cached weights L{L} Lq{Lq} d{d}")
    t = _problem(L + d, B, Hq, Hkv, L, Lq, d, 0, off)
    got = _call(t)
    for b in (0, B - 1):
        part = {k: v if isinstance(v, int) or v is None else v[b:b + 1] for k, v in t.items() if k != "cache"}
        part["cache"] = tuple(c[b:b + 1] for c in t["cache"])
        out, _, tol, _ = _reference(part, weight=2.0**-11)
        V = part["cache"][1].cpu().double() * part["cache"][3].cpu().double()[..., None]
        size = torch.maximum(V.abs().amax((2, 3)), part["v"].abs().double().cpu().amax((2, 3)))
        size = size.repeat_interleave(Hq // Hkv, 1)[..., None, None]
        _within(got[0][b:b + 1].cpu(), out, tol + L * 2.0**-24 * size, "weights")


@pytest.mark.parametrize("n_split", [1, 4])
def test_small_weights_count(n_split):
    """One key takes almost all of the weight but has no value: the output is what the others leave, whose
    weights are 2^-17 of it.  Each is off by at most 2^-11 of itself or 2^-25 in units where the largest is 2^3."""
    announce("attn_cached small weights")
    L, Lq, d = 1500, 4, 128
    r = _gen(4)
    q = torch.zeros(1, 1, Lq, d, device="cuda", dtype=BF16)
    q[..., 0] = 1.0
    k = torch.zeros(1, 1, L, d, device="cuda", dtype=BF16)
    k[0, 0, 700, 0] = 17 * math.log(2) * d**0.5
    v = (1 + 0.25 * r(1, 1, L, d)).to(BF16)
    v[0, 0, 700] = 0
    cache = _empty_cache(1, 1, L, d)
    cover.cover_cache_store(k, v, 0, *cache)
    live = torch.zeros(1, 1, Lq, d, device="cuda", dtype=BF16)
    got, _ = cover.cover_attn_cached(q, live, live, *cache, L - Lq, n_split=n_split)
    K, V = (cache[i].cpu().double() * cache[2 + i].cpu().double()[..., None] for i in (0, 1))
    K[:, :, L - Lq:], V[:, :, L - Lq:] = 0, 0
    s = (q.cpu().double() @ K.transpose(2, 3)) * d**-0.5
    p = torch.softmax(s, -1)
    want = p @ V
    # the scores' own rounding: 17 log2 units in fp32, 2^-19 relative of each weight
    tol = (2.0**-8 + 2.0**-11 + 2.0**-17) * want.abs() + 2.0**-28 * 4 * V.abs().sum(2, keepdim=True)
    _within(got.cpu(), want, tol.expand_as(want), "small weights")


@pytest.mark.parametrize("n_split", [1, 2])
@pytest.mark.parametrize("size", [2.0**-20, 2.0**30, 2.0**100])
def test_values_of_any_size(n_split, size):
    """Values of one size, whatever it is: the rounding is relative to it (weights half a step of fp16, 2^-11)."""
    announce(f"attn_cached values of size {size} n_split {n_split}")
    t = _problem(21, 2, 8, 4, 300, 40, 128, 6, 130)
    r = _gen(22)
    t["v"] = (t["v"].float() * size).to(BF16)
    cover.cover_cache_store((r(2, 4, 300, 128)).to(BF16), (r(2, 4, 300, 128) * size).to(BF16), 0, *t["cache"])
    got = _call(t, n_split=n_split)
    out, lse, tol, ltol = _reference(t, weight=2.0**-11)
    V = t["cache"][1].cpu().double() * t["cache"][3].cpu().double()[..., None]
    most = torch.maximum(V.abs().amax(), t["v"].double().cpu().abs().amax())
    _within(got[0].cpu(), out, tol + 300 * 2.0**-24 * most, "values out")
    _within(got[1].cpu(), lse, ltol, "values lse")


@pytest.mark.parametrize("at", [0, 37, 250])
def test_one_value_far_above_the_others(at):
    """A key of almost no weight whose value is 2^12 times the others': their weights are still off by no more than
    2^-11 of themselves or 2^-28 of the largest weight times the largest scale, per code (at most 448)."""
    announce(f"attn_cached one large value at {at}")
    L, Lq, d = 300, 5, 64
    r = _gen(31)
    q, k, v = r(1, 2, Lq, d).to(BF16), r(1, 2, L, d), r(1, 2, L, d)
    k[:, :, at] = -40 * q.float().mean(2) / q.float().mean(2).square().sum(-1, keepdim=True) * d**0.5 / 8
    v[:, :, at] *= 2.0**12
    cache = _empty_cache(1, 2, L, d)
    cover.cover_cache_store(k.to(BF16), v.to(BF16), 0, *cache)
    live = (r(1, 2, Lq, d).to(BF16), r(1, 2, Lq, d).to(BF16))
    t = {"q": q, "k": live[0], "v": live[1], "cache": cache, "off": 295, "len": None, "idx": None, "n": None}
    got = _call(t)
    out, lse, tol, ltol = _reference(t, weight=2.0**-11)
    codes = cache[1].float().abs().sum(2).cpu().double()[:, :, None]
    _within(got[0].cpu(), out, tol + 2.0**-28 * cache[3].max().item() * codes, "one value out")
    _within(got[1].cpu(), lse, ltol, "one value lse")
