"""Edges of the layer's operators: what lies far from the usual sizes of their inputs.

Tolerances: half a step of bf16 (2^-8 relative) for the output's rounding, 2^-11 for the rounding of a cached
key's weight, 2^-24 for an fp32 operation; a score sums d products, so it is off by (d + 8) 2^-24 of scale sum |q| |k|.
"""
import pytest
import torch

from helpers import announce
from paper_2602_06161_amd import cover
from test_layer_gpu import BF16, _call, _empty_cache, _gen, _problem, _same, _within

pytestmark = pytest.mark.gpu

# B, Hq, Hkv, L, Lq, off: few rows, more of them than a wave has stages of, few with key ranges, and many rows (each
# wave 32 of its own)
FEW, BLOCK, RANGES, MANY = (1, 4, 2, 300, 40, 200), (1, 2, 1, 700, 400, 200), (1, 4, 2, 8192, 4, 8000), (8, 32, 32, 300, 250, 40)


# ---- seeds that are not the block's ----------------------------------------------------------
@pytest.mark.parametrize("size,d", [(FEW, 128), (FEW, 64), (BLOCK, 128), (BLOCK, 64), (RANGES, 128), (RANGES, 64), (MANY, 128)])
def test_only_seeds_outside_the_block(size, d):
    """The cache's rows of the block are not read where no seed names them, whatever finite numbers they hold."""
    announce(f"attn_cached seeds outside the block {size} d{d}")
    B, Hq, Hkv, L, Lq, off = size
    t = _problem(17, B, Hq, Hkv, L, Lq, d, 0, off)
    t["idx"] = torch.tensor([[3, off - 1, off + Lq, 5]], device="cuda", dtype=torch.int32).repeat(B, 1)
    t["n"] = torch.full((B,), 4, device="cuda", dtype=torch.int32)
    want = _call(t)
    none = _call({**t, "idx": None, "n": None})
    _within(want[0], none[0].double(), 2.0**-7 * none[0].double().abs() + 2.0**-18, "no seeds")
    _within(want[1], none[1].double(), 2.0**-18 * (1 + none[1].double().abs()), "no seeds, lse")
    for scale in (2.0**120, 2.0**-120):
        kc, vc, ks, vs = (x.clone() for x in t["cache"])
        for s in (ks, vs):
            s[:, :, off:off + Lq] = scale
        got = _call({**t, "cache": (kc, vc, ks, vs)})
        assert _same(got[0], want[0]) and _same(got[1], want[1]), scale


# ---- scores far below zero -------------------------------------------------------------------
@pytest.mark.parametrize("best", ["cached", "live", "seed"])
@pytest.mark.parametrize("size,d", [(FEW, 128), (FEW, 64), (RANGES, 128), (RANGES, 64), (MANY, 128)])
def test_scores_far_below_zero(size, d, best):
    """Every score below -1e31, one key's (in front of the block, or in it) half of the others': the row is that key's value."""
    announce(f"attn_cached scores far below zero {size} d{d} best {best}")
    B, Hq, Hkv, L, Lq, off = size
    r = _gen(23)
    v, vl = r(B, Hkv, L, d).to(BF16), r(B, Hkv, Lq, d).to(BF16)
    q = torch.full((B, Hq, Lq, d), 2.0**50, device="cuda", dtype=BF16)
    k, kl = torch.full((B, Hkv, L, d), -2.0**54, device="cuda"), torch.full((B, Hkv, Lq, d), -2.0**54, device="cuda")
    seed_row = 2
    if best == "cached":
        k[:, :, 20] /= 2
    elif best == "live":
        kl[:, :, 1] /= 2
    else:
        k[:, :, 20] /= 2
        kl[:, :, seed_row] /= 4  # of its own row alone
    cache = _empty_cache(B, Hkv, L, d)
    cover.cover_cache_store(k.to(BF16), v, 0, *cache)
    t = {"q": q, "k": kl.to(BF16), "v": vl, "cache": cache, "off": off, "len": None,
         "idx": torch.full((B, 1), off + seed_row, device="cuda", dtype=torch.int32),
         "n": torch.ones(B, device="cuda", dtype=torch.int32)}
    out, lse = _call(t)
    torch.cuda.synchronize()
    back = cache[1].double() * cache[3].double()[..., None]
    want = (vl[:, :, 1].double() if best == "live" else back[:, :, 20])[:, :, None].repeat(1, 1, Lq, 1)
    score = torch.full((B, Hkv, Lq), -2.0**103 * d**0.5, device="cuda", dtype=torch.float64)
    if best == "seed":
        want[:, :, seed_row] = vl[:, :, seed_row].double()
        score[:, :, seed_row] /= 2
    want, score = want.repeat_interleave(Hq // Hkv, 1), score.repeat_interleave(Hq // Hkv, 1)
    _within(out, want, (2.0**-8 + 2.0**-11 + 2.0**-18) * want.abs(), "out")
    # (the cached key is its codes times its scale: two fp32 roundings)
    _within(lse, score, (d + 12) * 2.0**-24 * score.abs(), "lse")


@pytest.mark.parametrize("size_of_q", [2.0**10, 2.0**14, 2.0**50])
@pytest.mark.parametrize("sign", [-1, 1])
@pytest.mark.parametrize("size,d", [(FEW, 128), (FEW, 64), (RANGES, 128), (RANGES, 64), (MANY, 128)])
def test_scores_with_steps_beyond_one(size, d, sign, size_of_q):
    """Scores of 2^27 and more, where neighbouring fp32 numbers are 16 apart: the row is the best key's value."""
    announce(f"attn_cached scores of any size {size} d{d} sign {sign} q {size_of_q}")
    B, Hq, Hkv, L, Lq, off = size
    g = torch.Generator(device="cuda")
    g.manual_seed(29)
    u = lambda *shape: torch.rand(*shape, generator=g, device="cuda")  # noqa: E731
    q = (size_of_q * (1 + 0.3 * u(B, Hq, Lq, d))).to(BF16)
    k = sign * 16 * size_of_q * (1 + 0.1 * u(B, Hkv, L, d))
    k[:, :, 20] *= 0.5 if sign < 0 else 2.0
    v = u(B, Hkv, L, d) + 1
    cache = _empty_cache(B, Hkv, L, d)
    cover.cover_cache_store(k, v, 0, *cache)
    block = slice(off, off + Lq)
    out, lse = cover.cover_attn_cached(q, k[:, :, block].to(BF16), v[:, :, block].to(BF16), *cache, off)
    best = [(cache[i].double() * cache[2 + i].double()[..., None])[:, :, 20].repeat_interleave(Hq // Hkv, 1)[:, :, None] for i in (0, 1)]
    _within(out, best[1].expand_as(out), (2.0**-8 + 2.0**-11 + 2.0**-18) * best[1].abs().expand_as(out), "out")
    score = (q.double() * best[0]).sum(-1) * d**-0.5
    _within(lse, score, (d + 12) * 2.0**-24 * score.abs(), "lse")


# ---- products of the norm that leave fp32 ----------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.float32, BF16])
@pytest.mark.parametrize("x_size,w_size,eps", [(1e17, 1e23, 1e-6), (1e-17, 1e-24, 0.0), (1e-12, 1e-30, 0.0), (1e15, 1e-30, 1e-6)])
def test_norm_into_codes_where_row_times_weight_leaves_fp32(dtype, x_size, w_size, eps):
    """x and the weight far from 1: x * weight is beyond fp32, the normed row (about the weight's size) is not."""
    announce(f"norm codes {dtype} x {x_size} w {w_size}")
    r = _gen(7)
    x, w = (x_size * r(5, 1000)).to(dtype), (w_size * (1 + 0.1 * r(1000))).to(dtype)
    q, _, s = cover.cover_rms_norm(x, w, eps=eps, quantize=True)
    h = x.double()
    want = h / torch.sqrt((h * h).mean(1, keepdim=True) + eps) * w.double()
    top = want.abs().amax(1)
    fp32 = 2.0**-24 * (1000 / 128 + 12)
    _within(s, top / 448, (fp32 + 2.0**-23) * top / 448, "scale")
    half = torch.maximum(2.0**-4 * want.abs(), 2.0**-10 * s.double()[:, None])
    _within(q.double() * s.double()[:, None], want, half * (1 + 2.0**-12) + (fp32 + 2.0**-22) * want.abs(), "codes")
