"""The attention kernels on scores far from zero (up to 2^110, where neighbouring fp32 numbers are far apart): a row
whose best key leads by more than the others' rounding is that key's value.

Tolerances: the output's rounding to its type and the weights' of the bf16 kernels (half a step of bf16, 2^-8, each),
and 2^-20; lse is the best score, a sum of d products in fp32: (d + 12) 2^-24 relative, since all products have its sign."""
import pytest
import torch

from helpers import announce
from paper_2602_06161_amd import cover

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("late", [False, True])
@pytest.mark.parametrize("size", [2.0**10, 2.0**14, 2.0**50])
@pytest.mark.parametrize("sign", [-1, 1])
@pytest.mark.parametrize("kind,dtype,B,H,L,d", [
    ("fwd", F32, 1, 2, 100, 128), ("fwd", F32, 1, 2, 500, 64), ("fwd", BF16, 1, 2, 100, 128), ("fwd", BF16, 1, 2, 200, 64),
    ("fwd", BF16, 2, 32, 512, 128), ("fwd", BF16, 2, 32, 500, 64), ("fwd", BF16, 40, 32, 20, 128), ("rect", BF16, 1, 2, 512, 128),
    ("split", BF16, 1, 2, 4096, 128),
])
def test_the_best_key_takes_the_row(kind, dtype, B, H, L, d, sign, size, late):
    """late: the first 64 keys' scores are small, the others' far away."""
    announce(f"far scores {kind} {dtype} B{B} H{H} L{L} d{d} sign {sign} q {size} late {late}")
    g = torch.Generator(device="cuda")
    g.manual_seed(L + d)
    u = lambda *shape: torch.rand(*shape, generator=g, device="cuda")  # noqa: E731
    q = (size * (1 + 0.3 * u(B, H, L, d))).to(dtype)
    k = sign * 16 * size * (1 + 0.1 * u(B, H, L, d))
    best = 11 if sign < 0 or L < 100 else 90
    k[:, :, best] *= 0.5 if sign < 0 else 2.0
    if late:
        k[:, :, [j for j in range(min(L, 64)) if j != best]] *= 2.0**-20 if sign > 0 else 1.0
    k, v = k.to(dtype), (u(B, H, L, d) + 1).to(dtype)
    idx = torch.full((B, 1), L - 2, device="cuda", dtype=torch.int32)  # a seed with the same state in both
    n = torch.ones(B, device="cuda", dtype=torch.int32)
    if kind == "fwd":
        rows = slice(0, L)
        out, lse = cover.cover_attn_fwd(q, k, v, k, v, idx, n)
    else:
        rows = slice(L - 70, L)
        out, lse = cover.cover_attn_rect(q[:, :, rows].contiguous(), k, v, k, v, L - 70, idx, n, n_split=8 if kind == "split" else 1)
    torch.cuda.synchronize()
    want = v[:, :, best, None].double().expand_as(out)
    tol = (2.0**-20 + (2.0**-7 if dtype == BF16 else 0.0)) * want
    bad = ~((out.double() - want).abs() <= tol)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, {int(out.isnan().sum())} NaN"
    score = (q[:, :, rows].double() * k[:, :, best, None].double()).sum(-1) * d**-0.5
    bad = ~((lse.double() - score).abs() <= (d + 12) * 2.0**-24 * score.abs())
    assert not bad.any(), f"lse: {int(bad.sum())} of {bad.numel()} off"
