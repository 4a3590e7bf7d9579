"""cover_attn_cached in each form that it runs in: 32, 64 or 128 query rows per workgroup, one launch or key ranges that
a second one joins (one wave per row where the ranges are few, four where they are many), both head sizes.  Every case
names its form and checks it, so that a change of the rules that choose one cannot move a case to another.

Tolerances.  A score sums d products in fp32: off by (d + 8) 2^-24 of scale sum |q| |k|, twice as much relative in a
weight.  A cached key's weight times its value's scale is rounded to fp16: 2^-11 of itself, or 2^-28 of the row's largest
weight times the largest value scale read (at least 2^-30); live rows' weights to 2^-16.  2^-18 for exponentials, sums
and the join, 2^-8 for the output's rounding to bf16."""
import math

import pytest
import torch

from helpers import announce
from paper_2602_06161_amd import cover
from test_layer_gpu import BF16, _call, _empty_cache, _gen, _same, _within

pytestmark = pytest.mark.gpu

# (key ranges, query rows per workgroup) and sizes B, Hq, Hkv, L, Lq that take it
FORMS = [((1, 32), (2, 4, 2, 300, 40)), ((1, 64), (2, 40, 40, 400, 128)), ((6, 32), (3, 8, 2, 2048, 40)),
         ((33, 32), (1, 4, 2, 4096, 4)), ((3, 64), (1, 21, 3, 12000, 200))]
RAGGED = [((1, 32), (8, 4, 2, 300, 40)), ((1, 64), (24, 16, 8, 400, 100)), ((6, 32), (6, 4, 1, 2048, 40)),
          ((33, 32), (3, 2, 1, 4096, 4)), ((3, 64), (3, 7, 1, 12000, 200))]
MANY = ((1, 128), (8, 32, 32, 300, 250))
RAGGED_MANY = ((1, 128), (16, 48, 16, 300, 83))


def _cases(forms, many):
    return [(form, size, d) for form, size in forms for d in (128, 64)] + [(*many, 128)]


def _problem(seed, size, d, n_seeds, off, lens=None, grow=None):
    """Inputs of a call; grow(k, v) changes the cached keys and values before they are stored."""
    B, Hq, Hkv, L, Lq = size
    r = _gen(seed)
    t = {"q": r(B, Lq, Hq, d).to(BF16).transpose(1, 2), "k": r(B, Hkv, Lq, d).to(BF16),
         "v": r(B, Lq, Hkv, d).to(BF16).transpose(1, 2), "cache": _empty_cache(B, Hkv, L, d)}
    k, v = (r(B, Hkv, L, d) * torch.exp(0.3 * r(B, Hkv, L, 1)) for _ in range(2))
    if grow:
        grow(t, k, v)
    cover.cover_cache_store(k, v, 0, *t["cache"])
    offs = [off] * B if isinstance(off, int) else off
    t["off"] = off if isinstance(off, int) else torch.tensor(off, device="cuda", dtype=torch.int32)
    t["len"] = None if lens is None else torch.tensor(lens, device="cuda", dtype=torch.int32)
    t["idx"] = t["n"] = None
    if n_seeds:
        g = torch.Generator().manual_seed(seed)
        idx = torch.stack([offs[b] + torch.randperm(Lq, generator=g)[:n_seeds] for b in range(B)])
        t["idx"] = idx.to(device="cuda", dtype=torch.int32)
        t["n"] = torch.tensor([n_seeds - b % 2 * (n_seeds > 1) for b in range(B)], device="cuda", dtype=torch.int32)
    return t


def _places(t):
    """(keys, start, rows, seeds) of each batch row."""
    B, L, Lq = t["q"].shape[0], t["cache"][0].shape[2], t["q"].shape[2]
    for b in range(B):
        n = L if t["len"] is None else min(max(int(t["len"][b]), 0), L)
        o = t["off"] if isinstance(t["off"], int) else min(max(int(t["off"][b]), 0), n)
        rows = max(0, min(Lq, n - o))
        seeds = set() if t["idx"] is None else {j - o for j in t["idx"][b, :max(0, int(t["n"][b]))].tolist()}
        yield n, o, rows, sorted(s for s in seeds if 0 <= s < rows)


def _reference(t):
    """out, lse and their tolerances in 64 bits; NaN where no row exists."""
    q, (B, Hq, Lq, d) = t["q"].double(), t["q"].shape
    Hkv, G = t["k"].shape[1], Hq // t["k"].shape[1]
    out, tol = (torch.full((B, Hq, Lq, d), math.nan, device="cuda", dtype=torch.float64) for _ in range(2))
    lse, ltol = (torch.full((B, Hq, Lq), math.nan, device="cuda", dtype=torch.float64) for _ in range(2))
    for b, (n, o, rows, seeds) in enumerate(_places(t)):
        if rows == 0:
            continue
        seed = torch.zeros(rows, dtype=torch.bool, device="cuda")
        seed[seeds] = True
        j, i = torch.arange(n, device="cuda"), torch.arange(rows, device="cuda")
        block = (j >= o) & (j < o + rows)
        read = ~block
        read[o:o + rows] = seed
        see = torch.cat([read[None] & (j[None] != (o + i)[:, None]), ~seed[None] | (i[None] == i[:, None])], 1)
        for g in range(Hkv):
            kc, vc, ks, vs = (x[b, g, :n].double() for x in t["cache"])
            # (what is not read may hold anything)
            kc, vc = torch.where(read[:, None], kc, 0.0), torch.where(read[:, None], vc, 0.0)
            ks, vs = torch.where(read, ks, 0.0), torch.where(read, vs, 0.0)
            K = torch.cat([kc * ks[:, None], t["k"][b, g, :rows].double()])
            V = torch.cat([vc * vs[:, None], t["v"][b, g, :rows].double()])
            x = q[b, g * G:(g + 1) * G, :rows].reshape(-1, d)
            mask = see.repeat(G, 1)
            s = (x @ K.T.contiguous() * d**-0.5).masked_fill(~mask, -math.inf)
            size = (x.abs() @ K.abs().T.contiguous() * d**-0.5).masked_fill(~mask, 0.0).amax(1)
            err = (d + 8) * 2.0**-24 * size + 2.0**-20
            z = torch.logsumexp(s, 1)
            p = torch.exp(s - z[:, None])
            o_r = p @ V
            floor = 2.0**-28 * p.amax(1)[:, None] * vs.amax().clamp_min(2.0**-30) * (mask[:, :n].double() @ vc.abs())
            e = (2.0**-11 + 2 * err + 2.0**-18)[:, None] * (p @ V.abs()) + floor + 2.0**-8 * o_r.abs()
            h = slice(g * G, (g + 1) * G)
            out[b, h, :rows], tol[b, h, :rows] = o_r.view(G, rows, d), e.view(G, rows, d)
            lse[b, h, :rows], ltol[b, h, :rows] = z.view(G, rows), (err + 2.0**-20 * (1 + z.abs())).view(G, rows)
    return out, lse, tol, ltol


def _check(got, ref, what=""):
    out, lse, tol, ltol = ref
    there = ~torch.isnan(lse)
    _within(got[0][there], out[there], tol[there], f"{what} out")
    _within(got[1][there], lse[there], ltol[there], f"{what} lse")


def _form(size, d, form):
    assert cover.attn_cached_plan(*size, d) == form


@pytest.mark.parametrize("form,size,d", _cases(FORMS, MANY))
@pytest.mark.parametrize("n_seeds", [0, 1, 9])
def test_forms(form, size, d, n_seeds):
    announce(f"attn_cached form {form} {size} d{d} seeds {n_seeds}")
    _form(size, d, form)
    B, Hq, Hkv, L, Lq = size
    t = _problem(L + Lq, size, d, min(n_seeds, Lq), (L - Lq) * 2 // 3)
    got = _call(t)
    torch.cuda.synchronize()
    _check(got, _reference(t))
    again = _call(t, want_lse=False)
    assert _same(again[0], got[0]) and again[1] is None


@pytest.mark.parametrize("form,size,d", _cases(RAGGED, RAGGED_MANY))
def test_ragged_forms(form, size, d):
    """Rows of different lengths down to none, blocks that begin anywhere and end past the row's end; what is not read
    may hold anything, and rows that do not exist are left as they were."""
    announce(f"attn_cached ragged form {form} {size} d{d}")
    _form(size, d, form)
    B, Hq, Hkv, L, Lq = size
    cut = [(L, L - Lq), (L - 1, L - Lq // 2), (L // 2, L // 3), (0, 0), (1, 0), (Lq, 0), (L // 3, L // 3), (L * 3 // 4, 5)]
    cut = cut[:3] if B == 3 else (cut * B)[:B]
    lens, offs = [n for n, _ in cut], [o for _, o in cut]
    t = _problem(L + 7, size, d, min(9, Lq), offs, lens)
    out, lse = torch.full((B, Hq, Lq, d), 7.0, device="cuda", dtype=BF16), torch.full((B, Hq, Lq), 9.0, device="cuda")
    got = _call(t, out=out, lse=lse)
    torch.cuda.synchronize()
    assert got[0] is out and got[1] is lse
    ref = _reference(t)
    _check(got, ref, "ragged")
    gone = torch.isnan(ref[1])
    assert gone.any() and (out[gone] == 7).all() and (lse[gone] == 9).all()
    kc, vc, ks, vs = (x.clone() for x in t["cache"])
    k, v = t["k"].clone(), t["v"].clone()
    for b, (n, o, rows, seeds) in enumerate(_places(t)):
        dead = torch.ones(L, dtype=torch.bool, device="cuda")
        dead[:n] = False
        dead[o:o + rows] = True
        dead[[o + s for s in seeds]] = False
        for c, s in ((kc, ks), (vc, vs)):
            c.view(torch.uint8)[b, :, dead] = 0x7F
            s[b, :, dead] = math.nan
        k[b, :, rows:], v[b, :, rows:] = math.nan, math.inf
    poisoned = _call({**t, "k": k, "v": v, "cache": (kc, vc, ks, vs)})
    assert _same(poisoned[0][~gone], out[~gone]) and _same(poisoned[1][~gone], lse[~gone])


@pytest.mark.parametrize("form,size,d", _cases(FORMS, MANY))
def test_a_seed_that_is_nan(form, size, d):
    """A seed's cached state reaches every row but its own, its live state its own alone."""
    announce(f"attn_cached NaN seed form {form} {size} d{d}")
    _form(size, d, form)
    B, Hq, Hkv, L, Lq = size
    off = (L - Lq) // 2
    t = _problem(5, size, d, 3, off)
    clean = _call(t)
    seed = int(t["idx"][0, 1]) - off
    others = [r for r in range(Lq) if r != seed]
    for which in ((0,), (1,), (0, 1)):
        cache = [x.clone() for x in t["cache"]]
        for i in which:
            cache[i].view(torch.uint8)[0, :, off + seed] = 0x7F
            cache[2 + i][0, :, off + seed] = math.nan
        got = _call({**t, "cache": cache})
        assert _same(got[0][0, :, seed], clean[0][0, :, seed]) and _same(got[0][1:], clean[0][1:]), which
        assert torch.isnan(got[0][0][:, others]).all(), which
    for bad in (math.nan, math.inf, -math.inf):
        k, v = t["k"].clone(), t["v"].clone()
        k[0, :, seed], v[0, :, seed] = bad, bad
        got = _call({**t, "k": k, "v": v})
        assert _same(got[0][0][:, others], clean[0][0][:, others]) and _same(got[1][0][:, others], clean[1][0][:, others])
        assert _same(got[0][1:], clean[0][1:])


@pytest.mark.parametrize("order", ["rising", "falling", "steps"])
@pytest.mark.parametrize("form,size,d", _cases(FORMS, MANY))
def test_maxima_and_value_scales_that_move(form, size, d, order):
    """Scores that rise (fall) by 40 over the keys, so that a row's maximum keeps moving, and values whose scales rise
    by 2^14, so that their unit does; or both in steps, with rows of zeros between."""
    announce(f"attn_cached moving maxima form {form} {size} d{d} {order}")
    _form(size, d, form)
    B, Hq, Hkv, L, Lq = size

    def grow(t, k, v):
        along = torch.linspace(0, 1, L, device="cuda")
        if order == "steps":
            along = (along * 7).floor() / 7
        t["q"][..., 0] = 8.0
        score = 40 * (along if order != "falling" else 1 - along) - 20
        k[..., 0] = score * d**0.5 / 8
        v *= torch.exp2(14 * along - 7)[:, None]
        if order == "steps":
            v[:, :, ::5] = 0.0

    t = _problem(3, size, d, 2, (L - Lq) * 3 // 4, grow=grow)
    got = _call(t)
    torch.cuda.synchronize()
    _check(got, _reference(t), order)


@pytest.mark.parametrize("d", [128, 64])
def test_the_longest_block(d):
    """2048 rows that are the whole sequence, more seeds listed than a workgroup has threads, some twice."""
    announce(f"attn_cached longest block d{d}")
    t = _problem(9, (1, 2, 1, 2100, 2048), d, 1400, 20)
    idx = torch.cat([t["idx"][:, :700], t["idx"][:, :300], t["idx"][:, 700:], t["idx"][:, 1300:]], 1).contiguous()
    t["idx"], t["n"] = idx, torch.tensor([idx.shape[1]], device="cuda", dtype=torch.int32)
    _check(_call(t), _reference(t))


# ---- the weights' bits -----------------------------------------------------------------------
def _error(a, want):
    return ((a.double() - want).norm() / want.norm()).item()


@pytest.mark.parametrize("form,size,d", [*_cases(FORMS, MANY), ((1, 32), (1, 4, 4, 200, 200), 128), ((1, 32), (1, 4, 4, 200, 200), 64)])
def test_the_weights_rounding_stays_below_the_outputs(form, size, d):
    """Over all outputs, the error is that of rounding the exact ones to bf16, and 5 % more: in squares 10 %, where
    fp16 weights add (2^-3)^2 = 1.6 % and weights of bf16 would add 100 % (values of zero mean, so that the weights'
    errors add up as the outputs do).  The last two sizes have only live rows."""
    announce(f"attn_cached weights' bits form {form} {size} d{d}")
    _form(size, d, form)
    B, Hq, Hkv, L, Lq = size
    t = _problem(31, size, d, 0, L - Lq)
    out = _reference(t)[0]
    limit = 1.05 * _error(out.to(BF16), out)
    got = _error(_call(t)[0], out)
    assert got <= limit, (got, limit)
    # the same with weights of bf16, on the CPU: it would be seen
    n = min(L, 3000)
    q, k, v = t["q"][0, 0].cpu().double(), t["cache"][0][0, 0, :n].cpu().double(), t["cache"][1][0, 0, :n].cpu().double()
    k, v = (x * t["cache"][2 + i][0, 0, :n, None].cpu().double() for i, x in enumerate((k, v)))
    w = torch.exp(q @ k.T.contiguous() * d**-0.5)
    want = w @ v / w.sum(1, keepdim=True)
    rounded = (w.to(BF16).double() @ v / w.sum(1, keepdim=True)).to(BF16)
    assert _error(rounded, want) > 1.25 * _error(want.to(BF16), want)


# ---- graphs ----------------------------------------------------------------------------------
def test_key_ranges_in_graphs_that_share_memory():
    """Two captured calls whose workspaces come from one pool, replayed in turn with eager calls between."""
    announce("attn_cached graphs with key ranges")
    size = (1, 4, 2, 4096, 4)
    _form(size, 128, (33, 32))
    ts = [_problem(seed, size, 128, 2, 3000) for seed in (1, 2)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        _call(ts[0])
    s.synchronize()
    pool, graphs, got = torch.cuda.graph_pool_handle(), [], []
    for t in ts:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], pool=pool, stream=s):
            got.append(_call(t))
    for rep in range(4):
        for t in ts:
            t["q"].mul_(1.0 + rep / 4)
        want = [_call(t) for t in ts]
        torch.cuda.synchronize()
        for i in (0, 1):
            graphs[i].replay()
            torch.cuda.synchronize()
            assert _same(got[i][0], want[i][0]) and _same(got[i][1], want[i][1]), (rep, i)
