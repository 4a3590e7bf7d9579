"""The operators of a layer that decodes one block against a prefix held in an 8-bit cache, as a
program makes their calls: what is measured, in plain form and through the library.

Five kinds, over the ranges that the library's configurations and tests use:
  norm    the residual's addition and the root-mean-square norm (cover_rms_norm), written in the
          input's type or in e4m3 with a scale per row
  rope    rotary positions of q and k (cover_rope), read out of the fused projection's rows
  store   keys and values quantised into the cache's rows (cover_cache_store)
  load    rows of the cache read back (cover_cache_load)
  attn    the block's attention over the cache and its own live rows (cover_attn_cached)

The e4m3 form of a row x: s = max(max|x| / 448, 2^-126), codes x * (1 / s) rounded to e4m3.
"""
import math

import torch

own = False
cover = None  # the library's binding, imported by the first pass that runs through it

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
E4M3 = torch.float8_e4m3fn
EPS = 1e-6


def _norm(name, R, D, dtype="bf16", residual=True, e4m3=False):
    return {"name": name, "kind": "norm", "R": R, "D": D, "dtype": dtype, "residual": residual, "e4m3": e4m3}


def _rope(name, B, Hq, Hkv, L, d, rot, first, dtype="bf16", interleaved=False, scaling="none"):
    return {"name": name, "kind": "rope", "B": B, "Hq": Hq, "Hkv": Hkv, "L": L, "d": d, "rot": rot, "first": first,
            "dtype": dtype, "interleaved": interleaved, "scaling": scaling}


def _cache(name, kind, B, H, N, L, d, listed_rows, dtype="bf16"):
    return {"name": name, "kind": kind, "B": B, "H": H, "N": N, "L": L, "d": d, "listed_rows": listed_rows,
            "dtype": dtype}


def _attn(name, B, Hq, Hkv, L, Lq, after, seeds, d=128, ragged=False):
    return {"name": name, "kind": "attn", "B": B, "Hq": Hq, "Hkv": Hkv, "L": L, "Lq": Lq, "after": after,
            "seeds": seeds, "d": d, "ragged": ragged}


def listed():
    return [
        # one position of a model of hidden size 4096: the smallest call
        _norm("norm_token", 1, 4096),
        # the generated block of a LLaDA-8B step, normed for an 8-bit product
        _norm("norm_block_e4m3", 256, 4096, e4m3=True),
        # the prompts of a batch: 8 sequences of 2048 positions
        _norm("norm_prompt", 16384, 4096),
        # a 64-position block of LLaDA-8B out of the fused q, k, v projection
        _rope("rope_block", 1, 32, 32, 64, 128, 128, 832),
        # prompts of a grouped-query model (Dream-7B) with frequencies scaled by parts
        _rope("rope_prompt", 4, 28, 4, 2048, 128, 128, 0, scaling="parts"),
        # a finished 64-position block, by its list of positions
        _cache("store_block", "store", 1, 32, 64, 1024, 128, True),
        # the prompts of the serving batch
        _cache("store_prompt", "store", 8, 32, 1536, 2048, 128, False),
        # a prefix read back for a pass over the whole sequence; head size 64, an odd length
        _cache("load_prefix", "load", 4, 16, 1001, 1001, 64, False),
        # a single position behind a long prompt, grouped heads
        _attn("attn_token", 1, 32, 8, 8192, 1, 0, 0),
        # one 64-position block of a LLaDA-8B layer, with seeds
        _attn("attn_block", 1, 32, 32, 1024, 64, 128, 16),
        # a small block behind a very long prompt, Dream-7B heads
        _attn("attn_long", 1, 28, 4, 32768, 32, 0, 8),
        # the serving batch: whole generated blocks, rows of different lengths
        _attn("attn_batched", 8, 32, 32, 2048, 256, 0, 32, ragged=True),
    ]


def _log_int(rng, lo, hi):
    hi = max(lo, hi)
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    heads = [(32, 32), (28, 4), (32, 8), (16, 16), (12, 12), (40, 8)]
    kind = rng.choice(["norm", "norm", "rope", "rope", "store", "load", "attn", "attn", "attn"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    d = rng.choice([128, 128, 64])
    Hq, Hkv = rng.choice(heads)
    B = _log_int(rng, 1, 8)
    if kind == "norm":
        D = _log_int(rng, 60, 9000) if rng.random() < 0.5 else rng.choice([768, 1024, 2048, 3584, 4096, 5120, 8192])
        R = _log_int(rng, 1, min(16384, 16384 * 4096 // (D * (2 if dtype == "f32" else 1))))
        c = _norm("", R, D, dtype, rng.random() < 0.7, rng.random() < 0.4)
    elif kind == "rope":
        L = _log_int(rng, 1, 4 * 2048 // B)
        c = _rope("", B, Hq, Hkv, L, d, rng.choice([d, d, d // 2, 3 * d // 4, 20]), rng.choice([0, 832, 60000]), dtype,
                  rng.random() < 0.4, rng.choice(["none", "linear", "parts"]))
    elif kind in ("store", "load"):
        L = _log_int(rng, 64, min(4096, 8 * 32 * 1536 // (B * Hkv * (2 if dtype == "f32" else 1))))
        N = _log_int(rng, 1, L)
        c = _cache("", kind, B, Hkv, N, L, d, rng.random() < 0.5, dtype)
    else:
        Lq = _log_int(rng, 1, 256)
        most = min(8 * 32 * 256 * 2048 // (B * Hq * Lq), 8 * 32 * 2048 // (B * Hkv))  # no larger than the largest listed
        L = max(_log_int(rng, 40, min(32768, max(64, most))), Lq)
        c = _attn("", B, Hq, Hkv, L, Lq, rng.randint(0, min(L - Lq, 200)), rng.randint(0, min(32, Lq // 2)), d,
                  rng.random() < 0.4)
    del c["name"]
    return c


# ---- inputs ----------------------------------------------------------------------------------
def _rng(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _states(g, B, H, N, d, shift):
    """Keys (shift: with a few channels far from zero, as keys have) or values, rows of unlike size."""
    size = torch.exp(0.3 * _normal(g, B, H, N, 1))
    return _normal(g, B, H, N, d) * size + (3.0 * _normal(g, 1, H, 1, d) * (_normal(g, 1, H, 1, d) > 1.5) if shift else 0.0)


def _codes(x):
    s = (x.abs().amax(-1) / 448.0).clamp_min(2.0**-126)
    return (x * (1.0 / s)[..., None]).to(E4M3), s


def _positions(g, c):
    """N of the L positions of each row, ascending, a few of them padding (-1)."""
    B, N, L = c["B"], c["N"], c["L"]
    rank = torch.rand(B, L, generator=g, device="cuda").argsort(1)[:, :N].sort(1).values
    pos = rank.to(torch.int32)
    pos[:, N - N // 16:] = -1
    return pos.contiguous()


def _lengths(c):
    """Keys of each row: L, or (ragged) from L down to about half of it, by the row."""
    return [c["L"] - (b * (c["L"] // 2) // c["B"] if c["ragged"] else 0) for b in range(c["B"])]


def _offsets(c):
    """Where each row's block starts: `after` positions before the row's end, one of two rows a
    third shorter than the block."""
    short = lambda b: c["Lq"] // 3 if c["ragged"] and b % 2 else 0  # noqa: E731
    return [max(0, n - c["Lq"] - c["after"]) + (short(b) if c["after"] == 0 else 0) for b, n in enumerate(_lengths(c))]


def prepare(case, seed):
    c, g = case, _rng(seed)
    dev = "cuda"
    if c["kind"] == "norm":
        dt = TORCH[c["dtype"]]
        pad = -(-c["D"] * dt.itemsize // 16) * 16 // dt.itemsize  # rows start at 16-byte addresses
        rows = lambda scale: (scale * _normal(g, c["R"], pad)).to(dt)[:, :c["D"]]  # noqa: E731
        return {"c": c, "x": rows(0.5), "w": (1.0 + 0.1 * _normal(g, c["D"])).to(dt),
                "r": rows(2.0) if c["residual"] else None}
    if c["kind"] == "rope":
        B, L, d, dt = c["B"], c["L"], c["d"], TORCH[c["dtype"]]
        Hq, Hkv, rot = c["Hq"], c["Hkv"], c["rot"]
        qkv = _normal(g, B, L, Hq + 2 * Hkv, d).to(dt)  # the projection's rows: q, k, v heads
        q, k = qkv[:, :, :Hq].transpose(1, 2), qkv[:, :, Hq:Hq + Hkv].transpose(1, 2)
        # turns per position; plain, interpolated, or interpolated only where a turn is long
        f = 500000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=dev) / rot) / (2 * math.pi)
        if c["scaling"] == "linear":
            f = f / 4.0
        elif c["scaling"] == "parts":
            keep = ((8192 * f - 1.0) / 31.0).clamp(0, 1)
            f = f * keep + f / 4.0 * (1 - keep)
        pos = c["first"] + torch.arange(L, device=dev, dtype=torch.int32)[None] + 7 * torch.arange(
            B, device=dev, dtype=torch.int32)[:, None]
        return {"c": c, "q": q, "k": k, "pos": pos.contiguous(), "f": f,
                "m": 0.1 * math.log(4.0) + 1.0 if c["scaling"] == "parts" else 1.0}
    if c["kind"] in ("store", "load"):
        B, H, N, L, d, dt = c["B"], c["H"], c["N"], c["L"], c["d"], TORCH[c["dtype"]]
        kc, ks = _codes(_states(g, B, H, L, d, True))
        vc, vs = _codes(_states(g, B, H, L, d, False))
        s = {"c": c, "kc": kc, "vc": vc, "ks": ks, "vs": vs, "first": (L - N) // 2}
        s["pos"] = _positions(g, c) if c["listed_rows"] else None
        if c["kind"] == "store":
            s["k"] = _states(g, B, N, H, d, False).to(dt).transpose(1, 2)  # token-major rows
            s["v"] = _states(g, B, N, H, d, False).to(dt).transpose(1, 2)
        return s
    B, Hq, Hkv, L, Lq, d = (c[n] for n in ("B", "Hq", "Hkv", "L", "Lq", "d"))
    kc, ks = _codes(_states(g, B, Hkv, L, d, True))
    vc, vs = _codes(_states(g, B, Hkv, L, d, False))
    bf = lambda x: x.to(torch.bfloat16)  # noqa: E731
    s = {"c": c, "kc": kc, "vc": vc, "ks": ks, "vs": vs,
         "q": bf(_normal(g, B, Lq, Hq, d)).transpose(1, 2),  # token-major rows
         "k": bf(_states(g, B, Lq, Hkv, d, False)).transpose(1, 2),
         "v": bf(_states(g, B, Lq, Hkv, d, False)).transpose(1, 2)}
    lengths, offsets = _lengths(c), _offsets(c)
    s["len"] = torch.tensor(lengths, device=dev, dtype=torch.int32) if c["ragged"] else None
    s["off"] = torch.tensor(offsets, device=dev, dtype=torch.int32) if c["ragged"] else offsets[0]
    n = min(c["seeds"], Lq // 2)
    s["idx"] = s["n"] = None
    if n:  # seeds among the block's positions, ascending; rows of unlike count
        pick = torch.rand(B, Lq, generator=g, device=dev).argsort(1)[:, :n].sort(1).values
        s["idx"] = (pick + torch.tensor(offsets, device=dev)[:, None]).to(torch.int32).contiguous()
        s["n"] = torch.tensor([max(1, n - b % 3) for b in range(B)], device=dev, dtype=torch.int32)
    # rows past a row's end are left as they were
    s["out"] = torch.zeros(B, Lq, Hq, d, device=dev, dtype=torch.bfloat16).transpose(1, 2)
    s["lse"] = torch.zeros(B, Hq, Lq, device=dev, dtype=torch.float32)
    return s


# ---- one pass --------------------------------------------------------------------------------
def _import():
    global cover
    from paper_2602_06161_amd import cover


def run(state):
    s, c = state, state["c"]
    kind = c["kind"]
    if own:
        if cover is None:
            _import()
        if kind == "norm":
            y, r, scale = cover.cover_rms_norm(s["x"], s["w"], s["r"], EPS, quantize=c["e4m3"])
            return {"y": y, "r": r, "scale": scale}
        if kind == "rope":
            q, k = cover.cover_rope(s["q"], s["k"], s["pos"], s["f"], interleaved=c["interleaved"],
                                    attention_factor=s["m"])
            return {"q": q, "k": k}
        at = s["first"] if kind in ("store", "load") and s["pos"] is None else s.get("pos")
        if kind == "store":
            cover.cover_cache_store(s["k"], s["v"], at, s["kc"], s["vc"], s["ks"], s["vs"])
            return {"kc": s["kc"], "vc": s["vc"], "ks": s["ks"], "vs": s["vs"]}
        if kind == "load":
            k, v = cover.cover_cache_load(s["kc"], s["vc"], s["ks"], s["vs"], at, n=c["N"], dtype=TORCH[c["dtype"]])
            return {"k": k, "v": v}
        out, lse = cover.cover_attn_cached(s["q"], s["k"], s["v"], s["kc"], s["vc"], s["ks"], s["vs"], s["off"],
                                           s["idx"], s["n"], kv_len=s["len"], out=s["out"], lse=s["lse"])
        return {"out": out, "lse": lse}
    if kind == "norm":
        return _plain_norm(s, c)
    if kind == "rope":
        return {"q": _plain_rope(s["q"], s), "k": _plain_rope(s["k"], s)}
    if kind == "store":
        return _plain_store(s, c)
    if kind == "load":
        return {"k": _plain_load(s["kc"], s["ks"], s), "v": _plain_load(s["vc"], s["vs"], s)}
    return _plain_attn(s, c)


def _plain_norm(s, c):
    h = s["x"].float()
    if c["residual"]:
        h = h + s["r"].float()
    y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * s["w"].float()
    out = {"r": h.to(s["x"].dtype) if c["residual"] else None, "scale": None}
    if c["e4m3"]:
        out["y"], out["scale"] = _codes(y)
    else:
        out["y"] = y.to(s["x"].dtype)
    return out


def _plain_rope(x, s):
    c, rot = s["c"], s["c"]["rot"]
    angle = s["pos"].double()[:, None, :, None] * (2 * math.pi * s["f"])  # [B, 1, L, rot / 2]
    cos, sin = (angle.cos() * s["m"]).float(), (angle.sin() * s["m"]).float()
    y = x.float()
    if c["interleaved"]:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, y[..., rot:]), -1).to(x.dtype)


def _rows(s, c):
    """Positions [B, N] of the call's rows, and which of them are in the cache."""
    if s["pos"] is not None:
        pos = s["pos"].long()
    else:
        pos = (s["first"] + torch.arange(c["N"], device="cuda")).expand(c["B"], c["N"])
    return pos, (pos >= 0) & (pos < c["L"])


def _plain_store(s, c):
    pos, there = _rows(s, c)
    b, n = there.nonzero(as_tuple=True)
    p = pos[b, n]
    kq, ksc = _codes(s["k"].float())
    vq, vsc = _codes(s["v"].float())
    out = {x: s[x] for x in ("kc", "vc", "ks", "vs")}  # in place
    out["kc"].view(torch.uint8)[b, :, p] = kq.view(torch.uint8)[b, :, n]
    out["vc"].view(torch.uint8)[b, :, p] = vq.view(torch.uint8)[b, :, n]
    out["ks"][b, :, p] = ksc[b, :, n]
    out["vs"][b, :, p] = vsc[b, :, n]
    return out


def _plain_load(codes, scale, s):
    c = s["c"]
    pos, there = _rows(s, c)
    at = pos.clamp(0, c["L"] - 1)[:, None, :].expand(-1, c["H"], -1)
    x = codes.float() * scale[..., None]
    x = torch.gather(x, 2, at[..., None].expand(-1, -1, -1, c["d"]))
    return (x * there[:, None, :, None]).to(TORCH[c["dtype"]])


def _plain_attn(s, c):
    B, Hq, Hkv, L, Lq, d = (c[n] for n in ("B", "Hq", "Hkv", "L", "Lq", "d"))
    dev = s["q"].device
    length = s["len"].long() if s["len"] is not None else torch.full((B,), L, device=dev)
    off = s["off"].long() if s["len"] is not None else torch.full((B,), s["off"], device=dev)
    r = torch.arange(Lq, device=dev)
    at = off[:, None] + r  # absolute positions of the block's rows
    valid = at < length[:, None]
    seed = torch.zeros(B, L + Lq, device=dev, dtype=torch.bool)
    if s["idx"] is not None:
        used = torch.arange(s["idx"].shape[1], device=dev) < s["n"][:, None]
        seed.scatter_(1, torch.where(used, s["idx"].long(), L + Lq - 1), True)
        seed[:, L:] = False
    row_seed = torch.gather(seed, 1, at)
    # the memory: the cache's rows, with the block's rows that are no seeds in their places
    live = valid & ~row_seed
    b, n = live.nonzero(as_tuple=True)
    K, V = s["kc"].float() * s["ks"][..., None], s["vc"].float() * s["vs"][..., None]
    K[b, :, at[b, n]] = s["k"].float()[b, :, n]
    V[b, :, at[b, n]] = s["v"].float()[b, :, n]
    q = s["q"].float().reshape(B, Hkv, Hq // Hkv * Lq, d)
    S = torch.matmul(q, K.transpose(2, 3).contiguous()).view(B, Hq, Lq, L) * d**-0.5
    # a seed's row sees its own live key and value on its diagonal
    own_k = s["k"].float().repeat_interleave(Hq // Hkv, 1)
    own_v = s["v"].float().repeat_interleave(Hq // Hkv, 1)
    own_s = (s["q"].float() * own_k).sum(-1) * d**-0.5
    diag = (torch.arange(L, device=dev) == at[..., None]) & row_seed[..., None]  # [B, Lq, L]
    S = torch.where(diag[:, None], own_s[..., None], S)
    S.masked_fill_((torch.arange(L, device=dev) >= length[:, None])[:, None, None], -math.inf)
    top = S.amax(-1, keepdim=True)
    P = torch.exp(S - top)
    total = P.sum(-1, keepdim=True)
    P = P / total
    lse = (top + torch.log(total))[..., 0]
    own_p = (P * diag[:, None]).sum(-1, keepdim=True)
    P = P.masked_fill(diag[:, None], 0.0)
    out = torch.matmul(P.reshape(B, Hkv, -1, L), V).reshape(B, Hq, Lq, d) + own_p * own_v
    out = torch.where(valid[:, None, :, None], out, 0.0).to(torch.bfloat16)
    return {"out": out, "lse": torch.where(valid[:, None], lse, 0.0)}


# ---- what a pass cannot do without -----------------------------------------------------------
def work(case):
    c = case
    if c["kind"] == "norm":
        e, n = TORCH[c["dtype"]].itemsize, c["R"] * c["D"]
        moved = n * e * (3 if c["residual"] else 1) + c["D"] * e + (n + 4 * c["R"] if c["e4m3"] else n * e)
        return {"bytes": moved, "flops": 6 * n}
    if c["kind"] == "rope":
        e, n = TORCH[c["dtype"]].itemsize, c["B"] * c["L"] * (c["Hq"] + c["Hkv"])
        return {"bytes": 2 * n * c["d"] * e + 4 * c["B"] * c["L"] + 4 * c["rot"], "flops": 3 * n * c["rot"]}
    if c["kind"] in ("store", "load"):
        n = 2 * c["B"] * c["H"] * c["N"]
        return {"bytes": n * c["d"] * (1 + TORCH[c["dtype"]].itemsize) + 4 * n, "flops": 2 * n * c["d"]}
    d, Lq = c["d"], c["Lq"]
    keys = sum(_lengths(c))
    rows = sum(max(0, min(Lq, n - o)) for n, o in zip(_lengths(c), _offsets(c)))
    pairs = sum(max(0, min(Lq, n - o)) * n for n, o in zip(_lengths(c), _offsets(c)))
    moved = 2 * c["Hkv"] * (keys - rows) * (d + 4) + 2 * c["Hkv"] * rows * d * 2 + c["Hq"] * rows * (4 * d + 4)
    return {"bytes": moved, "flops": 4 * c["Hq"] * pairs * d}


# ---- the definitions in 64 bits --------------------------------------------------------------
def _exact_codes(x):
    scale = torch.maximum(x.abs().max(dim=-1).values / 448.0, torch.tensor(2.0**-126, dtype=torch.float64, device=x.device))
    y = x / scale.unsqueeze(-1)
    # to the nearest of the type's numbers: steps of 2^(e - 3) from 2^e on, of 2^-9 below 2^-6
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0**-6))) - 3)
    return torch.round(y / step) * step, scale


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["kind"] == "norm":
        h = s["x"].double() + (s["r"].double() if c["residual"] else 0.0)
        y = h / torch.sqrt(h.pow(2).sum(dim=1, keepdim=True) / c["D"] + EPS) * s["w"].double()
        codes, scale = _exact_codes(y) if c["e4m3"] else (y, None)
        return {"r": h if c["residual"] else None, "scale": scale, "y": codes}
    if c["kind"] == "rope":
        rot = c["rot"]
        z = torch.exp(2j * math.pi * (s["pos"].double()[..., None] * s["f"])) * s["m"]  # [B, L, rot / 2]

        def turn(x):
            x = x.double()
            part = x[..., :rot]
            pairs = part.unflatten(-1, (rot // 2, 2)) if c["interleaved"] else part.unflatten(-1, (2, rot // 2)).transpose(-1, -2)
            w = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * z[:, None])
            w = w if c["interleaved"] else w.transpose(-1, -2)
            return torch.cat([w.reshape(part.shape), x[..., rot:]], dim=-1)

        return {"q": turn(s["q"]), "k": turn(s["k"])}
    if c["kind"] in ("store", "load"):
        B, N, L, H, d = (c[n] for n in ("B", "N", "L", "H", "d"))
        pos = s["pos"].tolist() if s["pos"] is not None else [list(range(s["first"], s["first"] + N))] * B
        if c["kind"] == "load":
            out = {"k": torch.zeros(B, H, N, d, dtype=torch.float64, device="cuda"),
                   "v": torch.zeros(B, H, N, d, dtype=torch.float64, device="cuda")}
        else:
            out = {"kc": s["kc"].double(), "vc": s["vc"].double(), "ks": s["ks"].double(), "vs": s["vs"].double()}
        for b in range(B):
            ns = [n for n in range(N) if 0 <= pos[b][n] < L]
            ps = [pos[b][n] for n in ns]
            for x in ("k", "v"):
                if c["kind"] == "load":
                    out[x][b][:, ns] = s[x + "c"][b].double()[:, ps] * s[x + "s"][b].double()[:, ps].unsqueeze(-1)
                else:
                    codes, scale = _exact_codes(s[x][b].double()[:, ns])
                    out[x + "c"][b][:, ps] = codes
                    out[x + "s"][b][:, ps] = scale
        return out
    B, Hq, Hkv, L, Lq, d = (c[n] for n in ("B", "Hq", "Hkv", "L", "Lq", "d"))
    out = torch.zeros(B, Hq, Lq, d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(B, Hq, Lq, dtype=torch.float64, device="cuda")
    for b, (n, o) in enumerate(zip(_lengths(c), _offsets(c))):
        rows = max(0, min(Lq, n - o))
        seeds = [] if s["idx"] is None else s["idx"][b, :int(s["n"][b])].tolist()
        is_seed = torch.zeros(L, dtype=torch.bool, device="cuda")
        is_seed[[j for j in seeds if 0 <= j < L]] = True
        # every row over the cache's n keys and the block's own, with what it may see of each
        j, i = torch.arange(n, device="cuda"), torch.arange(rows, device="cuda")
        in_block = (j >= o) & (j < o + rows)
        see_cache = (~in_block | is_seed[:n])[None] & (j[None] != (o + i)[:, None])
        see_live = ~is_seed[o:o + rows][None] | (i[None] == i[:, None])
        see = torch.cat([see_cache, see_live], dim=1)
        for g in range(Hkv):
            heads = slice(g * (Hq // Hkv), (g + 1) * (Hq // Hkv))
            K = torch.cat([s["kc"][b, g, :n].double() * s["ks"][b, g, :n, None].double(), s["k"][b, g, :rows].double()])
            V = torch.cat([s["vc"][b, g, :n].double() * s["vs"][b, g, :n, None].double(), s["v"][b, g, :rows].double()])
            x = s["q"][b, heads, :rows].double().reshape(-1, d) @ K.T.contiguous() / math.sqrt(d)
            x = x.view(-1, rows, n + rows).masked_fill(~see, -math.inf)
            z = torch.logsumexp(x, dim=-1)
            lse[b, heads, :rows] = z
            out[b, heads, :rows] = (torch.exp(x - z.unsqueeze(-1)).view(-1, n + rows) @ V).view(-1, rows, d)
    return {"out": out, "lse": lse}
