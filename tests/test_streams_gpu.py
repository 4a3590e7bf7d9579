"""Calls with `stream` naming a stream that is not the current one: where their results' memory comes from, and that
work which is still pending on the current stream does not touch it."""
import math

import pytest
import torch

from helpers import announce
from paper_2602_06161_amd import cover

pytestmark = pytest.mark.gpu

BF16, I32, U8 = torch.bfloat16, torch.int32, torch.uint8


def _calls():
    """name -> call(**stream) of every entry point that allocates what it returns."""
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    r = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    B, H, L, d, off, Lq = 1, 4, 4096, 128, 3000, 32
    k, v, kc, vc = (r(B, H, L, d).to(BF16) for _ in range(4))
    q, qb = r(B, H, L, d).to(BF16), r(B, H, Lq, d).to(BF16)
    idx, n = torch.tensor([[3001, 3005]], device="cuda", dtype=I32), torch.tensor([2], device="cuda", dtype=I32)
    cache = [torch.empty(B, H, L, d, device="cuda", dtype=torch.float8_e4m3fn) for _ in range(2)] + \
            [torch.empty(B, H, L, device="cuda") for _ in range(2)]
    cover.cover_cache_store(k, v, 0, *cache)
    x, w = r(64, 1000).to(BF16), r(1000).to(BF16)
    pos, freq = torch.arange(L, device="cuda", dtype=I32), cover.rope_freq(d, device="cuda")
    Lr = 256
    logits = r(Lr, 5000).to(BF16)
    tokens = torch.randint(0, 5000, (Lr,), generator=g, device="cuda", dtype=I32)
    masked = (torch.rand(B, Lr, generator=g, device="cuda") < 0.5).to(U8)
    lse = cover.cover_attn_fwd(q, k, v, kc, vc, idx, n)[1]
    logp, d_in, d_out = (torch.rand(B, Lr, generator=g, device="cuda") for _ in range(3))
    top, conf = tokens.view(B, Lr).clone(), torch.rand(B, Lr, generator=g, device="cuda")

    def update(**kw):  # (in place on its first and sixth argument)
        t, m = torch.where(masked > 0, 7, tokens.view(B, Lr)).to(I32), torch.zeros(B, Lr, device="cuda", dtype=I32)
        if kw:
            (kw["stream"] if not isinstance(kw["stream"], int) else torch.cuda.ExternalStream(kw["stream"])).wait_stream(
                torch.cuda.current_stream())
            keep.append((t, m))
        return cover.cover_decode_update(t, top, conf, None, None, m, 7, 0.6, 64, 2, **kw)

    keep = []
    torch.cuda.synchronize()
    block = slice(off, off + Lq)
    return {
        "attn_fwd": lambda **kw: cover.cover_attn_fwd(q, k, v, kc, vc, idx, n, **kw),
        "attn_rect": lambda **kw: cover.cover_attn_rect(qb, k, v, kc, vc, off, idx, n, n_split=4, **kw),
        "attn_stats": lambda **kw: cover.cover_attn_stats(q, k, kc, idx, n, lse, masked, 1 - masked, L - Lr, **kw),
        "attn_cached": lambda **kw: cover.cover_attn_cached(qb, k[:, :, block], v[:, :, block], *cache, off, idx, n, **kw),
        "rms_norm": lambda **kw: cover.cover_rms_norm(x, w, x, quantize=True, **kw),
        "rope": lambda **kw: cover.cover_rope(q, k, pos, freq, **kw),
        "cache_load": lambda **kw: cover.cover_cache_load(*cache, 5, n=100, **kw),
        "token_stats": lambda **kw: cover.cover_token_stats(logits, tokens, **kw),
        "token_sample": lambda **kw: cover.cover_token_sample(logits, 0.7, 3, 4, **kw),
        "select_seeds": lambda **kw: cover.cover_select_seeds(logp, d_in, d_out, masked, 16, **kw),
        "decode_update": update,
    }


NAMES = ("attn_fwd", "attn_rect", "attn_stats", "attn_cached", "rms_norm", "rope", "cache_load", "token_stats",
         "token_sample", "select_seeds", "decode_update")


def _stream_of(t):
    """The stream whose memory holds t."""
    at = t.untyped_storage().data_ptr()
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= at < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("not in the allocator's memory")


def _same(a, b):
    return torch.equal(a.contiguous().view(U8), b.contiguous().view(U8))


def _busy():
    """Some milliseconds of work on the current stream."""
    a = torch.ones(8192, 8192, device="cuda", dtype=BF16)
    for _ in range(8):
        a @ a


@pytest.mark.parametrize("python_form", [False, True])
@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("name", NAMES)
def test_results_come_from_the_stream_that_writes_them(name, handle, python_form):
    announce(f"results of {name} on another stream, handle {handle}, python form {python_form}")
    call = _calls()[name]
    want = call()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    kw = {"stream": s.cuda_stream if handle else s}
    if python_form:
        with torch.device("cuda"):
            got = call(**kw)
    else:
        got = call(**kw)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert (a is None) == (b is None)
        if a is not None:
            assert _same(a, b) and a.stride() == b.stride()
            assert _stream_of(b) == s.cuda_stream != _stream_of(a)
    with torch.cuda.stream(s):  # the current one, by name: as without
        got = call(**kw)
    s.synchronize()
    assert all(_stream_of(t) == s.cuda_stream for t in got if t is not None)


@pytest.mark.parametrize("name", NAMES)
def test_pending_work_does_not_touch_the_results(name):
    """Memory that the current stream has freed with a write to it still pending is not what another stream's call
    writes its results to."""
    announce(f"pending work, {name}")
    call = _calls()[name]
    want = call()
    s = torch.cuda.Stream()
    call(stream=s)
    torch.cuda.synchronize()
    freed = [torch.empty_like(t) for t in want if t is not None for _ in range(4)]
    _busy()
    for t in freed:
        t.view(U8).fill_(0xFF) if t.is_contiguous() else t.zero_()
    del freed, t
    got = call(stream=s)
    s.synchronize()
    torch.cuda.synchronize()
    assert all(_same(a, b) for a, b in zip(want, got) if a is not None)


@pytest.mark.parametrize("name", NAMES)
def test_results_outlive_the_current_streams_use(name):
    """Results dropped while the current stream has yet to read them are not given to the other stream's next call."""
    announce(f"results in use, {name}")
    call = _calls()[name]
    want = call()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = call(stream=s)
    torch.cuda.current_stream().wait_stream(s)
    _busy()
    copies = [None if t is None else t.clone() for t in got]
    del got
    with torch.cuda.stream(s):
        junk = [torch.full_like(t.view(U8) if t.is_contiguous() else t, 1) for t in want if t is not None for _ in range(8)]
    torch.cuda.synchronize()
    del junk
    assert all(_same(a, b) for a, b in zip(want, copies) if a is not None)


def test_prepared_calls():
    announce("prepared calls on another stream")
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    k, v, kc, vc = (torch.randn(1, 4, 4096, 128, generator=g, device="cuda").to(BF16) for _ in range(4))
    q = torch.randn(1, 4, 32, 128, generator=g, device="cuda").to(BF16)
    want = cover.cover_attn_rect(q, k, v, kc, vc, 100, n_split=4)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    call = cover.PreparedRect(q, k, v, kc, vc, 100, n_split=4, stream=s)
    assert all(_stream_of(t) == s.cuda_stream for t in (call.out, call.lse, call._keep[-1]))
    s.synchronize()
    call.out.fill_(math.nan)
    torch.cuda.synchronize()
    call()
    torch.cuda.synchronize()
    assert _same(call.out, want[0]) and _same(call.lse, want[1])


def test_the_default_stream_by_its_handle():
    announce("the default stream by its handle")
    call = _calls()["rms_norm"]
    want = call()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = call(stream=0)
        assert torch.cuda.current_stream() == s
    torch.cuda.synchronize()
    assert all(_same(a, b) and _stream_of(b) == 0 for a, b in zip(want, got) if a is not None)


@pytest.mark.parametrize("name", ["attn_cached", "rms_norm", "cache_load", "attn_rect", "token_stats"])
def test_another_stream_within_a_capture(name):
    """A capture that forks to the stream named in the call and joins it: the graph's memory holds the results, and
    replays with eager calls between repeat them."""
    announce(f"capture with a fork, {name}")
    call = _calls()[name]
    want = [None if t is None else t.clone() for t in call()]
    s, other = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        call()
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        other.wait_stream(s)
        first = call(stream=other)
        second = call(stream=other)
        del first
        third = call(stream=other)
        s.wait_stream(other)
        copies = [None if t is None else t.clone() for t in third]
    for rep in range(4):
        for t in (*second, *third, *copies):
            if t is not None:
                t.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for got in (second, third, copies):
            assert all(_same(a, b) for a, b in zip(want, got) if a is not None), rep
        call()
        call(stream=other)
        torch.cuda.synchronize()
