"""pipeline.ModelCache on the GPU beside its plain use: layers counted from the last,
refused calls, far larger caches than their rows, and other streams."""
from __future__ import annotations

import pytest
import torch

from parity import log

pytestmark = pytest.mark.gpu

DEV = "cuda"


def lib():
    from paper_2508_02751_amd import pipeline as P
    from paper_2508_02751_amd import smallkv as S
    return P, S


def build(layers=2, n_rows=64, batch=2, heads=2, **kw):
    P, S = lib()
    freq, amp = S.rope_freqs(64, 10000.0)
    return P.ModelCache(batch, layers, 2 * heads, heads, 64, n_rows, S.RopeSpec(freq, S.ROPE_HALF, amp),
                        torch.bfloat16, DEV, **kw)


def tokens(g, T, heads=2):
    return [torch.randn(T, h, 64, generator=g).to(DEV, torch.bfloat16) for h in (2 * heads, heads, heads)]


def same(a, b):
    return all(torch.equal(x, y) for x, y in ((a.k, b.k), (a.v, b.v), (a.scores, b.scores)))


def test_layers_from_the_last():
    a, b = build(keep_scores=True), build(keep_scores=True)
    g = torch.Generator().manual_seed(1)
    log("[model cache] negative layers")
    for new in ([30, 12], [1, 1], [0, 20]):
        T = a.begin(new)
        assert b.begin(new) == T
        for layer in (0, 1):
            x = tokens(g, T)
            out, q = a.layer(layer, *x)
            out2, q2 = b.layer(layer - 2, *x)
            assert torch.equal(out, out2) and torch.equal(q, q2)
    torch.cuda.synchronize()
    assert a.rows == b.rows == [31, 33] and same(a, b)


def test_a_refused_call_changes_nothing():
    a, b = build(keep_scores=True), build(keep_scores=True)
    g = torch.Generator().manual_seed(2)
    log("[model cache] refused")
    for new in ([30, 12], [5, 0]):
        T = a.begin(new)
        b.begin(new)
        for layer in (0, 1):
            x = tokens(g, T)
            a.layer(layer, *x)
            before = b.k.clone(), b.v.clone(), b.scores.clone(), list(b.rows), list(b.tokens)
            for bad in ((layer, x[0], x[1], x[2][:-1]), (layer, x[0].float(), x[1], x[2]),
                        (layer, x[0], x[1].cpu(), x[2]), (2, *x), (-3, *x)):
                with pytest.raises((ValueError, IndexError)):
                    b.layer(*bad)
            torch.cuda.synchronize()
            now = b.k, b.v, b.scores
            assert all(torch.equal(p, q) for p, q in zip(before, now)) and before[3:] == (b.rows, b.tokens)
            b.layer(layer, *x)  # the same chunk, as if nothing had been refused
    torch.cuda.synchronize()
    assert a.rows == b.rows and a.tokens == b.tokens and same(a, b)


def test_compression_goes_by_the_rows_in_use():
    """A cache of more rows than an eviction takes, most of them unused."""
    import cache_ref as R
    n = (1 << 20) + 64
    c = build(1, n, 1, 1, keep_scores=True)
    g = torch.Generator().manual_seed(3)
    log("[model cache] a few rows of many")
    c.layer(0, *tokens(g, c.begin([150]), 1))
    small = c.compress([40], [5], 2)
    torch.cuda.synchronize()
    rows = R.kept_rows(c.scores[0, 0].tolist()[:150], 150, 40, 5, 2, 40)
    assert small.row_pos[0, 0, 0].tolist() == rows and small.rows == [40]
    assert torch.equal(small.k[0, 0, 0], c.k[0, 0, 0, rows]) and torch.equal(small.v[0, 0, 0], c.v[0, 0, 0, rows])
    # and with no rows at all
    assert build(1, n, 1, 1, keep_scores=True).compress([7]).rows == [0]


def busy(stream):
    """Work of some tens of milliseconds on the stream."""
    with torch.cuda.stream(stream):
        torch.cuda._sleep(100_000_000)


def ready(stream):
    stream.wait_stream(torch.cuda.current_stream())


@pytest.mark.parametrize("given", [False, True])
def test_memory_of_a_dropped_call_waits_for_its_stream(given):
    """A call prepared on one stream, run on another (given, or made the current one) that is
    still busy, and dropped: its output, lse and workspace are not handed out again before
    that stream has passed it."""
    _, S = lib()
    import cache_ref as R
    c = R.Case([(700, 3), (300, 1)], 8, 2, 128, torch.bfloat16, 16, seed=7)
    chunk, cache, q = c.to(DEV)
    side = torch.cuda.Stream()
    call = S.prepare_chunk_attn(chunk, cache, q, c.scale)
    ready(side)
    busy(side)
    log(f"[streams] dropped call, given={given}")
    if given:
        call.run(side)
    else:
        with torch.cuda.stream(side):
            call.run()
    mine = {t.data_ptr(): t.numel() * t.element_size() for t in (call.out, call.lse, call.ws)}
    del call
    others = [torch.zeros(n, dtype=torch.uint8, device=DEV) for n in mine.values()]
    assert not side.query(), "the stream was done too early to tell"
    assert not any(t.data_ptr() in mine for t in others)
    torch.cuda.synchronize()


def test_a_chunk_on_another_stream():
    """begin() on one stream, layer() on another that is still busy when the next chunk
    begins: the first chunk's lengths and positions are kept until it has read them."""
    a, b = build(1, keep_scores=True), build(1, keep_scores=True)
    g = torch.Generator().manual_seed(5)
    x, y = tokens(g, 42), tokens(g, 2)
    side = torch.cuda.Stream()
    log("[streams] chunk")
    b.begin([30, 12])
    b.layer(0, *x)
    b.begin([1, 1])
    b.layer(0, *y)
    a.begin([30, 12])
    ready(side)
    busy(side)
    ptrs = {t.data_ptr() for t in (a._chunk.start, a._chunk.length, a._positions)}
    with torch.cuda.stream(side):
        a.layer(0, *x)
    a.begin([1, 1])
    more = [torch.zeros(n, dtype=torch.int32, device=DEV) for n in (3, 2, 42)]
    assert not side.query(), "the stream was done too early to tell"
    assert not any(t.data_ptr() in ptrs for t in (a._chunk.start, a._chunk.length, a._positions, *more))
    torch.cuda.current_stream().wait_stream(side)
    a.layer(0, *y)
    torch.cuda.synchronize()
    assert a.rows == b.rows and same(a, b)
