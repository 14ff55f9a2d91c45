"""GPU parity of the cache operators (append, chunk attention, chunk scores,
eviction) against their plain forms in 64 bits, within derived bounds."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import cache_ref as R
from parity import log

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def lib():
    from paper_2508_02751_amd import smallkv as S
    return S


def within(got, want, tol, what):
    got, want = got.detach().cpu().double(), want.double()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    bad = ~(same | ((got - want).abs() <= tol))
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} out of bounds, first at "
                           f"{bad.nonzero()[0].tolist()}: {got[bad][0]} for {want[bad][0]} +- {tol.expand_as(got)[bad][0]}")


# (name, sequences (rows, new), hq, hk, d, dtype, page, rows_first)
CASES = [
    ("one row", [(1, 1)], 4, 2, 64, BF16, 0, False),
    ("one token", [(1000, 1)], 28, 4, 128, BF16, 0, False),
    ("one token f32", [(512, 1)], 28, 4, 128, F32, 0, False),
    ("one token f32 d64", [(131, 1)], 14, 2, 64, F32, 8, False),
    ("single tokens", [(300, 1), (1, 1), (777, 1), (64, 1), (0, 0), (129, 1)], 14, 2, 64, BF16, 16, False),
    ("single tokens, pages of one row", [(37, 1), (130, 1)], 8, 2, 128, BF16, 1, True),
    ("a few rows", [(257, 3), (40, 4), (4, 4)], 14, 2, 128, BF16, 32, False),
    ("a few rows f32", [(257, 2), (40, 1), (2, 2), (16, 2), (70, 0)], 14, 2, 128, F32, 32, False),
    ("a few rows f32 d64", [(500, 8), (23, 8), (5, 7)], 4, 2, 64, F32, 0, False),
    ("some rows f32", [(257, 3), (40, 4)], 14, 2, 64, F32, 16, False),
    ("a whole prompt", [(200, 200)], 8, 2, 64, BF16, 0, False),
    ("a whole prompt f32", [(150, 150)], 8, 4, 128, F32, 64, False),
    ("a whole prompt f32 d64", [(75, 75), (33, 20)], 6, 2, 64, F32, 2, True),
    ("a chunk", [(1300, 139)], 28, 4, 128, BF16, 64, False),
    ("a chunk, no groups", [(500, 77)], 3, 3, 128, BF16, 128, True),
    ("a chunk, one kv head", [(333, 41)], 16, 1, 64, BF16, 4, False),
    ("ragged chunks", [(700, 300), (65, 64), (129, 1), (64, 0), (2000, 33), (1, 1)], 8, 2, 128, BF16, 16, False),
    ("chunks and tokens", [(450, 1), (600, 150), (90, 2), (1025, 1)], 14, 2, 64, BF16, 32, True),
    ("chunks and tokens f32", [(450, 1), (260, 90), (90, 2)], 14, 2, 128, F32, 16, False),
    ("more new tokens than rows", [(5, 9), (30, 30), (0, 3)], 8, 2, 64, BF16, 8, False),
    ("many query heads, one token", [(400, 1), (70, 1)], 64, 1, 128, BF16, 16, False),
    ("long", [(9000, 1), (8191, 40)], 8, 2, 64, BF16, 256, False),
    ("few rows in tiles f32", [(300, 9), (41, 2), (9, 9), (17, 3)], 14, 2, 64, F32, 16, True),
    ("few rows in tiles over spans f32", [(5000, 8), (70, 1), (1100, 5)], 16, 2, 128, F32, 64, False),
    ("one token over many spans", [(20001, 1)], 14, 2, 128, BF16, 0, False),
    ("a hundred query heads", [(300, 5), (70, 1)], 100, 1, 64, BF16, 16, False),
    ("a hundred query heads f32", [(90, 2), (33, 1)], 200, 2, 64, F32, 0, False),
    ("tokens and a chunk over many spans", [(16000, 1), (3, 1), (12000, 37)], 14, 2, 64, BF16, 32, False),
]
IDS = [c[0].replace(" ", "-") for c in CASES]


def make(case, **kw):
    _, lens, hq, hk, d, dtype, page, rows_first = case
    return R.Case(lens, hq, hk, d, dtype, page, rows_first, seed=len(lens) + hq + d, **kw)


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_chunk_attention(case):
    S = lib()
    c = make(case, extra_tokens=3, gap=5)
    chunk, cache, q = c.to(DEV)
    out = torch.full(q.shape, 7.0, dtype=c.dtype, device=DEV)
    lse = torch.full(q.shape[:2], 7.0, device=DEV)
    log(f"[attn] {case[0]}")
    call = S.prepare_chunk_attn(chunk, cache, q, c.scale, out=out, lse=lse)
    call.run()
    torch.cuda.synchronize()
    want, wl, tol, ltol = R.attention(c)
    end = c.starts[-1]
    within(out[:end], want[:end], tol[:end], "out")
    within(lse[:end], wl[:end], ltol[:end], "lse")
    assert bool((out[end:] == 7).all()) and bool((lse[end:] == 7).all()), "tokens of no sequence"
    first = out.clone(), lse.clone()
    call.run()
    torch.cuda.synchronize()
    assert torch.equal(out, first[0]) and torch.equal(lse, first[1]), "the same call, other bits"


@pytest.mark.parametrize("per_kv", [False, True])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_chunk_scores(case, per_kv):
    S = lib()
    c = make(case, gap=5)
    chunk, cache, q = c.to(DEV)
    _, wl, _, _ = R.attention(c)
    lse = wl.float()
    heads = c.hk if per_kv else c.hq
    before = torch.rand(c.B, heads, c.rows + 3, generator=c.gen)
    out = torch.full(before.shape, 7.0, device=DEV)
    log(f"[scores] {case[0]} per_kv={per_kv}")
    S.prepare_chunk_scores(chunk, cache, q, lse.to(DEV), c.scale, out, before=before.to(DEV)).run()
    torch.cuda.synchronize()
    want, tol = R.scores(c, lse, before, per_kv)
    for b, (n, _) in enumerate(c.lens):
        within(out[b, :, :n], want[b, :, :n], tol[b, :, :n], f"sequence {b}")
        assert bool((out[b, :, n:] == 7).all()), "rows past the sequence"
    inplace = before.to(DEV)
    S.prepare_chunk_scores(chunk, cache, q, lse.to(DEV), c.scale, inplace, before=inplace).run()
    zero = torch.full(before.shape, 7.0, device=DEV)
    S.prepare_chunk_scores(chunk, cache, q, lse.to(DEV), c.scale, zero).run()
    torch.cuda.synchronize()
    want0, tol0 = R.scores(c, lse, torch.zeros_like(before), per_kv)
    for b, (n, _) in enumerate(c.lens):
        assert torch.equal(inplace[b, :, :n], out[b, :, :n]), "in place"
        within(zero[b, :, :n], want0[b, :, :n], tol0[b, :, :n], "from zero")


@pytest.mark.parametrize("per_kv", [False, True])
@pytest.mark.parametrize("dtype,d", [(BF16, 64), (F32, 128)])
def test_chunk_scores_with_many_workgroups(dtype, d, per_kv):
    """Enough of them that a workgroup's waves own different keys."""
    S = lib()
    lens = [(n, new) for n, new in ((1100, 60), (700, 700), (33, 7), (1024, 129))] * 8
    c = R.Case(lens, 8, 2, d, dtype, 64, seed=41)
    chunk, cache, q = c.to(DEV)
    _, wl, _, _ = R.attention(c)
    lse = wl.float()
    before = torch.rand(c.B, c.hk if per_kv else c.hq, c.rows, generator=c.gen)
    out = torch.full(before.shape, 7.0, device=DEV)
    log(f"[scores] many {dtype} {per_kv}")
    S.prepare_chunk_scores(chunk, cache, q, lse.to(DEV), c.scale, out, before=before.to(DEV)).run()
    torch.cuda.synchronize()
    want, tol = R.scores(c, lse, before, per_kv)
    for b, (n, _) in enumerate(c.lens):
        within(out[b, :, :n], want[b, :, :n], tol[b, :, :n], f"sequence {b}")
        assert bool((out[b, :, n:] == 7).all())


@pytest.mark.parametrize("new,hq,hk,batch", [(9, 14, 2, 2), (16, 8, 2, 40), (17, 14, 2, 40), (32, 5, 1, 30),
                                             (33, 14, 2, 40), (64, 3, 3, 4), (65, 9, 1, 30), (128, 14, 2, 20)])
@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 128), (F32, 64)])
def test_chunk_scores_of_several_heads_a_workgroup(dtype, d, new, hq, hk, batch):
    """Tokens around the sizes at which heads share a tile; groups that do not fill it;
    many workgroups and few; sequences with fewer tokens, none, and fewer rows than tokens."""
    S = lib()
    some = [(400, new), (new, new), (131, 1), (260, new // 2), (150, 0), (max(new - 3, 0), new)]
    c = R.Case((some * batch)[:batch], hq, hk, d, dtype, 32, seed=67)
    chunk, cache, q = c.to(DEV)
    _, wl, _, _ = R.attention(c)
    lse = wl.float()
    before = torch.rand(c.B, hq, c.rows, generator=c.gen)
    out = before.to(DEV)
    log(f"[scores] heads {dtype} {d} {new} {hq}/{hk} {batch}")
    S.prepare_chunk_scores(chunk, cache, q, lse.to(DEV), c.scale, out, before=out).run()
    torch.cuda.synchronize()
    want, tol = R.scores(c, lse, before, False)
    for b, (n, _) in enumerate(c.lens):
        within(out[b, :, :n], want[b, :, :n], tol[b, :, :n], f"sequence {b}")
        assert torch.equal(out[b, :, n:].cpu(), before[b, :, n:])


def test_scores_add_up_to_the_query_rows():
    """Each query row's weights sum to 1: attention's lse and the scores agree."""
    S = lib()
    c = R.Case([(900, 200), (333, 33)], 14, 2, 64, BF16, 16, seed=3)
    chunk, cache, q = c.to(DEV)
    log("[scores] sums")
    att = S.prepare_chunk_attn(chunk, cache, q, c.scale)
    out = torch.zeros(c.B, c.hq, c.rows, device=DEV)
    sc = S.prepare_chunk_scores(chunk, cache, q, att.lse, c.scale, out)
    att.run()
    sc.run()
    torch.cuda.synchronize()
    for b, (n, new) in enumerate(c.lens):
        # per weight 2^-20 (lse and logits of size 10 in fp32), sums of up to 1e3
        assert torch.allclose(out[b, :, :n].double().sum(1).cpu(), torch.full((c.hq,), float(new)).double(),
                              rtol=2 ** -19, atol=0)


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 128), (F32, 64)])
def test_absent_pages(dtype, d):
    """Page numbers outside the pool: their rows are not attended, get no
    weight, are not written and not copied."""
    S = lib()
    c = R.Case([(200, 40), (90, 1), (48, 20)], 8, 2, d, dtype, 16, seed=11)
    c.table[0, 2] = -1
    c.table[0, 7] = c.k.shape[0]
    c.table[1, 0] = 1 << 30
    c.table[2, :] = -5
    chunk, cache, q = c.to(DEV)
    log(f"[absent] {dtype} {d}")
    call = S.prepare_chunk_attn(chunk, cache, q, c.scale)
    call.run()
    want, wl, tol, ltol = R.attention(c)
    out = torch.zeros(c.B, c.hq, c.rows, device=DEV)
    S.prepare_chunk_scores(chunk, cache, q, wl.float().to(DEV), c.scale, out).run()
    torch.cuda.synchronize()
    within(call.out, want, tol, "out")
    within(call.lse, wl, ltol, "lse")
    assert bool((call.out[61:] == 0).all()) and bool(torch.isneginf(call.lse[61:]).all())
    ws, wt = R.scores(c, wl.float(), torch.zeros(c.B, c.hq, c.rows), False)
    for b, (n, _) in enumerate(c.lens):
        within(out[b, :, :n], ws[b, :, :n], wt[b, :, :n], f"scores {b}")


@pytest.mark.parametrize("lens,hq,hk", [([(300, 100)], 8, 2), ([(70, 4), (66, 3)], 8, 2),
                                        ([(70, 2), (66, 3)], 8, 2), ([(600, 129)], 4, 4)])
@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 128), (F32, 64)])
def test_infinities_reach_only_the_rows_that_see_them(lens, hq, hk, dtype, d):
    """Values and keys of later tokens that are infinite or NaN leave earlier
    tokens' outputs finite and right; rows that see them get them."""
    S = lib()
    c = R.Case(lens, hq, hk, d, dtype, 16, seed=17)
    for b, (n, new) in enumerate(lens):
        for r, x in ((n - 1, math.nan), (n - 2, math.inf), (n - new + 1, -math.inf)):
            p, i = c.slot(b, r)
            c.v[p, :, i, (3 * r) % d] = x
        # (no key: a NaN logit would be its row's whole output)
    chunk, cache, q = c.to(DEV)
    log(f"[inf] {dtype} {d} {lens}")
    call = S.prepare_chunk_attn(chunk, cache, q, c.scale)
    call.run()
    torch.cuda.synchronize()
    want, wl, tol, ltol = R.attention(c)
    within(call.out, want, tol, "out")
    within(call.lse, wl, ltol, "lse")
    if lens[0][1] > 2:  # (of two new tokens the first one's own row is the infinite one)
        assert bool(torch.isfinite(call.out[:1]).all())


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 64)])
def test_nan_keys_of_later_tokens(dtype, d):
    S = lib()
    c = R.Case([(150, 60)], 8, 2, d, dtype, 8, seed=19)
    p, i = c.slot(0, 149)
    c.k[p, :, i] = math.nan
    chunk, cache, q = c.to(DEV)
    log(f"[nan key] {dtype} {d}")
    call = S.prepare_chunk_attn(chunk, cache, q, c.scale)
    call.run()
    torch.cuda.synchronize()
    want, wl, tol, ltol = R.attention(c)
    within(call.out[:59], want[:59], tol[:59], "out")
    within(call.lse[:59], wl[:59], ltol[:59], "lse")
    assert bool(torch.isnan(call.out[59]).all())


@pytest.mark.parametrize("new", [0, 1, 3, 40])
@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 64)])
def test_logits_of_minus_infinity(dtype, d, new):
    """Rows that every query sees with a logit of -inf count as little as absent ones."""
    S = lib()
    c = R.Case([(300, new), (70, min(new, 1))], 8, 2, d, dtype, 8, seed=37)
    c.q = c.q.abs()
    c.k[int(c.table[0, 5]), :, :, 3] = -math.inf
    chunk, cache, q = c.to(DEV)
    c.table = c.table.clone()
    c.table[0, 5] = -1  # for the plain form
    want, wl, tol, ltol = R.attention(c)
    log(f"[-inf] {dtype} {new}")
    if new:
        call = S.prepare_chunk_attn(chunk, cache, q, c.scale)
        call.run()
    lse = wl.float()
    for heads in (c.hq, c.hk):
        before = torch.rand(c.B, heads, c.rows, generator=c.gen)
        out = before.to(DEV)
        S.prepare_chunk_scores(chunk, cache, q, lse.to(DEV), c.scale, out, before=out).run()
        torch.cuda.synchronize()
        ws, wt = R.scores(c, lse, before, heads == c.hk)
        for b, (n, _) in enumerate(c.lens):
            within(out[b, :, :n], ws[b, :, :n], wt[b, :, :n], f"scores {b}")
    if new:
        within(call.out, want, tol, "out")
        within(call.lse, wl, ltol, "lse")


def test_large_logits():
    """Logits of several hundred with a maximum that moves many times."""
    S = lib()
    for dtype in (BF16, F32):
        c = R.Case([(700, 90), (513, 1)], 8, 2, 128, dtype, 32, seed=23)
        for b, (n, _) in enumerate(c.lens):
            for r in range(n):
                p, i = c.slot(b, r)
                c.k[p, :, i] *= 0.02 * r
        chunk, cache, q = c.to(DEV)
        log(f"[large logits] {dtype}")
        call = S.prepare_chunk_attn(chunk, cache, q, c.scale)
        call.run()
        torch.cuda.synchronize()
        want, wl, tol, ltol = R.attention(c)
        within(call.out, want, tol, "out")
        within(call.lse, wl, ltol, "lse")


@pytest.mark.parametrize("batch,longest,new,hk,dtype", [
    (100, 500, 1, 2, BF16), (400, 40, 1, 2, BF16), (130, 300, 2, 1, F32), (90, 90, 30, 2, BF16)])
def test_many_sequences(batch, longest, new, hk, dtype):
    """More sequences than a wave has lanes, with and without spans; some without new
    tokens or rows."""
    S = lib()
    g = torch.Generator().manual_seed(batch)
    lens = []
    for b in range(batch):
        n = int(torch.randint(0, longest + 1, (1,), generator=g))
        lens.append((n, min(n, int(torch.randint(0, new + 1, (1,), generator=g)) if b % 3 else new)))
    c = R.Case(lens, 4 * hk, hk, 64, dtype, 16, seed=batch)
    chunk, cache, q = c.to(DEV)
    log(f"[many] {batch} sequences")
    call = S.prepare_chunk_attn(chunk, cache, q, c.scale)
    call.run()
    want, wl, tol, ltol = R.attention(c)
    out = torch.zeros(c.B, c.hk, c.rows, device=DEV)
    S.prepare_chunk_scores(chunk, cache, q, wl.float().to(DEV), c.scale, out).run()
    torch.cuda.synchronize()
    within(call.out, want, tol, "out")
    within(call.lse, wl, ltol, "lse")
    ws, wt = R.scores(c, wl.float(), torch.zeros(c.B, c.hk, c.rows), True)
    for b, (n, _) in enumerate(lens):
        within(out[b, :, :n], ws[b, :, :n], wt[b, :, :n], f"scores {b}")
    # the same sequences appended
    kv = torch.randn(c.T, 2 * hk, 64, generator=g).to(dtype)
    freq, amp = S.rope_freqs(64, 10000.0)
    S.prepare_append(chunk, cache, S.RopeSpec(freq, S.ROPE_HALF, amp), q, kv.to(DEV)[:, :hk], kv.to(DEV)[:, hk:]).run()
    torch.cuda.synchronize()
    v = cache.v.cpu()
    for b, (n, m) in enumerate(lens):
        for i in range(m):
            p, at = c.slot(b, n - m + i)
            assert torch.equal(v[p, :, at], kv[c.starts[b] + i, hk:])


def test_strided_queries_and_outputs():
    """q inside a fused projection, out in a [heads][tokens] layout; one layer of
    a dense [B][L][Hkv][n_cap][d] cache."""
    S = lib()
    c = R.Case([(130, 40), (77, 9)], 8, 2, 64, BF16, seed=29)
    chunk, cache, q = c.to(DEV)
    big = torch.zeros(c.T, 12, 64, dtype=BF16, device=DEV)
    big[:, 2:10] = q
    layers = torch.full((2, c.B, 3, 2, c.rows, 64), math.nan, dtype=BF16, device=DEV)
    layers[0, :, 1], layers[1, :, 1] = cache.k, cache.v
    out = torch.zeros(8, c.T, 64, dtype=BF16, device=DEV)
    log("[strides]")
    view = S.CacheSpec(layers[0][:, 1], layers[1][:, 1])
    S.prepare_chunk_attn(chunk, view, big[:, 2:10], c.scale, out=out.transpose(0, 1)).run()
    torch.cuda.synchronize()
    want, _, tol, _ = R.attention(c)
    within(out.transpose(0, 1), want, tol, "out")


def test_another_stream_and_a_graph():
    S = lib()
    c = R.Case([(700, 130), (300, 1)], 8, 2, 128, BF16, 16, seed=31)
    chunk, cache, q = c.to(DEV)
    call = S.prepare_chunk_attn(chunk, cache, q, c.scale)
    out = torch.zeros(c.B, c.hq, c.rows, device=DEV)
    sc = S.prepare_chunk_scores(chunk, cache, q, call.lse, c.scale, out)
    want, _, tol, _ = R.attention(c)
    log("[stream]")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call.run(side)
    sc.run(side)
    torch.cuda.synchronize()
    within(call.out, want, tol, "out")
    eager = call.out.clone(), out.clone()
    log("[graph]")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call.run()
        sc.run()
    for scale in (1.0, 0.5, 2.0):
        q.mul_(scale)
        graph.replay()
        torch.cuda.synchronize()
        got = call.out.clone(), out.clone()
        call.run()
        sc.run()
        torch.cuda.synchronize()
        assert torch.equal(got[0], call.out) and torch.equal(got[1], out)
        if scale == 1.0:
            assert torch.equal(got[0], eager[0]) and torch.equal(got[1], eager[1])


@pytest.mark.parametrize("new,dtype", [(1, BF16), (40, BF16), (5, F32)])
def test_lengths_out_of_range_are_clamped(new, dtype):
    """Starts past the tokens, negative lengths and ones past the cache or the hints, more
    new tokens than max_new: as the clamped values, nothing else written."""
    S = lib()
    cap, hq, hk, d = 96, 8, 2, 64
    lens = [(cap, new), (0, new), (80, new), (50, 0)]
    c = R.Case(lens, hq, hk, d, dtype, 16, seed=59, cap=cap, extra_tokens=2)
    chunk, cache, q = c.to(DEV)
    start = torch.tensor([-7, *c.starts[1:3], c.starts[3], c.T + 900], dtype=torch.int32, device=DEV)
    length = torch.tensor([10 ** 9, -10 ** 9, 80, 50], dtype=torch.int32, device=DEV)
    # the last sequence claims two tokens: the clamped one has them
    c.lens[3] = (50, 2 if new > 1 else 1)
    tail = c.T - c.starts[3]
    c.starts[4:] = [c.starts[3] + tail]
    T = c.T
    wild = S.ChunkSpec(start, length, T, max(new, c.lens[3][1]), cap + 1000)
    if new == 1:  # two claimed, one allowed: the second token is in no sequence
        c.starts[4] = c.starts[3] + 1
    log(f"[clamp] {new} {dtype}")
    k0 = cache.k.clone()
    qo = torch.full_like(q, 7.0)
    kv = torch.randn(T, 2 * hk, d, generator=c.gen).to(DEV, dtype)
    freq, amp = S.rope_freqs(d, 10000.0)
    pos = torch.full((c.B, hk, 10), -1, dtype=torch.int32, device=DEV)
    S.prepare_append(wild, cache, S.RopeSpec(freq, S.ROPE_HALF, amp), q, kv[:, :hk], kv[:, hk:], q_out=qo,
                     row_pos=pos).run()
    torch.cuda.synchronize()
    end = c.starts[4]
    assert bool((qo[end:] == 7).all()) and not bool((qo[:end] == 7).all(-1).any())
    bits = torch.int16 if dtype == BF16 else torch.int32
    changed = (cache.k.view(bits) != k0.view(bits)).any(-1).any(1).nonzero().tolist()
    rows = [list(c.slot(b, r)) for b, (n, m) in enumerate(c.lens) for r in range(max(n - m, 0), n)]
    assert sorted(changed) == sorted(rows)
    c.k, c.v, c.q = cache.k.cpu(), cache.v.cpu(), qo.cpu()
    out = torch.full_like(q, 7.0)
    lse = torch.full((T, hq), 7.0, device=DEV)
    S.prepare_chunk_attn(wild, cache, qo, c.scale, out=out, lse=lse).run()
    sc = torch.full((c.B, hk, cap + 1000), 7.0, device=DEV)
    S.prepare_chunk_scores(wild, cache, qo, lse, c.scale, sc).run()
    torch.cuda.synchronize()
    want, wl, tol, ltol = R.attention(c)
    within(out[:end], want[:end], tol[:end], "out")
    within(lse[:end], wl[:end], ltol[:end], "lse")
    assert bool((out[end:] == 7).all()) and bool((lse[end:] == 7).all())
    ws, wt = R.scores(c, lse.cpu(), torch.zeros(c.B, hk, cap), True)
    for b, (n, _) in enumerate(c.lens):
        within(sc[b, :, :n], ws[b, :, :n], wt[b, :, :n], f"scores {b}")
        assert bool((sc[b, :, n:] == 7).all())


@pytest.mark.parametrize("lens", [[(130, 40), (77, 9)], [(700, 1), (64, 1)]])
def test_broadcast_queries_and_keys(lens):
    """One query row for all heads, one layer's rows for all sequences, no lse."""
    S = lib()
    c = R.Case(lens, 8, 2, 64, BF16, seed=53)
    chunk, cache, q = c.to(DEV)
    n = min(n for n, _ in lens)  # rows that sequence 0 and its readers share
    chunk = S.ChunkSpec(chunk.start, torch.full_like(chunk.length, n), c.T, c.max_new, c.rows)
    one, (k, v) = q[:, :1].expand(-1, 8, -1), (x[:1].expand(c.B, -1, -1, -1) for x in (cache.k, cache.v))
    log("[broadcast]")
    call = S.prepare_chunk_attn(chunk, S.CacheSpec(k, v), one, c.scale, lse=False)
    call.run()
    torch.cuda.synchronize()
    assert call.lse is None
    c.lens, c.q = [(n, new) for _, new in lens], one.cpu()
    c.k, c.v = k.cpu(), v.cpu()
    want, _, tol, _ = R.attention(c)
    within(call.out, want, tol, "out")


@pytest.mark.parametrize("page", [0, 16])
def test_offsets_past_32_bits(page):
    """Caches, queries and outputs whose elements lie more than 2^32 bytes apart: every
    operator as over compact tensors."""
    S = lib()
    hq, hk, d, new = 4, 2, 64, 3
    c = R.Case([(150, new), (90, new), (130, new)], hq, hk, d, BF16, page, seed=47)
    chunk, cache, q = c.to(DEV)
    far = (1 << 31) + 5 * 64  # elements between pages, bf16: past 2^32 bytes
    pool = torch.empty(far + (1 << 22), dtype=BF16, device=DEV)
    pool2 = torch.empty_like(pool)
    n_pages = c.k.shape[0]
    if page:  # every other page far away: pages of 4 KB, numbered over the whole pool
        per = page * hk * d
        spread = torch.tensor([i if i % 2 else far // per + i for i in range(n_pages)], dtype=torch.int32)
        shape = (pool.numel() // per, hk, page, d)
        k, v = pool[:shape[0] * per].view(shape), pool2[:shape[0] * per].view(shape)
        k[spread.long().to(DEV)], v[spread.long().to(DEV)] = cache.k, cache.v
        wide = S.CacheSpec(k, v, spread[c.table.long()].to(DEV).contiguous())
    else:
        st = (far // 2, c.rows * d, d, 1)
        k, v = (x.as_strided((3, hk, c.rows, d), st) for x in (pool, pool2))
        k.copy_(cache.k)
        v.copy_(cache.v)
        wide = S.CacheSpec(k, v)
    log(f"[far] page {page}")
    freq, amp = S.rope_freqs(d, 10000.0)
    rope = S.RopeSpec(freq, S.ROPE_HALF, amp)
    kv = torch.randn(c.T, 2 * hk, d, generator=c.gen).to(DEV, BF16)
    big = torch.empty((c.T - 1) * (far // 8) + hq * d, dtype=BF16, device=DEV)
    big2 = torch.empty_like(big)
    fq, fo = (x.as_strided((c.T, hq, d), (far // 8 - far // 8 % 8, d, 1)) for x in (big, big2))
    fq.copy_(q)
    outs = []
    for ca, x, o in ((cache, q.clone(), torch.empty_like(q)), (wide, fq, fo)):
        S.prepare_append(chunk, ca, rope, x, kv[:, :hk], kv[:, hk:], q_out=x).run()
        attn = S.prepare_chunk_attn(chunk, ca, x, c.scale, out=o)
        attn.run()
        sc = torch.zeros(c.B, hk, c.rows, device=DEV)
        S.prepare_chunk_scores(chunk, ca, x, attn.lse, c.scale, sc).run()
        dst = [torch.zeros(c.B, hk, 40, d, dtype=BF16, device=DEV) for _ in range(2)]
        keep = torch.full((c.B,), 40, dtype=torch.int32, device=DEV)
        ev = S.prepare_evict(ca, S.CacheSpec(*dst), chunk.length, keep, sc, sinks=2)
        ev.run()
        torch.cuda.synchronize()
        outs.append([x.clone(), o.clone(), attn.lse, sc, *dst, ev.out_pos, ev.held])
    for x, y in zip(*outs):
        assert torch.equal(x, y)


def test_a_graph_follows_the_lengths():
    """A captured decode step of capacity lengths, replayed as its sequences grow."""
    S = lib()
    cap, hq, hk, d = 700, 8, 2, 64
    c = R.Case([(cap, 1)] * 3, hq, hk, d, BF16, 16, seed=43)
    _, cache, q = c.to(DEV)
    start = torch.arange(4, dtype=torch.int32, device=DEV)
    length = torch.zeros(3, dtype=torch.int32, device=DEV)
    chunk = S.ChunkSpec(start, length, 3, 1, cap)
    kv = torch.randn(3, 2 * hk, d, generator=c.gen).to(DEV, BF16)
    freq, amp = S.rope_freqs(d, 10000.0)
    add = S.prepare_append(chunk, cache, S.RopeSpec(freq, S.ROPE_HALF, amp), q, kv[:, :hk], kv[:, hk:])
    call = S.prepare_chunk_attn(chunk, cache, add.q_out, c.scale)
    sc = torch.zeros(3, hk, cap, device=DEV)
    score = S.prepare_chunk_scores(chunk, cache, add.q_out, call.lse, c.scale, sc, before=sc)
    calls = (add, call, score)

    def state():
        return [t.clone() for t in (cache.k, cache.v, call.out, call.lse, sc)]
    log("[graph] lengths")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for x in calls:
            x.run()
    for lens in ((1, 300, 40), (2, 301, 0), (3, 302, 699), (400, 0, 700), (401, 1, 1)):
        length.copy_(torch.tensor(lens, dtype=torch.int32))
        first = state()
        graph.replay()
        torch.cuda.synchronize()
        got = state()
        for t, x in zip((cache.k, cache.v, call.out, call.lse, sc), first):
            t.copy_(x)
        for x in calls:
            x.run()
        torch.cuda.synchronize()
        for x, y in zip(got, state()):
            bits = torch.int16 if x.dtype == BF16 else torch.int32
            assert torch.equal(x.view(bits), y.view(bits))
        now = R.Case([(n, 1) for n in lens], hq, hk, d, BF16, 16, seed=43, cap=cap)
        now.table, now.q = c.table, add.q_out.cpu()
        now.k, now.v = cache.k.cpu(), cache.v.cpu()
        want, wl, tol, ltol = R.attention(now)
        within(call.out, want, tol, "out")
        within(call.lse, wl, ltol, "lse")


# ------------------------------------------------------------------ append --

ROPES = [("half", 64, 64), ("half", 128, 128), ("half", 128, 32), ("half", 128, 20), ("half", 64, 2),
         ("half", 64, 0), ("interleaved", 128, 128), ("interleaved", 64, 22), ("interleaved", 128, 6)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout,d,rot", ROPES)
@pytest.mark.parametrize("page,rows_first,many", [(0, False, False), (16, True, False), (32, False, True)])
def test_append(dtype, layout, d, rot, page, rows_first, many):
    S = lib()
    lens = [(70, 30), (5, 8), (33, 0), (64, 1)] if not many else [(2100, 1500), (900, 611), (40, 1)]
    c = R.Case(lens, 6, 2, d, dtype, page, rows_first, seed=rot + d, extra_tokens=2, cap=2200 if many else 90)
    chunk, cache, _ = c.to(DEV)
    qkv = torch.randn(c.T, 10, d, generator=c.gen).to(dtype)
    pos = torch.randint(0, 1 << 20, (c.T,), generator=c.gen).int()
    pos[0], pos[1] = (1 << 31) - 1, -12345
    freq, amp = S.rope_freqs(rot, 10000.0, S.ROPE_RAMP, 8.0, orig_len=4096) if rot else \
        (torch.zeros(0, dtype=torch.float64, device=DEV), 1.0)
    x = qkv.to(DEV)
    q_out = torch.full((c.T, 6, d), 7.0, dtype=dtype, device=DEV)
    row_pos = torch.full((c.B, 2, c.rows), -1, dtype=torch.int32, device=DEV)
    k0, v0 = cache.k.clone(), cache.v.clone()
    log(f"[append] {layout} {d} {rot} {dtype} page {page}")
    S.prepare_append(chunk, cache, S.RopeSpec(freq, S.ROPE_HALF if layout == "half" else S.ROPE_INTERLEAVED, amp),
                     x[:, :6], x[:, 6:8], x[:, 8:], positions=pos.to(DEV), q_out=q_out, row_pos=row_pos).run()
    torch.cuda.synchronize()
    angle = pos.double()[:, None] * freq.cpu()
    y, size = R.turned(qkv[:, :8], angle, amp, rot, layout == "interleaved")
    # sines and cosines within 2^-23, two products and a sum, the rounding
    tol = size * 2.0 ** -22 + R.HALF[dtype] * y.abs()
    tol[..., rot:] = 0
    end = c.starts[-1]
    within(q_out[:end], y[:end, :6], tol[:end, :6], "q")
    assert bool((q_out[end:] == 7).all())
    k1, v1, rp = cache.k.cpu(), cache.v.cpu(), row_pos.cpu()
    want_pos = torch.full(rp.shape, -1, dtype=torch.int32)
    for b, (n, new) in enumerate(lens):
        for i in range(new):
            r, t = n - new + i, c.starts[b] + i
            if r < 0:
                continue
            p, at = c.slot(b, r)
            if i % 97 == 0 or new < 50:
                within(k1[p, :, at], y[t, 6:], tol[t, 6:], f"k {b} {i}")
            assert torch.equal(v1[p, :, at], qkv[t, 8:])
            k1[p, :, at], v1[p, :, at] = k0[p, :, at].cpu(), v0[p, :, at].cpu()
            want_pos[b, :, r] = pos[t]
    bits = torch.int16 if dtype == BF16 else torch.int32
    assert torch.equal(k1.contiguous().view(bits), k0.cpu().contiguous().view(bits)), "other rows"
    assert torch.equal(v1.contiguous().view(bits), v0.cpu().contiguous().view(bits)), "other rows"
    assert torch.equal(rp, want_pos)


def test_append_in_place_and_by_row():
    """q turned in place; positions None are the cached rows."""
    S = lib()
    for layout, rot in ((S.ROPE_HALF, 20), (S.ROPE_HALF, 64), (S.ROPE_INTERLEAVED, 64)):
        c = R.Case([(50, 20), (11, 11)], 4, 2, 64, BF16, 8, seed=5)
        chunk, cache, q = c.to(DEV)
        kv = torch.randn(c.T, 4, 64, generator=c.gen).to(BF16).to(DEV)
        freq, amp = S.rope_freqs(rot, 10000.0)
        log(f"[append] in place {layout} {rot}")
        S.prepare_append(chunk, cache, S.RopeSpec(freq, layout, amp), q, kv[:, :2], kv[:, 2:], q_out=q).run()
        torch.cuda.synchronize()
        pos = torch.cat([torch.arange(30, 50), torch.arange(11)]).double()
        y, size = R.turned(c.q, pos[:, None] * freq.cpu(), amp, rot, layout == S.ROPE_INTERLEAVED)
        within(q, y, size * 2.0 ** -22 + R.HALF[BF16] * y.abs(), "q")


def test_append_leaves_absent_pages():
    S = lib()
    c = R.Case([(40, 12)], 4, 2, 64, BF16, 8, seed=7)
    c.table[0, 4] = -1
    chunk, cache, q = c.to(DEV)
    kv = torch.randn(c.T, 4, 64, generator=c.gen).to(BF16).to(DEV)
    k0 = cache.k.clone()
    freq, amp = S.rope_freqs(64, 10000.0)
    log("[append] absent page")
    S.prepare_append(chunk, cache, S.RopeSpec(freq, S.ROPE_HALF, amp), q, kv[:, :2], kv[:, 2:]).run()
    torch.cuda.synchronize()
    changed = (cache.k.view(torch.int16) != k0.view(torch.int16)).any(-1).any(1).nonzero().tolist()
    assert changed == [[int(c.table[0, 3]), i] for i in range(4, 8)]


# ------------------------------------------------------------------- evict --

def evict_case(lens, keep, recent, sinks, group, hk, d, dtype, page, to_page, scores=None, cap=None,
               seed=0, row_pos=True):
    S = lib()
    c = R.Case([(n, 0) for n in lens], hk, hk, d, dtype, page, seed=seed)
    chunk, cache, _ = c.to(DEV)
    c.k, c.v = cache.k.cpu(), cache.v.cpu()
    if scores is None:
        scores = torch.rand(c.B, hk * group, c.rows + 1, generator=c.gen)
    pos = (torch.randint(1, 4, (c.B, hk, c.rows + 2), generator=c.gen).cumsum(2)).int() if row_pos else None
    cap = cap or max(max(keep), 1)
    dst = R.Case([(0, 0)] * c.B, hk, hk, d, dtype, to_page, seed=seed + 1, cap=cap)
    _, to, _ = dst.to(DEV)
    k0, v0 = to.k.clone(), to.v.clone()
    outs = torch.full((c.B, hk * group, cap), 7.0, device=DEV)
    opos = torch.full((c.B, hk, cap), -7, dtype=torch.int32, device=DEV)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device=DEV)
    log(f"[evict] {lens} keep {keep} recent {recent} sinks {sinks} group {group} {dtype}")
    call = S.prepare_evict(cache, to, chunk.length, ints(keep), scores.to(DEV),
                           recent=None if recent is None else ints(recent), sinks=sinks,
                           row_pos=None if pos is None else pos.to(DEV), out_pos=opos, out_scores=outs)
    call.run()
    torch.cuda.synchronize()
    held = call.held.cpu().tolist()
    bits = torch.int16 if dtype == BF16 else torch.int32
    for b, n in enumerate(lens):
        for h in range(hk):
            x = scores[b, h * group: (h + 1) * group, :n]
            f = x[0].clone()
            for i in range(1, group):
                f += x[i]
            rows = R.kept_rows(f.tolist(), n, keep[b], (recent or [0] * c.B)[b], sinks, cap)
            assert held[b] == len(rows)
            m = len(rows)
            want = pos[b, h, rows] if pos is not None else torch.tensor(rows, dtype=torch.int32)
            assert torch.equal(opos[b, h, :m].cpu(), want), f"positions of {b} {h}"
            assert bool((opos[b, h, m:] == -7).all())
            got = outs[b, h * group: (h + 1) * group].cpu()
            assert torch.equal(got[:, :m].view(torch.int32),
                               scores[b, h * group: (h + 1) * group][:, rows].view(torch.int32))
            assert bool((got[:, m:] == 7).all())
            for pool, first, src in ((to.k, k0, c.k), (to.v, v0, c.v)):
                for i, r in enumerate(rows):
                    p, at = dst.slot(b, i)
                    sp, sat = c.slot(b, r)
                    assert torch.equal(pool[p, h, at].cpu().view(bits), src[sp, h, sat].view(bits))
                for i in range(m, cap):
                    p, at = dst.slot(b, i)
                    assert torch.equal(pool[p, h, at].view(bits), first[p, h, at].view(bits))


@pytest.mark.parametrize("lens,keep,recent,sinks,group,hk,d,dtype,page,to_page", [
    ([100], [40], [10], 4, 1, 2, 64, BF16, 0, 0),
    ([1], [1], [0], 0, 1, 1, 128, BF16, 0, 0),
    ([1, 0, 7], [1, 3, 0], None, 2, 2, 2, 64, F32, 8, 0),
    ([300, 77, 1025], [100, 200, 1025], [5, 0, 20], 1, 7, 2, 128, BF16, 16, 32),
    ([65, 64], [64, 64], [64, 70], 4, 3, 4, 64, BF16, 4, 8),
    ([1500], [333], [0], 0, 1, 3, 64, F32, 64, 0),
    ([500], [10], [10], 4, 1, 2, 64, BF16, 0, 16),
    ([500], [10], [4], 9, 1, 2, 64, BF16, 0, 16),
])
def test_evict(lens, keep, recent, sinks, group, hk, d, dtype, page, to_page):
    evict_case(lens, keep, recent, sinks, group, hk, d, dtype, page, to_page)


def test_evict_ties_and_special_scores():
    g = torch.Generator().manual_seed(1)
    n = 700
    x = torch.randint(0, 3, (1, 2, n + 1), generator=g).float()  # ties everywhere
    evict_case([n], [200], [7], 2, 1, 2, 64, BF16, 16, 0, scores=x)
    evict_case([n], [650], [0], 0, 1, 2, 64, BF16, 16, 0, scores=torch.zeros_like(x))
    y = x.clone()
    special = torch.tensor([math.nan, -math.nan, math.inf, -math.inf, -0.0, 0.0, 1e-45, -1e-45, 3e38, -3e38])
    y[0] = special[torch.randint(0, 10, y[0].shape, generator=g)]
    for keep in (5, 100, 400, 640, 699):
        evict_case([n], [keep], [0], 0, 1, 2, 64, BF16, 0, 0, scores=y)
    evict_case([n], [300], [3], 1, 1, 2, 64, BF16, 0, 0, scores=torch.full_like(x, math.nan))


def test_evict_caps_and_rows_as_positions():
    evict_case([900, 50], [600, 50], [10, 3], 4, 1, 2, 64, BF16, 32, 0, cap=77, row_pos=False)


def test_evict_in_a_graph():
    """Captured, replayed with other scores, lengths and budgets, out-of-range ones too."""
    S = lib()
    c = R.Case([(700, 0), (300, 0)], 2, 2, 64, BF16, 32, seed=61)
    chunk, cache, _ = c.to(DEV)
    k, v = (torch.zeros(2, 2, 100, 64, dtype=BF16, device=DEV) for _ in range(2))
    length, keep, recent = (torch.zeros(2, dtype=torch.int32, device=DEV) for _ in range(3))
    scores = torch.zeros(2, 4, 700, device=DEV)
    outs = torch.zeros(2, 4, 100, device=DEV)
    call = S.prepare_evict(cache, S.CacheSpec(k, v), length, keep, scores, recent=recent, sinks=2,
                           out_scores=outs)
    log("[evict] graph")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call.run()
    everything = (k, v, outs, call.out_pos, call.held)
    for lens, kept, rec in (((700, 300), (90, 20), (5, 0)), ((650, 0), (100, 7), (0, 3)),
                            ((10 ** 9, -4), (10 ** 9, 5), (-3, 10 ** 9)), ((1, 300), (50, -9), (9, 9))):
        for t, x in ((length, lens), (keep, kept), (recent, rec)):
            t.copy_(torch.tensor(x, dtype=torch.int32))
        scores.copy_(torch.rand(scores.shape, generator=c.gen))
        for t in everything:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in everything]
        for t in everything:
            t.zero_()
        call.run()
        torch.cuda.synchronize()
        for x, y in zip(got, everything):
            assert torch.equal(x, y)
        for b in range(2):
            n = min(max(lens[b], 0), 700)
            for h in range(2):
                f = scores[b, 2 * h, :n].cpu() + scores[b, 2 * h + 1, :n].cpu()
                rows = R.kept_rows(f.tolist(), n, kept[b], rec[b], 2, 100)
                assert call.held[b] == len(rows)
                assert call.out_pos[b, h, :len(rows)].tolist() == rows


def test_evict_long():
    evict_case([40000, 9000], [300, 100], [20, 1], 4, 2, 1, 64, BF16, 256, 0)


@pytest.mark.parametrize("longest", [512, 513, 2049, 8193, 16385, 32768])
def test_evict_lengths(longest):
    """Lengths around those at which the lanes' share of the keys changes, each batch
    with short sequences beside the longest."""
    evict_case([longest, 37, longest - 1, 1], [250, 30, 511, 1], [16, 2, 0, 1], 4, 1, 1, 64, BF16, 64, 0)


@pytest.mark.parametrize("group", [1, 2])
def test_evict_ranks_in_32_bits(group):
    """Sums that differ only past fp32 are ties."""
    x = torch.zeros(1, group, 65)
    x[0, 0] = 1.0
    if group == 2:
        x[0, 1] = torch.arange(65) * 2.0 ** -30  # lost in the sum
    evict_case([65], [9], [0], 0, group, 1, 64, BF16, 0, 0, scores=x)
