"""GPU parity of the packed cache's operators (append, read, attention, scores, eviction)
with their plain forms in 64 bits: codes and scales bit by bit, the rest within the bounds
of the plain cache's operators."""
from __future__ import annotations

import math

import pytest
import torch

import cache_ref as R
import packed_ref as P
from parity import log

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
FORMATS = [P.MXFP8, P.MXFP4]
NAMES = {P.MXFP8: "mxfp8", P.MXFP4: "mxfp4"}


def lib():
    from paper_2508_02751_amd import smallkv as S
    return S


def within(got, want, tol, what):
    got, want = got.detach().cpu().double(), want.double()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    bad = ~(same | ((got - want).abs() <= tol))
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} out of bounds, first at "
                           f"{bad.nonzero()[0].tolist()}: {got[bad][0]} for {want[bad][0]} +- {tol.expand_as(got)[bad][0]}")


def same(got, want, what):
    got, want = got.detach().cpu(), want.cpu()
    bad = ~((got == want) | (torch.isnan(got) & torch.isnan(want)) if got.is_floating_point() else got == want)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} differ, first at "
                           f"{bad.nonzero()[0].tolist()}: {got[bad][0]} for {want[bad][0]}")


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
    ("one token over many spans", [(20001, 1)], 14, 2, 128, BF16, 0, False),
    ("one token over many spans f32", [(9001, 1)], 14, 2, 128, F32, 64, True),
    ("a hundred query heads", [(300, 5), (70, 1)], 100, 1, 64, BF16, 16, False),
]
IDS = [c[0] for c in CASES]


def make(case, fmt, seed=0, **kw):
    name, lens, hq, hk, d, dtype, page, rows_first = case
    log(f"[packed] {name} {NAMES[fmt]}")
    return P.Case(lens, hq, hk, d, dtype, fmt, page, rows_first, seed=seed, **kw)


def check_attn(c, out=None, lse=None, **kw):
    S = lib()
    chunk, cache, q = c.to(DEV)
    call = S.prepare_chunk_attn(chunk, cache, q, c.scale, **kw)
    call.run()
    torch.cuda.synchronize()
    want, want_lse, tol, ltol = R.attention(c)
    rows = slice(0, c.starts[-1])
    within(call.lse[rows], want_lse[rows], ltol[rows], "lse")
    within(call.out[rows], want[rows], tol[rows], "out")
    return call


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_attention(case, fmt):
    check_attn(make(case, fmt, outliers=True))


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_scores(case, fmt):
    S = lib()
    c = make(case, fmt, seed=5)
    chunk, cache, q = c.to(DEV)
    _, lse, _, _ = R.attention(c)
    lse = lse.float()
    for heads in {c.hq, c.hk}:
        before = torch.rand(c.B, heads, c.rows, generator=c.gen)
        out = torch.full_like(before, -7.0).to(DEV)
        S.prepare_chunk_scores(chunk, cache, q, lse.to(DEV), c.scale, out, before=before.to(DEV)).run()
        torch.cuda.synchronize()
        want, tol = R.scores(c, lse, before, per_kv=heads != c.hq)
        for b, (n, _) in enumerate(c.lens):
            n = max(n, 0)
            within(out[b, :, :n], want[b, :, :n], tol[b, :, :n], f"scores of {b}")
            assert (out[b, :, n:] == -7.0).all()


# ----------------------------------------------------------------- append --

def run_append(c, rot, layout, far=0, amp=1.0, new_k=None, new_v=None, in_place=False):
    """The append of random (or given) rows: all four pools and q_out against the plain form."""
    S = lib()
    T = c.T
    hk, d = c.hk, c.d
    k = torch.randn(T, hk, d, generator=c.gen).to(c.dtype) if new_k is None else new_k
    v = torch.randn(T, hk, d, generator=c.gen).to(c.dtype) if new_v is None else new_v
    pos = torch.zeros(T, dtype=torch.int32)
    rows, seqs = torch.full((T,), -1), torch.full((T,), -1)
    for b, (n, new) in enumerate(c.lens):
        i = slice(c.starts[b], c.starts[b] + new)
        rows[i] = n - new + torch.arange(new)
        seqs[i] = b
    pos = (rows.clamp_min(0) + far).int()
    freq = 10000.0 ** (-torch.arange(0, max(rot, 2), 2, dtype=torch.float64) / max(rot, 2))[: rot // 2]
    chunk, cache, q = c.to(DEV)
    before = [t.clone() for t in cache.tensors[:4]]
    rope = S.RopeSpec(freq.to(DEV), layout, amp)
    call = S.prepare_append(chunk, cache, rope, q, k.to(DEV), v.to(DEV), positions=pos.to(DEV),
                            q_out=q if in_place else None)
    call.run()
    torch.cuda.synchronize()
    angle = pos.double()[:, None] * freq
    amp = float(torch.tensor(amp))
    turned, size = R.turned(c.q, angle, amp, rot, layout == S.ROPE_INTERLEAVED)
    live = seqs >= 0
    h = R.HALF[c.dtype]
    within(call.q_out[live], turned[live], (h * turned.abs() + 16 * R.U * size)[live], "q_out")
    tk, _ = R.turned(k, angle, amp, rot, layout == S.ROPE_INTERLEAVED)
    want = [t.cpu().clone() for t in before]
    for x, codes, scales in ((tk, 0, 2), (v, 1, 3)):
        pc, ps = P.pack(x, c.fmt)
        for t in range(T):
            if rows[t] < 0:
                continue
            p, i = c.slot(int(seqs[t]), int(rows[t]))
            if 0 <= p < c.k.shape[0]:
                want[codes][p, :, i], want[scales][p, :, i] = pc[t], ps[t]
    for t, w, what in zip(cache.tensors, want, ("k", "v", "k_scale", "v_scale")):
        same(t, w, what)
    return call


APPENDS = [
    # sequences, hq, hk, d, dtype, page, rows_first, rot, layout, far
    ([(1, 1)], 4, 2, 64, BF16, 0, False, 64, 0, 0),
    ([(300, 1), (1, 1), (777, 1)], 28, 4, 128, BF16, 16, False, 128, 0, 1000003),
    ([(70, 70), (40, 3), (9, 0)], 14, 2, 64, F32, 8, True, 64, 0, 0),
    ([(70, 70), (40, 3)], 6, 3, 128, BF16, 32, False, 128, 1, 131072),
    ([(33, 33)], 4, 2, 128, BF16, 0, False, 96, 0, 0),
    ([(33, 33)], 4, 2, 128, F32, 4, False, 50, 0, 17),
    ([(33, 20)], 4, 2, 64, BF16, 4, False, 6, 1, 17),
    ([(33, 20)], 4, 2, 64, BF16, 4, True, 22, 0, 0),
    ([(33, 20)], 4, 2, 64, F32, 4, False, 0, 0, 0),
    ([(2500, 2500), (3, 3)], 4, 2, 64, BF16, 64, False, 64, 0, 0),
    ([(2100, 2100)], 2, 1, 128, F32, 0, False, 128, 1, 0),
    ([(5, 9), (0, 3)], 4, 2, 64, BF16, 8, False, 64, 0, 0),
]


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("case", APPENDS, ids=[f"{i}" for i in range(len(APPENDS))])
def test_append(case, fmt):
    lens, hq, hk, d, dtype, page, rows_first, rot, layout, far = case
    log(f"[packed append] {case} {NAMES[fmt]}")
    run_append(P.Case(lens, hq, hk, d, dtype, fmt, page, rows_first, seed=3), rot, layout, far,
               amp=1.0 if far == 0 else 1.138)


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("layout", [0, 1])
def test_append_turns_queries_in_place(fmt, layout):
    log(f"[packed append] in place {NAMES[fmt]}")
    run_append(P.Case([(90, 90), (200, 1)], 14, 2, 64, BF16, fmt, 16, seed=4), 64, layout, in_place=True)


def hard_rows(fmt, dtype):
    """Blocks at the borders of the format, [T][1][64]: a block each, beside a usual one."""
    top = 464.0 if fmt == P.MXFP8 else 7.0
    vals = P.code_values(fmt)[: 127 if fmt == P.MXFP8 else 8]
    ties = ((vals[1:] + vals[:-1]) / 2).tolist()
    most = float(vals[-1])
    blocks = [[0.0] * 32, [-0.0] * 32, [1e-38] * 32, [-1e-30] + [0.0] * 31, [3e38] + [1e30] * 31,
              [2.0 ** -100] * 32, [2.0 ** -109] * 32, [top * 2.0 ** -100] + [2.0 ** -101] * 31,
              [math.inf] + [1.0] * 31, [1.0] * 31 + [-math.inf], [math.nan] * 32, [1.0] * 16 + [math.nan] * 16,
              [top] + [1.0] * 31, [-top] + [1.0] * 31, [top * (1 + 2.0 ** -7)] + [1.0] * 31,
              [top * (1 + 2.0 ** -23)] + [1.0] * 31, [most] + [0.4] * 31, [3.3895e38] * 32]
    for i in range(0, len(ties), 31):
        blocks.append(([most] + ties[i: i + 31] + [0.0] * 31)[:32])
        blocks.append(([-most] + [-x * (1 + 2.0 ** -23) for x in ties[i: i + 31]] + [0.0] * 31)[:32])
        blocks.append(([most] + [x * (1 - 2.0 ** -8) for x in ties[i: i + 31]] + [0.0] * 31)[:32])
    g = torch.Generator().manual_seed(1)
    x = torch.randn(len(blocks), 1, 64, generator=g)
    x[:, 0, 32:] = torch.tensor(blocks, dtype=torch.float64).float()
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
def test_append_blocks_at_the_borders(fmt, dtype):
    x = hard_rows(fmt, dtype)
    T = x.shape[0]
    log(f"[packed append] borders {NAMES[fmt]} {dtype}")
    # rot 0 and 32: the block in question is copied, or in the part that does not turn
    for rot in (0, 32):
        c = P.Case([(T, T)], 1, 1, 64, dtype, fmt, 0, seed=2)
        run_append(c, rot, 0, new_k=x, new_v=x.flip(0))


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
def test_append_writes_positions_and_leaves_the_rest(fmt):
    """Bad pages, tokens of no sequence, rows past max_new: nothing of theirs is written."""
    S = lib()
    log(f"[packed append] bad pages {NAMES[fmt]}")
    c = P.Case([(40, 20), (30, 2)], 4, 2, 64, BF16, fmt, 8, seed=9, extra_tokens=5)
    c.table[0, 3], c.table[1, 3] = -1, 1000
    run_append(c, 64, 0)
    chunk, cache, q = c.to(DEV)
    pos = torch.full((2, 2, 33), -5, dtype=torch.int32, device=DEV)
    k = torch.randn(c.T, 2, 64).to(DEV, BF16)
    freq, _ = S.rope_freqs(64, 10000.0)
    S.prepare_append(chunk, cache, S.RopeSpec(freq), q, k, k, row_pos=pos).run()
    torch.cuda.synchronize()
    want = torch.full((2, 2, 33), -5, dtype=torch.int32)
    want[0, :, 20:33] = torch.arange(20, 33, dtype=torch.int32)
    want[1, :, 28:30] = torch.arange(28, 30, dtype=torch.int32)
    same(pos, want, "row_pos")


# ------------------------------------------------------------------- read --

READS = [
    ([(1, 1)], 2, 64, 0, False, 0), ([(300, 0), (17, 0), (0, 0)], 4, 128, 16, False, 8),
    ([(300, 0), (129, 0)], 2, 64, 64, True, 0), ([(5000, 0), (4097, 0)], 3, 128, 0, False, 32),
]


@pytest.mark.parametrize("out", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("case", READS, ids=[f"{i}" for i in range(len(READS))])
def test_read(case, fmt, out):
    S = lib()
    lens, hk, d, page, rows_first, to_page = case
    log(f"[packed read] {case} {NAMES[fmt]} {out}")
    c = P.Case([(n, 0) for n, _ in lens], hk, hk, d, F32, fmt, page, rows_first, seed=7, outliers=True)
    if c.table is not None:
        c.table[0, 1] = 4097  # an absent page
    c.codes[1][0, 0, 0, :] = 255  # a row of NaN
    c.codes[2][0, :, 0, 5] = 0x83  # and a code of each
    c.refresh()
    _, cache, _ = c.to(DEV)
    B = len(lens)
    length = torch.tensor([n for n, _ in lens], dtype=torch.int32, device=DEV)
    for begin in (None, [max(0, n - 7) for n, _ in lens], [-3] + [100000] * (B - 1)):
        plain = R.Case([(n, 0) for n, _ in lens], hk, hk, d, out, to_page, False, seed=8)
        _, to, _ = plain.to(DEV)
        at = None if begin is None else torch.tensor(begin, dtype=torch.int32, device=DEV)
        S.prepare_read(cache, to, length, begin=at).run()
        torch.cuda.synchronize()
        for pool, src, dst in ((to.k, c.k, plain.k), (to.v, c.v, plain.v)):
            want = dst.clone()
            for b, (n, _) in enumerate(lens):
                first = 0 if begin is None else min(max(begin[b], 0), n)
                for r in range(first, n):
                    p, i = c.slot(b, r)
                    if 0 <= p < src.shape[0]:
                        p2, i2 = plain.slot(b, r)
                        want[p2, :, i2] = src[p, :, i].to(out)
            same(pool, want, "rows")


# ------------------------------------------------------------------ evict --

@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("d,page,to_page", [(64, 16, 0), (128, 0, 32)])
def test_evict(fmt, d, page, to_page):
    S = lib()
    lens = [(700, 0), (33, 0), (1, 0), (0, 0), (1300, 0)]
    log(f"[packed evict] {NAMES[fmt]} {d} {page} {to_page}")
    H, gs, sinks = 3, 2, 4
    c = P.Case(lens, H, H, d, BF16, fmt, page, page > 0, seed=11)
    scores = torch.rand(5, H * gs, c.rows, generator=c.gen)
    scores[:, :, ::7] = 0.25
    keep, recent = [100, 40, 1, 5, 1299], [10, 3, 0, 0, 700]
    _, cache, _ = c.to(DEV)
    dst = P.Case([(max(1, k), 0) for k in keep], H, H, d, BF16, fmt, to_page, False, seed=12)
    _, to, _ = dst.to(DEV)
    before = [t.cpu().clone() for t in to.tensors[:4]]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    out_scores = torch.zeros(5, H * gs, to.capacity, device=DEV)
    call = S.prepare_evict(cache, to, ints([n for n, _ in lens]), ints(keep), scores.to(DEV), recent=ints(recent),
                           sinks=sinks, out_scores=out_scores)
    call.run()
    torch.cuda.synchronize()
    for b, (n, _) in enumerate(lens):
        kept = min(keep[b], n)
        assert int(call.held[b]) == kept
        for h in range(H):
            f = (scores[b, h * gs] + scores[b, h * gs + 1]).tolist()
            rows = R.kept_rows(f, n, keep[b], recent[b], sinks, to.capacity)
            assert call.out_pos[b, h, :kept].tolist() == rows
            for i, r in enumerate(rows):
                p, at = c.slot(b, r)
                p2, at2 = dst.slot(b, i)
                for w, src in zip((0, 2, 1, 3), c.codes):  # k, v, k_scale, v_scale of tensors
                    before[w][p2, h, at2] = src[p, h, at]
            same(out_scores[b, h * gs: h * gs + gs, :kept], scores[b, h * gs: h * gs + gs][:, rows], "scores")
    for t, w in zip(to.tensors, before):
        same(t, w, "rows")


# ----------------------------------------------------- masked, absent, NaN --

def nan_block(c, which, b, r, head, block):
    """Makes a block of a row NaN: of keys (0) or values (1)."""
    p, i = c.slot(b, r)
    c.codes[2 * which + 1][p, head, i, block] = 255
    c.refresh()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("lens", [[(70, 5)], [(200, 100)], [(9000, 40), (33, 33)]], ids=["few", "chunk", "spans"])
def test_nan_values_reach_only_the_tokens_that_see_them(lens, fmt, dtype):
    log(f"[packed] NaN values {lens} {NAMES[fmt]} {dtype}")
    c = P.Case(lens, 4, 2, 64, dtype, fmt, 16, seed=21)
    n, new = lens[0]
    seen = n - new + 2  # the third token's own row
    clean = R.attention(c)
    nan_block(c, 1, 0, seen, 1, 1)
    S = lib()
    chunk, cache, q = c.to(DEV)
    call = S.prepare_chunk_attn(chunk, cache, q, c.scale)
    call.run()
    torch.cuda.synchronize()
    out = call.out.cpu()
    hit = torch.zeros_like(out, dtype=torch.bool)
    hit[2: new, 2:, 32:] = True  # from that token on, the second kv head's queries, the second block
    assert torch.isnan(out[hit]).all()
    within(out[~hit], clean[0][~hit], clean[2][~hit], "out")
    within(call.lse, clean[1], clean[3], "lse")


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_nan_keys_reach_only_the_tokens_that_see_them(fmt, dtype):
    S = lib()
    log(f"[packed] NaN keys {NAMES[fmt]} {dtype}")
    for lens in ([(70, 5)], [(200, 100)]):
        c = P.Case(lens, 4, 2, 64, dtype, fmt, 16, seed=22)
        n, new = lens[0]
        clean = R.attention(c)
        nan_block(c, 0, 0, n - 2, 0, 1)  # the last but one token's row
        chunk, cache, q = c.to(DEV)
        call = S.prepare_chunk_attn(chunk, cache, q, c.scale)
        call.run()
        torch.cuda.synchronize()
        hit = torch.zeros(new, 4, dtype=torch.bool)
        hit[new - 2:, :2] = True
        out, lse = call.out.cpu(), call.lse.cpu()
        assert torch.isnan(out[hit]).all() and torch.isnan(lse[hit]).all()
        within(out[~hit], clean[0][~hit], clean[2][~hit], "out")
        within(lse[~hit], clean[1][~hit], clean[3][~hit], "lse")


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_absent_pages(fmt, dtype):
    log(f"[packed] absent pages {NAMES[fmt]} {dtype}")
    for lens in ([(100, 1), (50, 1), (20, 1)], [(300, 70), (50, 9), (20, 20)]):
        c = P.Case(lens, 14, 2, 64, dtype, fmt, 16, seed=23)
        c.table[0, 2], c.table[0, 6] = -1, 5000
        c.table[2, :] = -7  # a sequence without any
        c.table[1, 0] = c.table[1, 1]  # the same page twice
        call = check_attn(c)
        i = slice(c.starts[2], c.starts[3])
        assert (call.out[i] == 0).all() and torch.isinf(call.lse[i]).all()


def test_calls_of_two_streams_and_captured_ones():
    """A decode step captured into a graph, replayed while its lengths grow, beside eager calls
    on another stream with workspaces of their own."""
    S = lib()
    log("[packed] graph")
    freq, _ = S.rope_freqs(64, 10000.0)
    c = P.Case([(500, 1), (300, 1)], 14, 2, 64, BF16, P.MXFP8, 16, seed=31, cap=640)
    chunk, cache, q = c.to(DEV)
    twin = S.PackedSpec(*(t.clone() for t in cache.tensors[:2]), *(t.clone() for t in cache.tensors[2:4]),
                        P.MXFP8, cache.page_table)
    chunk2 = S.ChunkSpec(chunk.start, chunk.length.clone(), chunk.n_tokens, 1, c.rows)
    scores = torch.zeros(2, 2, c.rows, device=DEV)
    scores2 = torch.zeros_like(scores)
    kv = torch.randn(2, 2, 64).to(DEV, BF16)

    def step(chunk, cache, scores):
        add = S.prepare_append(chunk, cache, S.RopeSpec(freq), q, kv, kv)
        attn = S.prepare_chunk_attn(chunk, cache, add.q_out, c.scale)
        score = S.prepare_chunk_scores(chunk, cache, add.q_out, attn.lse, c.scale, scores, before=scores)
        return [add, attn, score]
    calls, calls2 = step(chunk, cache, scores), step(chunk2, twin, scores2)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for x in calls:
            x.run()
    for i in range(4):
        g.replay()
        with torch.cuda.stream(side):
            for x in calls2:
                x.run()
        torch.cuda.synchronize()
        assert torch.equal(calls[1].out, calls2[1].out) and torch.equal(calls[1].lse, calls2[1].lse)
        assert torch.equal(scores, scores2)
        for a, b in zip(cache.tensors[:4], twin.tensors[:4]):
            assert torch.equal(a, b)
        chunk.length += 1
        chunk2.length += 1
        torch.cuda.synchronize()


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
def test_model_cache(fmt):
    """Prompts and tokens through a packed ModelCache, compressed, grown again and read back:
    what the same steps give on plain caches that hold what its rows stand for."""
    from paper_2508_02751_amd import pipeline as L
    S = lib()
    log(f"[packed] model cache {NAMES[fmt]}")
    freq, amp = S.rope_freqs(64, 10000.0)
    rope = S.RopeSpec(freq, S.ROPE_HALF, amp)
    c = L.ModelCache(2, 2, 4, 2, 64, 96, rope, keep_scores=True, packed=fmt)
    g = torch.Generator().manual_seed(5)

    def fill(c, new):
        T = c.begin(new)
        for layer in range(2):
            q, k, v = (torch.randn(T, h, 64, generator=g).to(DEV, BF16) for h in (4, 2, 2))
            out, tq = c.layer(layer, q, k, v)
            pk, pv = c.read_back()
            plain = S.CacheSpec(pk[:, layer], pv[:, layer])
            want = S.prepare_chunk_attn(c._chunk, plain, tq, L.softmax_scale(64))
            want.run()
            torch.cuda.synchronize()
            # (the same sums of the same values, in another order: a rounding of each weight
            # and of the output apart)
            d = (out.double() - want.out.double()).abs()
            assert float(d.max()) <= 4 * 2.0 ** -8 * float(pv.abs().max()), float(d.max())
    for new in ([50, 31], [1, 1], [0, 3]):
        fill(c, new)
    assert c.rows == [51, 35]
    small = c.compress([20, 12], recent=[4, 2], sinks=2, n_rows=40)
    assert small.rows == [20, 12] and small.tokens == [51, 35] and small.packed == fmt
    a, b = c.read_back()[0], small.read_back()[0]
    for s in range(2):
        for layer in range(2):
            for h in range(2):
                rows = small.row_pos[s, layer, h, : small.rows[s]].long()
                assert torch.equal(b[s, layer, h, : small.rows[s]], a[s, layer, h, rows])
    fill(small, [5, 1])
    x = small.small_inputs()
    assert x["s_k"].dtype == BF16 and x["s_k"].shape == (2, 2, 2, 40, 64)
    assert x["s_held"].tolist() == [25, 13]
    again = small.read_back(out=(x["s_k"].clone().fill_(3.0), x["s_v"].clone()), begin=[24, 0])[0]
    torch.cuda.synchronize()
    assert (again[0, :, :, :24] == 3.0).all() and torch.equal(again[0, :, :, 24], x["s_k"][0, :, :, 24])
