"""Packed caches in batches of more sequences than a wave holds, with head counts that are no power
of two, and reads and evictions captured into a graph, against the plain forms in 64 bits."""
from __future__ import annotations

import pytest
import torch

import packed_ref as P
from parity import log
from test_gpu_packed_long import Long
from test_gpu_packed_ops import NAMES, check_attn, lib, same

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
FORMATS = [P.MXFP8, P.MXFP4]

CASES = [
    ("spans of a hundred", [(1100 + 37 * (i * 29 % 100), 1) for i in range(100)], 7, 1, 128, BF16, 16, True),
    ("spans of ninety f32", [(1100 + 41 * (i * 13 % 90), 1) for i in range(90)], 7, 1, 64, F32, 32, True),
    ("spans of seventy, two columns", [(1500 + 23 * (i * 11 % 70), 1 + i % 3) for i in range(70)], 14, 2, 64, BF16,
     16, False),
    ("chunks among a hundred", [(600 + 7 * i, 1 if i % 9 else 40) for i in range(100)], 8, 2, 64, BF16, 16, True),
    ("three heads", [(900 + 100 * i, 1) for i in range(13)], 6, 3, 64, BF16, 16, True),
    ("three heads in spans", [(4000 + 900 * i, 1) for i in range(3)], 15, 3, 128, BF16, 64, True),
    ("five heads f32", [(700 + 300 * i, 2) for i in range(5)], 15, 5, 128, F32, 0, False),
    ("five heads, chunks", [(700 + 300 * i, 30 + i) for i in range(5)], 15, 5, 64, F32, 8, True),
]


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_batches(case, fmt):
    name, lens, hq, hk, d, dtype, page, absent = case
    log(f"[packed batch] {name} {NAMES[fmt]}")
    S = lib()
    c = Long(lens, hq, hk, d, dtype, fmt, page, absent, seed=len(name))
    call = S.prepare_chunk_attn(c.chunk, c.spec, c.q, c.scale)
    call.run()
    torch.cuda.synchronize()
    c.check(call)


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
def test_single_tokens_of_more_sequences_than_units(fmt):
    for n, hk in ((9, 3), (65, 1), (17, 5)):
        log(f"[packed batch] {n} sequences {hk} heads {NAMES[fmt]}")
        check_attn(P.Case([(1 + 31 * i % 90, 1) for i in range(n)], 2 * hk, hk, 64, BF16, fmt, 8, seed=n))


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
def test_captured_reads_and_evictions(fmt):
    """Replayed while rows are appended and lengths grow, against eager calls on the same rows."""
    S = lib()
    log(f"[packed batch] graph {NAMES[fmt]}")
    c = P.Case([(200, 1), (90, 1)], 4, 2, 64, BF16, fmt, 16, seed=51, cap=256)
    chunk, cache, q = c.to(DEV)
    freq, _ = S.rope_freqs(64, 10000.0)
    kv = torch.randn(2, 2, 64, generator=c.gen).to(DEV, BF16)
    keep = torch.tensor([50, 20], dtype=torch.int32, device=DEV)
    scores = torch.rand(2, 2, c.rows, generator=c.gen).to(DEV)

    def calls():
        plain = S.CacheSpec(*(torch.full((2, 2, c.rows, 64), 3.0, dtype=BF16, device=DEV) for _ in range(2)))
        to = S.PackedSpec.empty(2, 2, 64, 64, fmt)
        begin = chunk.length - 1
        return plain, to, begin, [S.prepare_read(cache, plain, chunk.length, begin=begin),
                                  S.prepare_evict(cache, to, chunk.length, keep, scores, sinks=1)]
    add = S.prepare_append(chunk, cache, S.RopeSpec(freq), q, kv, kv)
    plain, to, begin, run = calls()
    add.run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for x in [add, *run]:
            x.run()
    for _ in range(4):
        g.replay()
        torch.cuda.synchronize()
        plain2, to2, _, run2 = calls()
        for x in run2:
            x.run()
        torch.cuda.synchronize()
        for b, n in enumerate(chunk.length.tolist()):
            for x, y in ((plain.k, plain2.k), (plain.v, plain2.v)):
                same(x[b, :, n - 1], y[b, :, n - 1], "the new row")
                assert (x[b, :, n:] == 3.0).all()
        for x, y in zip(to.tensors[:4], to2.tensors[:4]):
            same(x, y, "kept rows")
        same(run[1].out_pos, run2[1].out_pos, "positions")
        chunk.length += 1
        begin += 1
        torch.cuda.synchronize()
