"""Attention scores over packed caches where a wave walks several rounds of keys, and where long
chunks in fp32 take each of the forms: against the plain form in 64 bits, within the bounds of
cache_ref.scores."""
from __future__ import annotations

import math

import pytest
import torch

import cache_ref as R
import packed_ref as P
from parity import log
from test_gpu_packed_long import Long
from test_gpu_packed_ops import NAMES, lib, within

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def per_head(c, b, kv):
    """Of one sequence and kv head: logits [new][g][n] in 64 bits (-inf: not seen) and the bound
    of their errors, as cache_ref.logits."""
    n, new = c.lens[b]
    g = c.hq // c.hk
    k, have = c.gather(c.spec.k, c.spec.k_scale, b, kv)
    q = c.q[c.starts[b]: c.starts[b + 1], kv * g: kv * g + g].double().reshape(new * g, c.d)
    x = (q @ k.t().contiguous()).view(new, g, n) * c.scale
    size = (q.abs() @ k.abs().t().contiguous()).view(new, g, n) * c.scale * (c.d + 4) * R.U
    own = n - new + torch.arange(new, device=DEV)
    seen = ((torch.arange(n, device=DEV) <= own[:, None]) & have)[:, None]
    return x.masked_fill(~seen, -math.inf), size * seen


def check_scores(c):
    """Per kv head and per query head, added to earlier scores in place and beside them."""
    S = lib()
    g, gen = c.hq // c.hk, torch.Generator(device=DEV).manual_seed(9)
    parts = {(b, kv): per_head(c, b, kv) for b in range(len(c.lens)) for kv in range(c.hk)}
    lse = torch.full((c.T, c.hq), -math.inf, device=DEV)
    for (b, kv), (x, _) in parts.items():
        lse[c.starts[b]: c.starts[b + 1], kv * g: kv * g + g] = torch.logsumexp(x, -1).float()
    for heads in sorted({c.hk, c.hq}):
        before = torch.rand(len(c.lens), heads, c.rows, device=DEV, generator=gen)
        out = torch.full_like(before, -7.0)
        S.prepare_chunk_scores(c.chunk, c.spec, c.q, lse, c.scale, out, before=before).run()
        same = before.clone()
        S.prepare_chunk_scores(c.chunk, c.spec, c.q, lse, c.scale, same, before=same).run()
        torch.cuda.synchronize()
        for b, (n, new) in enumerate(c.lens):
            assert torch.equal(same[b, :, :n], out[b, :, :n])
            assert (out[b, :, n:] == -7.0).all() and torch.equal(same[b, :, n:], before[b, :, n:])
            for kv in range(c.hk):
                x, dx = parts[b, kv]
                e = lse[c.starts[b]: c.starts[b + 1], kv * g: kv * g + g].double()[..., None]
                unseen = torch.isinf(x)
                p = torch.exp(x - e)
                arg = (x.masked_fill(unseen, 0.0).abs() + e.abs() + 1) * 4 * R.U
                w = p * (dx + arg + 4 * R.U + (new * g + 64) * R.U)
                s, t = p.sum(0), w.sum(0)
                hs = slice(kv * g, kv * g + g)
                if heads != c.hq:
                    s, t, hs = s.sum(0, keepdim=True), t.sum(0, keepdim=True), slice(kv, kv + 1)
                s[:, : n - new] += before[b, hs, : n - new].double()
                tol = t + 2 * R.U * s.abs()
                within(out[b, hs, :n], s.cpu(), tol.cpu(), f"scores of {b}, head {kv} of {heads}")


def ragged(count, lo, hi, new=1):
    return [(lo + (hi - lo) * (i * 7 % count) // max(count - 1, 1), 1 + i % new) for i in range(count)]


CASES = [
    # decode steps: up to 11 rounds of 128 keys a wave
    ("a token each", ragged(24, 1000, 8000), 28, 4, 128, BF16, 16, True),
    ("a token each, dense", ragged(40, 1, 5000), 14, 2, 64, BF16, 0, False),
    ("a token each f32", ragged(24, 1000, 8000), 14, 2, 64, F32, 32, True),
    ("a token each f32 of 128", ragged(16, 900, 7001), 28, 4, 128, F32, 64, False),
    ("one to three tokens", ragged(30, 700, 6000, 3), 14, 2, 128, BF16, 16, True),
    ("two tokens of 64", ragged(30, 700, 6000, 2), 32, 2, 64, BF16, 8, True),
    ("one to three tokens f32", ragged(30, 700, 6000, 3), 14, 2, 64, F32, 16, True),
    ("a token each of many heads", ragged(20, 2000, 7000), 32, 1, 128, BF16, 16, False),
    # chunks: heads that share a workgroup's keys, long ones
    ("short chunks f32", [(3000, 16), (2500, 9), (40, 5)], 14, 2, 64, F32, 16, True),
    ("chunks f32", [(5000, 60), (4000, 33), (4500, 40)], 8, 4, 64, F32, 32, False),
    ("chunks f32 of 128", [(3000, 100), (2222, 41)], 8, 2, 128, F32, 0, False),
    ("long chunks f32", [(2500, 200), (1700, 131)], 8, 4, 128, F32, 64, True),
    ("long chunks f32 of 64", [(4100, 300), (64, 64)], 14, 2, 64, F32, 16, False),
    ("long chunks", [(2500, 200), (1700, 131)], 8, 4, 64, BF16, 64, True),
]


@pytest.mark.parametrize("fmt", [P.MXFP8, P.MXFP4], ids=NAMES.get)
@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_scores_over_long_sequences(case, fmt):
    name, lens, hq, hk, d, dtype, page, absent = case
    log(f"[packed scores] {name} {NAMES[fmt]}")
    check_scores(Long(lens, hq, hk, d, dtype, fmt, page, absent, seed=len(name)))
