"""Values at the edges of packed caches and of the queries over them: NaN of every payload, rows
of codes 0 under any scale, every code under every scale that an append writes, each read back
and attended to, against the plain forms in 64 bits."""
from __future__ import annotations

import math

import pytest
import torch

import cache_ref as R
import packed_ref as P
from parity import log
from test_gpu_packed_ops import NAMES, lib, same, within

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
FORMATS = [P.MXFP8, P.MXFP4]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("lens", [[(70, 5)], [(300, 100)], [(5000, 1)]], ids=["few", "many", "spans"])
def test_nan_queries_whatever_their_payload(lens, fmt, dtype):
    """A NaN element makes its query's output NaN, also where only its lowest bit says so, over
    keys of one sign there (an infinite one would leave every logit -inf, or one of them +inf)."""
    S = lib()
    log(f"[packed] NaN queries {lens} {NAMES[fmt]} {dtype}")
    for d, sign in ((64, -1.0), (128, 1.0)):
        c = P.Case(lens, 4, 2, d, dtype, fmt, 16, seed=41)
        c.k[..., 5] = sign * 2.0
        c.pack()
        clean = R.attention(c)
        bits = c.q.view(torch.int32 if dtype == F32 else torch.int16)
        low = 0x7F800001 if dtype == F32 else 0x7F81
        bits[0, 1, 5] = low
        bits[-1, 3, 5] = low - (1 << (31 if dtype == F32 else 15))  # the same, negative
        assert int(torch.isnan(c.q).sum()) == 2
        chunk, cache, q = c.to(DEV)
        call = S.prepare_chunk_attn(chunk, cache, q, c.scale)
        call.run()
        torch.cuda.synchronize()
        out, lse = call.out.cpu(), call.lse.cpu()
        hit = torch.zeros(c.T, 4, dtype=torch.bool)
        hit[0, 1] = hit[-1, 3] = True
        assert torch.isnan(out[hit]).all() and torch.isnan(lse[hit]).all(), (out[hit], lse[hit])
        within(out[~hit], clean[0][~hit], clean[2][~hit], "out")
        within(lse[~hit], clean[1][~hit], clean[3][~hit], "lse")


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("lens", [[(70, 1), (9, 1)], [(300, 70), (40, 1)]], ids=["few", "many"])
def test_codes_of_0_are_0_under_every_scale(lens, fmt, dtype):
    """Rows of zeros (PackedSpec.empty's have scales 0): read, attended to and scored."""
    S = lib()
    log(f"[packed] codes 0 {lens} {NAMES[fmt]} {dtype}")
    c = P.Case(lens, 14, 2, 64, dtype, fmt, 16, seed=42)
    zeros = torch.tensor([0, 128] if fmt == P.MXFP8 else [0, 8, 128, 136], dtype=torch.uint8)
    for i, t in enumerate(c.codes):
        if i % 2:
            t.copy_(torch.randint(0, 255, t.shape, generator=c.gen, dtype=torch.uint8))
        else:
            t.copy_(zeros[torch.randint(0, len(zeros), t.shape, generator=c.gen)])
    c.codes[1][:, :, ::3] = 0
    c.codes[3][:, :, 1::3] = 254
    c.refresh()
    chunk, cache, q = c.to(DEV)
    call = S.prepare_chunk_attn(chunk, cache, q, c.scale)
    call.run()
    scores = torch.zeros(c.B, 14, c.rows, device=DEV)
    S.prepare_chunk_scores(chunk, cache, q, call.lse, c.scale, scores).run()
    to = S.CacheSpec(*(torch.full((c.B, 2, c.rows, 64), 5.0, dtype=dtype, device=DEV) for _ in range(2)))
    S.prepare_read(cache, to, chunk.length).run()
    torch.cuda.synchronize()
    assert (call.out == 0).all()
    _, lse, _, ltol = R.attention(c)
    within(call.lse, lse, ltol, "lse")
    want, tol = R.scores(c, call.lse.cpu(), torch.zeros(c.B, 14, c.rows), per_kv=False)
    for b, (n, _) in enumerate(c.lens):
        assert (to.k[b, :, :n] == 0).all() and (to.v[b, :, :n] == 0).all()
        within(scores[b, :, :n], want[b, :, :n], tol[b, :, :n], f"scores of {b}")


def test_an_empty_cache_holds_zeros():
    S = lib()
    log("[packed] empty")
    for fmt in FORMATS:
        cache = S.PackedSpec.empty(3, 2, 32, 128, fmt)
        to = S.CacheSpec(*(torch.full((3, 2, 32, 128), 5.0, dtype=F32, device=DEV) for _ in range(2)))
        length = torch.tensor([32, 1, 17], dtype=torch.int32, device=DEV)
        S.prepare_read(cache, to, length).run()
        chunk = S.ChunkSpec(torch.tensor([0, 1, 2, 3], dtype=torch.int32, device=DEV), length, 3, 1, 32)
        q = torch.randn(3, 4, 128, device=DEV)
        call = S.prepare_chunk_attn(chunk, cache, q, 0.1)
        call.run()
        torch.cuda.synchronize()
        for b, n in enumerate((32, 1, 17)):
            assert (to.k[b, :, :n] == 0).all() and (to.v[b, :, n:] == 5.0).all()
        assert (call.out == 0).all()
        want = length.cpu().double().log()[:, None].expand(3, 4)
        within(call.lse, want, 8 * R.U * (1 + want), "lse")


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
def test_every_code_under_every_scale(fmt, dtype):
    """Read back, under every scale that an append writes; and attended to by a token whose
    weights are equal (keys 0): the mean of the values, under those that do not overflow in it."""
    S = lib()
    log(f"[packed] every code {NAMES[fmt]} {dtype}")
    g = torch.Generator().manual_seed(43)
    codes = torch.arange(256, dtype=torch.uint8)
    if fmt == P.MXFP8:
        codes[127], codes[255] = 0, 128  # (no NaN)
    codes = codes[torch.randperm(256, generator=g)]
    width = 64 if fmt == P.MXFP8 else 32
    rows = codes.view(-1, width)
    n = rows.shape[0]
    cache = S.PackedSpec.empty(1, 1, n, 64, fmt)
    cache.v.copy_(rows.view(1, 1, n, width).to(DEV))
    to = S.CacheSpec(*(torch.zeros(1, 1, n, 64, dtype=dtype, device=DEV) for _ in range(2)))
    length = torch.tensor([n], dtype=torch.int32, device=DEV)
    chunk = S.ChunkSpec(torch.tensor([0, 1], dtype=torch.int32, device=DEV), length, 1, 1, n)
    q = torch.randn(1, 2, 64, generator=g).to(DEV, dtype)
    read = S.prepare_read(cache, to, length)
    attn = S.prepare_chunk_attn(chunk, cache, q, 0.125)
    for x in range(27, 247 if fmt == P.MXFP8 else 253):
        cache.v_scale.fill_(x)
        read.run()
        attn.run()
        torch.cuda.synchronize()
        want = P.unpack(rows, torch.full((n, 2), x, dtype=torch.uint8), fmt)
        same(to.v.view(n, 64), want.to(dtype), f"scale {x}")
        if x > 240:  # (a sum of n values of up to 448 * 2^113, or 6 * 2^113, is below 2^128)
            continue
        # n sums, a division and its product, each off by a rounding of fp32 of at most the sum of
        # magnitudes; the output's rounding
        mean, size = want.mean(0), want.abs().mean(0)
        tol = (n + 4) * R.U * size + 1.01 * R.HALF[dtype] * mean.abs()
        within(attn.out.view(2, 64), mean.expand(2, 64), tol.expand(2, 64), f"mean under scale {x}")
        within(attn.lse, torch.full((1, 2), math.log(n)), torch.full((1, 2), 8 * R.U * (1 + math.log(n))), "lse")
    # what an append makes of a block with an infinity: codes 0, scale 255
    cache.v.zero_()
    cache.v_scale.zero_()
    cache.v_scale[0, 0, 1, 1] = 255
    read.run()
    attn.run()
    torch.cuda.synchronize()
    hit = torch.zeros(64, dtype=torch.bool)
    hit[32:] = True
    assert torch.isnan(to.v[0, 0, 1, 32:]).all() and (to.v[0, 0, 1, :32] == 0).all() and (to.v[0, 0, 2:] == 0).all()
    assert torch.isnan(attn.out[0, :, hit]).all() and (attn.out[0, :, ~hit] == 0).all()
