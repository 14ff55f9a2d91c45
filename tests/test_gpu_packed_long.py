"""The packed cache's operators over sequences whose tiles a wave walks one after another, in
whole sequences and in spans, over far-apart and shared memory, and around what a batch
leaves out.  Plain forms in 64 bits of the rows that the codes stand for."""
from __future__ import annotations

import math

import pytest
import torch

import cache_ref as R
import packed_ref as P
from parity import log
from test_gpu_packed_ops import NAMES, same, within

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def lib():
    from paper_2508_02751_amd import smallkv as S
    return S


class Long:
    """Packed caches of long sequences, made and gathered on the GPU; codes and scales are random
    bytes that stand for numbers, those of rows that belong to nobody all ones (NaN)."""

    def __init__(self, lens, hq, hk, d, dtype, fmt, page, absent=False, seed=0):
        S = lib()
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.lens, self.hq, self.hk, self.d, self.dtype, self.fmt = lens, hq, hk, d, dtype, fmt
        self.rows = max(n for n, _ in lens)
        B, per = len(lens), page or self.rows
        width = (self.rows + per - 1) // per
        pages = B * width + (2 if page else 0)
        table = None
        if page:
            table = torch.randperm(pages, device=DEV, generator=g)[: B * width].view(B, width).int()
            if absent:  # every 23rd page, not the first
                table[:, 22::23] = torch.tensor(-1, device=DEV, dtype=torch.int32)
        self.spec = S.PackedSpec.empty(pages, hk, per, d, fmt, table)
        for t in self.spec.tensors[:4]:
            t.fill_(255)
        self.at, self.starts = [], [0]
        for b, (n, new) in enumerate(lens):
            r = torch.arange(n, device=DEV)
            p = r * 0 + b if table is None else table[b].long()[r // per]
            have = p >= 0
            self.at.append((p.clamp(min=0), r % per, have))
            for codes, scales in ((self.spec.k, self.spec.k_scale), (self.spec.v, self.spec.v_scale)):
                x = torch.randint(0, 256, (n, hk, codes.shape[3]), device=DEV, generator=g, dtype=torch.uint8)
                if fmt == P.MXFP8:  # numbers up to 15 (the exponent's top bit cleared: no NaN)
                    x = x & 0xBF
                e = torch.randint(124, 128, (n, hk, d // 32), device=DEV, generator=g, dtype=torch.uint8)
                codes[p[have], :, (r % per)[have]] = x[have]
                scales[p[have], :, (r % per)[have]] = e[have]
            self.starts.append(self.starts[-1] + new)
        self.T = self.starts[-1]
        self.q = torch.randn(self.T, hq, d, device=DEV, generator=g).to(dtype)
        self.scale = 1.0 / math.sqrt(d)
        self.chunk = S.ChunkSpec(torch.tensor(self.starts, dtype=torch.int32, device=DEV),
                                 torch.tensor([n for n, _ in lens], dtype=torch.int32, device=DEV), self.T,
                                 max(new for _, new in lens), self.rows)
        self.table = P.code_values(fmt).to(DEV)

    def gather(self, codes, scales, b, h):
        """[n][d] in 64 bits (0: absent)."""
        p, i, have = self.at[b]
        c = codes[p, h, i].long()
        x = self.table[c] if self.fmt == P.MXFP8 else torch.stack([self.table[c % 16], self.table[c // 16]],
                                                                  -1).flatten(-2)
        x = x * torch.exp2(scales[p, h, i].double() - 127).repeat_interleave(32, -1)
        return torch.where(have[:, None], x, torch.zeros(()).double().to(DEV)), have

    def check(self, call):
        """out and lse against the plain form, within the bounds of cache_ref.attention."""
        g, U, h = self.hq // self.hk, R.U, R.HALF[self.dtype]
        for b, (n, new) in enumerate(self.lens):
            rows = slice(self.starts[b], self.starts[b + 1])
            own = n - new + torch.arange(new, device=DEV)
            for kv in range(self.hk):
                k, have = self.gather(self.spec.k, self.spec.k_scale, b, kv)
                v, _ = self.gather(self.spec.v, self.spec.v_scale, b, kv)
                hs = slice(kv * g, kv * g + g)
                q = self.q[rows, hs].double().reshape(new * g, self.d)
                x = (q @ k.t().contiguous()).view(new, g, n) * self.scale
                size = (q.abs() @ k.abs().t().contiguous()).view(new, g, n) * self.scale * (self.d + 4) * U
                seen = ((torch.arange(n, device=DEV) <= own[:, None]) & have)[:, None]
                x = x.masked_fill(~seen, -math.inf)
                e = torch.logsumexp(x, -1)
                w = torch.exp(x - e[..., None])
                d = (size * seen).amax(-1)
                out = (w.view(new * g, n) @ v).view(new, g, self.d)
                a = (w.view(new * g, n) @ v.abs()).view(new, g, self.d)
                tol = a * (2 * d + (n + 64) * U)[..., None] + (
                    1.01 * h * (a + out.abs()) if self.dtype == BF16 else h * out.abs())
                ltol = d + (n + 64) * U + 8 * U * e.abs() + 8 * U
                within(call.out[rows, hs], out.cpu(), tol.cpu(), f"out of {b}, head {kv}")
                within(call.lse[rows, hs], e.cpu(), ltol.cpu(), f"lse of {b}, head {kv}")


CASES = [
    # whole sequences by eight waves, by four; spans; one sequence in many
    ("whole, eight waves", [(1500 - 37 * i, 1) for i in range(40)], 8, 4, 64, BF16, 16, True),
    ("whole, eight waves f32", [(1100 - 23 * i, 1) for i in range(40)], 8, 4, 128, F32, 32, False),
    ("whole, four waves", [(700 - 7 * i, 1) for i in range(70)], 8, 4, 64, BF16, 16, True),
    ("spans", [(20011, 1), (33, 1), (9000, 1), (1, 1)], 14, 2, 128, BF16, 16, True),
    ("spans f32", [(9000, 1), (128, 1), (5001, 1)], 14, 2, 128, F32, 64, True),
    ("spans, two columns", [(9000, 4), (130, 2), (5001, 3)], 14, 2, 128, BF16, 64, True),
    ("spans, two columns of 64", [(6000, 2), (5001, 1)], 32, 2, 64, BF16, 8, False),
    ("tiles of 16 f32", [(6000, 8), (5001, 5), (40, 2)], 14, 2, 64, F32, 16, True),
    ("tiles of 256", [(3000, 500), (2500, 700)], 8, 2, 128, BF16, 64, True),
    ("tiles of 256 of 64, spans", [(9000, 800)], 8, 2, 64, BF16, 0, False),
    ("many rows f32", [(3000, 300), (700, 40)], 8, 2, 128, F32, 16, True),
    ("dense, one sequence", [(30000, 1)], 8, 1, 128, BF16, 0, False),
]


@pytest.mark.parametrize("fmt", [P.MXFP8, P.MXFP4], ids=NAMES.get)
@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_long_sequences(case, fmt):
    name, lens, hq, hk, d, dtype, page, absent = case
    log(f"[packed long] {name} {NAMES[fmt]}")
    S = lib()
    c = Long(lens, hq, hk, d, dtype, fmt, page, absent, seed=len(name))
    call = S.prepare_chunk_attn(c.chunk, c.spec, c.q, c.scale)
    call.run()
    torch.cuda.synchronize()
    c.check(call)
    first = call.out.clone(), call.lse.clone()
    call.run()  # the same workspace again, the same bits
    torch.cuda.synchronize()
    assert torch.equal(call.out, first[0]) and torch.equal(call.lse, first[1])


@pytest.mark.parametrize("fmt", [P.MXFP8, P.MXFP4], ids=NAMES.get)
def test_lengths_that_a_captured_step_meets_later(fmt):
    """One prepared call, whose lengths change on the device: every split of the rows."""
    S = lib()
    log(f"[packed long] growing lengths {NAMES[fmt]}")
    full = [(6000, 1), (6000, 1)]
    c = Long(full, 8, 2, 64, BF16, fmt, 16, seed=3)
    call = S.prepare_chunk_attn(c.chunk, c.spec, c.q, c.scale)
    for lens in ([1, 31], [32, 33], [129, 127], [513, 4000], [6000, 2], [0, 5999]):
        c.chunk.length.copy_(torch.tensor(lens, dtype=torch.int32))
        call.run()
        torch.cuda.synchronize()
        c.lens = [(max(n, 1), 1) for n in lens]
        at, c.at = c.at, [tuple(x[: max(n, 1)] for x in a) for a, n in zip(c.at, lens)]
        if 0 in lens:
            assert (call.out[lens.index(0)] == 0).all() and torch.isinf(call.lse[lens.index(0)]).all()
            i = 1 - lens.index(0)
            c.lens = [x if j == i else (1, 0) for j, x in enumerate(c.lens)]
            starts, c.starts = c.starts, [0, 0, 1] if i else [0, 1, 1]
            rows = call.out[i: i + 1], call.lse[i: i + 1]
            q, c.q = c.q, c.q[i: i + 1]
            c.check(type("Call", (), dict(out=rows[0], lse=rows[1])))
            c.q, c.starts = q, starts
        else:
            c.check(call)
        c.at = at


def test_far_apart_pages():
    """Codes and scales whose offsets pass 32 bits, of pages that share one large buffer."""
    S = lib()
    log("[packed long] far apart")
    c = P.Case([(70, 1), (40, 1)], 4, 2, 128, BF16, P.MXFP8, 16, seed=5)
    chunk, cache, q = c.to(DEV)
    pages = cache.k.shape[0]
    stride = (6 << 30) // pages // 4096 * 4096
    buf = torch.empty(stride * pages, dtype=torch.uint8, device=DEV)
    far = []
    for i, t in enumerate(cache.tensors[:4]):
        x = torch.as_strided(buf, t.shape, (stride, *t.stride()[1:]), i << 20)
        x.copy_(t)
        far.append(x)
    assert far[0].stride(0) * (pages - 1) > 1 << 32
    spec = S.PackedSpec(*far, P.MXFP8, cache.page_table)
    want = S.prepare_chunk_attn(chunk, cache, q, c.scale)
    got = S.prepare_chunk_attn(chunk, spec, q, c.scale)
    scores = [torch.zeros(2, 2, c.rows, device=DEV) for _ in range(2)]
    freq, _ = S.rope_freqs(128, 10000.0)
    kv = torch.randn(2, 2, 128).to(DEV, BF16)
    plain = [S.CacheSpec(*(torch.zeros(2, 2, c.rows, 128, dtype=BF16, device=DEV) for _ in range(2))) for _ in range(2)]
    for x, call, s, to in ((cache, want, scores[0], plain[0]), (spec, got, scores[1], plain[1])):
        call.run()
        S.prepare_chunk_scores(chunk, x, q, want.lse, c.scale, s).run()
        S.prepare_append(chunk, x, S.RopeSpec(freq), q, kv, kv).run()
        S.prepare_read(x, to, chunk.length).run()
    torch.cuda.synchronize()
    same(got.out, want.out, "out")
    same(got.lse, want.lse, "lse")
    same(scores[1], scores[0], "scores")
    same(plain[1].k, plain[0].k, "k")
    same(plain[1].v, plain[0].v, "v")
    for x, y in zip(far, cache.tensors):
        same(x, y, "codes")
    to = S.PackedSpec.empty(2, 2, 64, 128)
    to2 = S.PackedSpec.empty(2, 2, 64, 128)
    for x, y in ((cache, to), (spec, to2)):
        S.prepare_evict(x, y, chunk.length, chunk.length // 2, scores[0], sinks=1).run()
    torch.cuda.synchronize()
    for x, y in zip(to.tensors[:4], to2.tensors[:4]):
        same(x, y, "kept rows")


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 60])
def test_shared_rows_and_strided_tokens(new, dtype):
    """One kv head's rows for all of them (a stride of 0), queries and outputs inside wider rows."""
    S = lib()
    log(f"[packed long] shared rows {new} {dtype}")
    c = P.Case([(90, new), (70, new)], 4, 1, 64, dtype, P.MXFP4, 16, seed=6)
    chunk, cache, q = c.to(DEV)
    wide = torch.zeros(c.T, 3, 8, 64, dtype=dtype, device=DEV)
    qs, out = wide[:, 0, ::2], torch.full_like(wide, 9.0)[:, 1, 1::2]
    qs.copy_(q)
    spec = S.PackedSpec(*(t.expand(-1, 2, -1, -1) for t in cache.tensors[:4]), P.MXFP4, cache.page_table)
    call = S.prepare_chunk_attn(chunk, spec, qs, c.scale, out=out)
    call.run()
    torch.cuda.synchronize()
    want, want_lse, tol, ltol = R.attention(c)
    within(call.out, want, tol, "out")
    within(call.lse, want_lse, ltol, "lse")
    base = out._base
    touched = torch.zeros_like(base, dtype=torch.bool)
    touched[:, 1, 1::2] = True
    assert (base[~touched] == 9.0).all()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("lens", [[(50, 1), (0, 0), (9, 1)], [(300, 70), (64, 0), (30, 30)]], ids=["few", "many"])
def test_what_a_batch_leaves_out(lens, dtype):
    """Tokens of no sequence, past max_new, and lengths past max_len: nothing of theirs is read or
    written; an empty chunk does nothing."""
    S = lib()
    log(f"[packed long] left out {lens} {dtype}")
    c = P.Case(lens, 4, 2, 64, dtype, P.MXFP8, 8, seed=7, extra_tokens=3)
    chunk, cache, q = c.to(DEV)
    q[c.starts[-1]:] = math.nan
    out = torch.full_like(q, 5.0)
    lse = torch.full((c.T, 4), 6.0, device=DEV)
    S.prepare_chunk_attn(chunk, cache, q, c.scale, out=out, lse=lse).run()
    torch.cuda.synchronize()
    want, want_lse, tol, ltol = R.attention(c)
    n = c.starts[-1]
    within(out[:n], want[:n], tol[:n], "out")
    within(lse[:n], want_lse[:n], ltol[:n], "lse")
    assert (out[n:] == 5.0).all() and (lse[n:] == 6.0).all()
    # fewer new tokens than the batch has: the first of each sequence
    few = S.ChunkSpec(chunk.start, chunk.length, c.T, 1, c.rows)
    out.fill_(5.0)
    S.prepare_chunk_attn(few, cache, q, c.scale, out=out).run()
    torch.cuda.synchronize()
    first = torch.zeros(c.T, dtype=torch.bool)
    for b, (_, new) in enumerate(lens):
        if new:
            first[c.starts[b]] = True
    assert (out[~first.to(DEV)] == 5.0).all() and not (out[first.to(DEV)] == 5.0).all()
    # no tokens at all
    none = S.ChunkSpec(torch.zeros_like(chunk.start), chunk.length, 0, 1, c.rows)
    before = [t.clone() for t in cache.tensors[:4]]
    empty = q[:0]
    S.prepare_chunk_attn(none, cache, empty, c.scale).run()
    freq, _ = S.rope_freqs(64, 10000.0)
    S.prepare_append(none, cache, S.RopeSpec(freq), empty, empty[:, :2], empty[:, :2]).run()
    scores = torch.full((len(lens), 2, c.rows), 3.0, device=DEV)
    S.prepare_chunk_scores(none, cache, empty, lse[:0], c.scale, scores, before=scores).run()
    torch.cuda.synchronize()
    assert (scores == 3.0).all()
    for x, y in zip(cache.tensors, before):
        same(x, y, "rows")


def test_a_packed_cache_of_every_code():
    """Every code of 8 bits under every scale that a number has, read back and attended to by one
    token whose weights are equal (keys 0): the mean of the values."""
    S = lib()
    log("[packed long] every code")
    v = torch.arange(256, dtype=torch.uint8)
    v[127], v[255] = 0, 128
    rows = v.view(8, 32).repeat(1, 2).view(8, 1, 64)
    spec = S.PackedSpec.empty(1, 1, 8, 64, device=DEV)
    to = S.CacheSpec(*(torch.zeros(1, 1, 8, 64, dtype=F32, device=DEV) for _ in range(2)))
    spec.v.copy_(rows.view(1, 1, 8, 64).to(DEV))
    n = torch.tensor([8], dtype=torch.int32, device=DEV)
    for x in range(27, 246):
        spec.v_scale.fill_(x)
        S.prepare_read(spec, to, n).run()
        want = P.unpack(rows.view(8, 64), torch.full((8, 2), x, dtype=torch.uint8), P.MXFP8)
        same(to.v.view(8, 64), want.float(), f"scale {x}")
