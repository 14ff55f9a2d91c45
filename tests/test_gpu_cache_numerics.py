"""How exactly the cache operators weigh rows: the probabilities of bf16 models, against
plain forms in 64 bits, within derived bounds."""
from __future__ import annotations

import math

import pytest
import torch

import cache_ref as R
from parity import log
from test_gpu_cache_ops import within

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def lib():
    from paper_2508_02751_amd import smallkv as S
    return S


# (name, sequences (rows, new), hq, hk, d, page, rows of a token's group that share a tile:
# few or many)
SHAPES = [
    ("chunk in spans", [(700, 150), (300, 90)], 8, 2, 128, 16, False),
    ("chunk in spans d64", [(700, 150), (300, 90)], 8, 2, 64, 16, False),
    ("chunks without spans", [(300, 40)] * 32, 16, 16, 128, 32, False),
    ("chunks without spans d64", [(200, 200), (150, 70)] * 24, 16, 16, 64, 0, False),
    ("tokens in spans", [(1500, 1), (700, 1), (33, 1)], 14, 2, 64, 16, True),
    ("tokens in spans d128", [(1500, 3), (700, 2)], 8, 2, 128, 16, True),
    ("tokens without spans", [(400, 1)] * 40, 16, 16, 128, 0, True),
]
IDS = [c[0].replace(" ", "-") for c in SHAPES]


def build(case, spread):
    _, lens, hq, hk, d, page, few = case
    c = R.Case(lens, hq, hk, d, BF16, page, seed=71)
    # logits of this spread, the largest of them anywhere in the sequence: single rows
    # with most of the weight, whose probabilities are not powers of two
    c.q = (c.q.float() * spread).to(BF16)
    return c, few


@pytest.mark.parametrize("case", SHAPES, ids=IDS)
def test_the_weights_add_up_to_one(case):
    """With every value 1 the output is 1: what the weights are rounded to adds up to what
    they are divided by, up to sums in fp32 (and 2^-16 for P in two parts), less than
    half a step of bf16 below 1 (2^-9)."""
    S = lib()
    c, _ = build(case, 3.0)
    c.v[~torch.isnan(c.v)] = 1.0
    chunk, cache, q = c.to(DEV)
    log(f"[ones] {case[0]}")
    call = S.prepare_chunk_attn(chunk, cache, q, c.scale)
    call.run()
    torch.cuda.synchronize()
    assert bool((call.out == 1.0).all()), f"{int((call.out != 1.0).sum())} of {call.out.numel()}"


@pytest.mark.parametrize("spread", [0.3, 1.0, 3.0])
@pytest.mark.parametrize("case", SHAPES, ids=IDS)
def test_probabilities_of_bf16_models(case, spread):
    """Few rows: P in two bf16 parts, 2^-16 relative.  Many: one part, each weight w off by
    up to w 2^-8, and divided by the sum of the rounded ones, so that a row's output o moves
    by at most 2^-8 sum w |v - o| (and second order, below 2^-7 of it)."""
    S = lib()
    c, few = build(case, spread)
    c.v += 2.0  # a common part, which the weights must not scale
    chunk, cache, q = c.to(DEV)
    log(f"[bf16 weights] {case[0]} {spread}")
    call = S.prepare_chunk_attn(chunk, cache, q, c.scale)
    call.run()
    torch.cuda.synchronize()
    h, g = R.HALF[BF16], c.hq // c.hk
    for b, (n, new) in enumerate(c.lens):
        x, dx = R.logits(c, b)
        v, _ = c.gather(c.v, b, n)
        p = torch.softmax(x, -1)
        o = torch.matmul(p, v[:, None])
        away = torch.zeros_like(o)  # sum w |v - o|
        for t in range(new):
            away[:, :, t] = (p[:, :, t, :, None] * (v[:, None] - o[:, :, t, None]).abs()).sum(2)
        a = torch.matmul(p, v.abs()[:, None])
        tol = a * (2 * dx.amax(-1) + 2 * (n + 64) * R.U)[..., None] + 1.01 * h * o.abs()
        tol += a * 2.0 ** -16 if few else 1.01 * h * away
        rows = slice(c.starts[b], c.starts[b] + new)

        def flat(t):
            return t.movedim(2, 0).reshape(new, c.hq, c.d)
        within(call.out[rows], flat(o), flat(tol), f"sequence {b}")


@pytest.mark.parametrize("lens,per_kv", [
    ([(300, 1), (77, 1)], True), ([(300, 1), (77, 3)], False),     # rows of K streamed
    ([(300, 20), (90, 12)], False), ([(400, 60)], False),          # several heads a workgroup
    ([(400, 30)], True), ([(500, 140)], False),                    # keys in 32s, rows dealt
    ([(300, 40)] * 30, True), ([(300, 130)] * 12, False)])         # keys in 128s
@pytest.mark.parametrize("d", [64, 128])
def test_fp32_scores_of_large_logits(d, lens, per_kv):
    """Logits of 4000 that are exact (whole numbers times the scale): what is left is the
    rounding of logit - lse, of its product with log2(e) and of the exponential, each
    relative to the difference and not to the logit, and the sums."""
    S = lib()
    c = R.Case(lens, 8, 2, d, F32, 16, seed=73)
    g = torch.Generator().manual_seed(d)
    u = torch.randint(1, 4, (d,), generator=g).float() * (2 * torch.randint(0, 2, (d,), generator=g) - 1)

    def near(x, shape):  # x and a few elements of it changed
        change = torch.randint(-1, 2, (*shape, d), generator=g) * (torch.rand(*shape, d, generator=g) < 0.05)
        return x + change.float()
    c.scale = float(torch.tensor(1.0 / math.sqrt(d)))
    size = int(4000 / (float((u * u).sum()) * c.scale) / 4)
    for b, (n, _) in enumerate(lens):
        for r in range(n):
            p, i = c.slot(b, r)
            c.k[p, :, i] = near(u * size, (c.hk,))
    c.q = near(u * 4, (c.T, c.hq))
    chunk, cache, q = c.to(DEV)
    x = [R.logits(c, b)[0] for b in range(c.B)]
    lse = torch.cat([torch.logsumexp(x[b], -1).permute(2, 0, 1).reshape(new, c.hq)
                     for b, (_, new) in enumerate(lens)]).float()
    assert 3000 < float(lse.min()) and float(lse.max()) < 5000
    heads = c.hk if per_kv else c.hq
    out = torch.zeros(c.B, heads, c.rows, device=DEV)
    log(f"[fp32 scores] {d} {len(lens)} {lens[0]} per_kv={per_kv}")
    S.prepare_chunk_scores(chunk, cache, q, lse.to(DEV), c.scale, out).run()
    torch.cuda.synchronize()
    group = c.hq // c.hk
    for b, (n, new) in enumerate(lens):
        e = lse[c.starts[b]: c.starts[b] + new].double().view(new, c.hk, group).permute(1, 2, 0)[..., None]
        t = x[b] - e
        w = torch.exp(t)
        tol = w * ((3 * t.abs().nan_to_num(0, 0, 0) + 4 + (new * group if per_kv else new) + 64) * R.U)
        w, tol = w.sum(2), tol.sum(2)
        if per_kv:
            w, tol = w.sum(1), tol.sum(1)
        within(out[b, :, :n], w.reshape(heads, n), tol.reshape(heads, n), f"sequence {b}")


@pytest.mark.parametrize("dtype,d", [(BF16, 64), (BF16, 128), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("new,hq", [(40, 8), (3, 8), (1, 8), (8, 16)])
@pytest.mark.parametrize("pages", [[5], [33], [37], list(range(16, 32)), [4, 34, 36]], ids=str)
def test_infinite_values_of_rows_without_weight(pages, new, hq, dtype, d):
    """Rows that are seen with a logit of -inf, in tiles that every token sees whole, in the
    last ones and over whole spans: 0 times their infinite and NaN values is NaN for
    the tokens that see them, and nothing else of the output changes."""
    S = lib()
    c = R.Case([(300, new), (70, min(new, 1))], hq, 2, d, dtype, 8, seed=79)
    c.q = c.q.abs()
    lo, at = {}, [3, d // 2, d - 1]
    for j, page in enumerate(pages):
        p, e = int(c.table[0, page]), at[j % 3]
        c.k[p, :, :, 3] = -math.inf
        c.v[p, :, 2, e] = (math.inf, -math.inf, math.nan)[j % 3]
        lo[e] = min(lo.get(e, 1 << 30), 8 * page + 2)
    chunk, cache, q = c.to(DEV)
    c.table = c.table.clone()
    c.table[0, pages] = -1  # for the plain form: no weight
    want, wl, tol, ltol = R.attention(c)
    for t in range(new):
        for e, row in lo.items():
            if row <= 300 - new + t:
                want[t, :, e] = math.nan
    log(f"[0 * inf] {dtype} {d} {new} {hq} pages {pages}")
    call = S.prepare_chunk_attn(chunk, cache, q, c.scale)
    call.run()
    torch.cuda.synchronize()
    within(call.out, want, tol, "out")
    within(call.lse, wl, ltol, "lse")


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 64)])
@pytest.mark.parametrize("lens", [[(70, 40), (1000, 3)], [(5, 1), (1000, 2)], [(64, 64), (9, 9)], [(20, 1)] * 300],
                         ids=str)
def test_rows_of_minus_infinity_only(lens, dtype, d):
    """Logits that are all -inf: an output of 0 and an lse of -inf, whatever the values."""
    S = lib()
    c = R.Case(lens, 8, 2, d, dtype, 8, seed=83)
    c.q = c.q.abs()
    c.k[..., 7] = -math.inf
    c.v[..., 2] = math.inf
    c.v[..., 5] = math.nan
    chunk, cache, q = c.to(DEV)
    log(f"[only -inf] {dtype} {lens[:2]}")
    call = S.prepare_chunk_attn(chunk, cache, q, c.scale)
    call.run()
    torch.cuda.synchronize()
    assert bool((call.out == 0).all()) and bool(torch.isneginf(call.lse).all())


@pytest.mark.parametrize("dtype,d", [(BF16, 64), (BF16, 128), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("lens", [[(1500, 1), (300, 1)], [(700, 60)], [(300, 3)], [(200, 1)] * 70], ids=str)
def test_infinite_values_that_every_token_sees(lens, dtype, d):
    """In tiles that nothing is taken out of: infinite times any weight is infinite."""
    S = lib()
    c = R.Case(lens, 8, 8, d, dtype, 16, seed=89)
    for b in range(c.B):
        for r, e, x in ((2, 1, math.inf), (40, 5, -math.inf), (130, 9, math.nan), (41, 1, math.inf),
                        (129, 20, math.inf), (131, 20, -math.inf)):
            p, i = c.slot(b, r)
            c.v[p, :, i, e] = x
    chunk, cache, q = c.to(DEV)
    log(f"[inf seen] {dtype} {d} {lens[:2]}")
    call = S.prepare_chunk_attn(chunk, cache, q, c.scale)
    call.run()
    torch.cuda.synchronize()
    want, wl, tol, ltol = R.attention(c)
    assert bool(torch.isposinf(want[..., 1]).all()) and bool(torch.isneginf(want[..., 5]).all())
    within(call.out, want, tol, "out")
    within(call.lse, wl, ltol, "lse")
