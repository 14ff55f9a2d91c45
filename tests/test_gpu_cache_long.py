"""The cache operators where a wave walks many tiles of keys: batches of long sequences,
with and without spans, whose copies and look-ups stay in flight from tile to tile.
Plain forms in 64 bits; values that tell every 32 rows of a sequence apart."""
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


class Long:
    """Caches of long sequences, made and gathered on the GPU.  absent: some pages of every
    sequence are outside the pool.  Rows that belong to nobody hold NaN."""

    def __init__(self, lens, hq, hk, d, dtype, page, absent=False, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.lens, self.hq, self.hk, self.d, self.dtype = lens, hq, hk, d, dtype
        self.rows = max(n for n, _ in lens)
        B, per = len(lens), page or self.rows
        width = (self.rows + per - 1) // per
        pages = B * width + (2 if page else 0)
        self.per, self.table = per, None
        if page:
            self.table = torch.randperm(pages, device=DEV, generator=g)[: B * width].view(B, width).int()
            if absent:  # every 23rd page, not the first
                self.table[:, 22::23] = torch.tensor(-1, device=DEV, dtype=torch.int32)
        self.k, self.v = (torch.full((pages, hk, per, d), math.nan, dtype=dtype, device=DEV) for _ in range(2))
        self.at, self.starts = [], [0]
        for b, (n, new) in enumerate(lens):
            r = torch.arange(n, device=DEV)
            p = r * 0 + b if self.table is None else self.table[b].long()[r // per]
            have = p >= 0
            self.at.append((p.clamp(min=0), r % per, have))
            for pool in (self.k, self.v):
                x = torch.randn(n, hk, d, device=DEV, generator=g).to(dtype)
                pool[p[have], :, (r % per)[have]] = x[have]
            self.starts.append(self.starts[-1] + new)
        self.T = self.starts[-1]
        self.q = torch.randn(self.T, hq, d, device=DEV, generator=g).to(dtype)
        self.scale = 1.0 / math.sqrt(d)
        self.gen = g

    def plant(self):
        """Element (r // 32) % d of row r's values is 100, the others 0: the outputs are the
        weights of blocks of 32 rows."""
        for p, i, have in self.at:
            r = torch.arange(p.numel(), device=DEV)[have]
            x = torch.zeros(r.numel(), self.hk, self.d, device=DEV)
            x[torch.arange(r.numel(), device=DEV), :, r // 32 % self.d] = 100.0
            self.v[p[have], :, i[have]] = x.to(self.dtype)

    def specs(self, max_len=None):
        S = lib()

        def ints(x):
            return torch.tensor(x, dtype=torch.int32, device=DEV)
        chunk = S.ChunkSpec(ints(self.starts), ints([n for n, _ in self.lens]), self.T,
                            max(new for _, new in self.lens), max_len or self.rows)
        return chunk, S.CacheSpec(self.k, self.v, self.table)

    def gather(self, pool, b):
        p, i, have = self.at[b]
        return torch.where(have[:, None, None], pool[p, :, i].double(), 0.0).transpose(0, 1).contiguous()

    def logits(self, b):
        """[hk][new][g][n] (-inf: not seen), and the bound on their error."""
        n, new = self.lens[b]
        g = self.hq // self.hk
        q = self.q[self.starts[b]: self.starts[b] + new].double().view(new, self.hk, g, self.d)
        q = q.transpose(0, 1).reshape(self.hk, new * g, self.d)
        k = self.gather(self.k, b).transpose(1, 2).contiguous()
        x = (torch.matmul(q, k) * self.scale).view(self.hk, new, g, n)
        size = (torch.matmul(q.abs(), k.abs()) * self.scale).view(self.hk, new, g, n)
        own = n - new + torch.arange(new, device=DEV)
        seen = (torch.arange(n, device=DEV)[None] <= own[:, None]) & self.at[b][2]
        x = torch.where(seen[:, None], x, -math.inf)
        return x, torch.where(seen[:, None], size, 0.0) * (self.d + 4) * R.U

    def flat(self, t):  # [hk][new][g]... -> [new][hq]...
        return t.transpose(0, 1).reshape(t.shape[1], self.hq, *t.shape[3:])


def ragged(batch, lo, hi, new):
    """Lengths spread over [lo, hi], new tokens 1..new (all of them in the first)."""
    return [(lo + (hi - lo) * (b * 37 % batch) // max(batch - 1, 1), new - b % new) for b in range(batch)]


# (name, sequences, hq, hk, d, dtype, page, absent, few rows)
CASES = [
    # spans of some 1700 rows, over ten tiles a wave
    ("token step", ragged(64, 1000, 4000, 1), 28, 4, 128, BF16, 16, False, True),
    ("token step, absent pages", ragged(64, 1000, 4000, 1), 28, 4, 128, BF16, 16, True, True),
    ("token step, dense", ragged(64, 1000, 4000, 1), 28, 4, 128, BF16, 0, False, True),
    ("token step d64", ragged(64, 1000, 4000, 1), 8, 4, 64, BF16, 32, True, True),
    ("token step d64, dense", ragged(64, 1000, 4000, 1), 28, 4, 64, BF16, 0, False, True),
    ("a few tokens each", ragged(48, 1000, 3001, 4), 32, 4, 128, BF16, 64, True, True),
    # no spans: a tile per sequence, and as many kv heads as fill the GPU
    ("tokens without spans", ragged(40, 600, 1500, 1), 16, 16, 128, BF16, 16, True, True),
    ("tokens without spans d64", ragged(64, 600, 1500, 3), 32, 16, 64, BF16, 0, False, True),
    ("fp32 token step", ragged(40, 1000, 2000, 1), 16, 8, 128, F32, 16, True, True),
    ("fp32 token step d64, dense", ragged(40, 1000, 2000, 1), 16, 8, 64, F32, 0, False, True),
    ("fp32 tokens without spans", ragged(40, 600, 1500, 1), 16, 16, 128, F32, 0, False, True),
    ("fp32 tiles without spans", ragged(40, 600, 1500, 5), 64, 16, 64, F32, 32, True, True),
    ("fp32 tiles in spans", ragged(6, 2000, 6000, 8), 24, 4, 128, F32, 32, True, True),
    # four waves that share tiles
    ("chunks without spans", ragged(34, 600, 1500, 40), 16, 16, 128, BF16, 16, True, False),
    ("chunks without spans d64", ragged(50, 600, 1500, 40), 16, 16, 64, BF16, 0, False, False),
    ("chunks in spans", ragged(6, 3000, 8001, 50), 28, 4, 128, BF16, 32, True, False),
    ("chunks in spans d64, dense", ragged(6, 3000, 8001, 150), 14, 2, 64, BF16, 0, False, False),
    ("fp32 chunks without spans", ragged(34, 600, 1100, 70), 16, 16, 64, F32, 16, True, False),
    ("fp32 chunks in spans", ragged(4, 2000, 3001, 40), 28, 4, 128, F32, 0, False, False),
]
IDS = [c[0].replace(" ", "-") for c in CASES]


@pytest.mark.parametrize("planted", [True, False])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_attention_over_many_tiles(case, planted):
    """Bounds: fp32 logits and sums (`rel`), the output's rounding, and of bf16 models the
    probabilities': 2^-16 relative in two parts (few rows), in one part 2^-8 sum w |v - o|
    and second order.  Of planted rows' weight that is 1.6% at most; a lost,
    repeated or stale tile is one block of 32 rows of the four or fewer that share an
    element."""
    S = lib()
    few, c = case[8], Long(*case[1:8], seed=len(case[0]))
    if planted:
        c.plant()
    chunk, cache = c.specs()
    log(f"[long attn] {case[0]} planted={planted}")
    call = S.prepare_chunk_attn(chunk, cache, c.q, c.scale)
    call.run()
    torch.cuda.synchronize()
    h = R.HALF[c.dtype]
    for b, (n, new) in enumerate(c.lens):
        x, dx = c.logits(b)
        v = c.gather(c.v, b)
        e = torch.logsumexp(x, -1)
        p = torch.exp(x - e[..., None])
        hk, g = c.hk, c.hq // c.hk
        o = torch.matmul(p.view(hk, new * g, n), v)
        a = torch.matmul(p.view(hk, new * g, n), v.abs())
        rel = (2 * dx.amax(-1) + 2 * (n + 64) * R.U).view(hk, new * g, 1)
        tol = a * rel + 1.01 * h * o.abs()
        if c.dtype == BF16 and few:
            tol += a * 2.0 ** -16
        elif c.dtype == BF16:
            away = torch.stack([(p.view(hk, new * g, n)[:, i, :, None] * (v - o[:, i, None]).abs()).sum(1)
                                for i in range(new * g)], 1)
            tol += 1.01 * h * away
        rows = slice(c.starts[b], c.starts[b] + new)
        shape = (hk, new, g, c.d)
        within(call.out[rows], c.flat(o.view(shape)).cpu(), c.flat(tol.view(shape)).cpu(), f"sequence {b}")
        within(call.lse[rows], c.flat(e).cpu(),
               c.flat(dx.amax(-1) + (n + 64) * R.U + 8 * R.U * e.abs() + 8 * R.U).cpu(), f"lse {b}")


SCORE_CASES = [(c, kv, None) for c in CASES[:12] if c[1][0][1] * c[2] // c[3] <= 32 for kv in (False, True)]
# capacities far above the lengths, and sequences far shorter than the others
SHORT = ("short among long", [(9000, 1), (5, 1), (700, 1), (129, 0), (128, 1), (1, 1)] * 12, 16, 4, 128, BF16, 32, True, True)
SCORE_CASES += [(SHORT, kv, cap) for kv in (False, True) for cap in (None, 200000)]


@pytest.mark.parametrize("case,per_kv,max_len", SCORE_CASES,
                         ids=[f"{c[0].replace(' ', '-')}-{kv}-{m}" for c, kv, m in SCORE_CASES])
def test_scores_over_many_blocks(case, per_kv, max_len):
    S = lib()
    c = Long(*case[1:8], seed=len(case[0]) + 1)
    if max_len:  # a table of that capacity
        c.table = torch.nn.functional.pad(c.table, (0, max_len // c.per - c.table.shape[1]), value=-1)
    chunk, cache = c.specs(max_len)
    heads, g = c.hk if per_kv else c.hq, c.hq // c.hk
    width = max_len or c.rows
    before = torch.rand(len(c.lens), heads, width, device=DEV, generator=c.gen)
    out = torch.full_like(before, 7.0)
    x = [c.logits(b) for b in range(len(c.lens))]
    lse = torch.cat([c.flat(torch.logsumexp(t, -1)) for t, _ in x]).float()
    log(f"[long scores] {case[0]} per_kv={per_kv} max_len={max_len}")
    S.prepare_chunk_scores(chunk, cache, c.q, lse, c.scale, out, before=before).run()
    torch.cuda.synchronize()
    for b, ((n, new), (t, dt)) in enumerate(zip(c.lens, x)):
        e = lse[c.starts[b]: c.starts[b] + new].double().view(new, c.hk, g).transpose(0, 1)[..., None]
        w = torch.where(torch.isinf(t), 0.0, torch.exp(t - e))
        arg = (torch.where(torch.isinf(t), 0.0, t).abs() + e.abs() + 1) * 4 * R.U
        tol = w * (dt + arg + 4 * R.U + (new * g + 64) * R.U)
        w, tol = w.sum(1), tol.sum(1)  # [hk][g][n]
        w, tol = (y.sum(1) if per_kv else y.reshape(heads, n) for y in (w, tol))
        w[:, : n - new] += before[b, :, : n - new].double()
        within(out[b, :, :n], w.cpu(), (tol + 2 * R.U * w).cpu(), f"sequence {b}")
        assert bool((out[b, :, n:] == 7).all())
