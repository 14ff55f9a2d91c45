"""The cache operators together, as a prompt and its decode steps use them: both
models' caches filled in chunks, the small one compressed by the attention its rows
received, the next token appended, and the compensated decode step over what that
left, against plain forms in 64 bits and the oracle's step."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import cache_ref as R
from parity import compare_step, log, oracle_step

pytestmark = pytest.mark.gpu

DEV = "cuda"


def rotated(x, pos, freq, amp):
    return R.turned(x, pos.double()[:, None] * freq.cpu(), amp, x.shape[-1], False)[0]


class Plain:
    """A layer's keys and values per sequence in 64 bits, rounded where they are stored."""

    def __init__(self, batch, dtype):
        self.k, self.v, self.dtype = [[] for _ in range(batch)], [[] for _ in range(batch)], dtype

    def attend(self, b, q, scale):
        """q [new][Hq][d] of the sequence's last rows: output and weights [Hq][new][n]."""
        k, v = torch.cat(self.k[b]), torch.cat(self.v[b])  # [n][Hkv][d]
        n, new, g = k.shape[0], q.shape[0], q.shape[1] // k.shape[1]
        k, v = (t.repeat_interleave(g, 1).transpose(0, 1) for t in (k, v))
        x = torch.einsum("nhd,hrd->hnr", q, k) * scale
        seen = torch.arange(n)[None] <= (n - new + torch.arange(new))[:, None]
        p = torch.softmax(torch.where(seen, x, torch.tensor(-math.inf).double()), -1)
        return torch.einsum("hnr,hrd->nhd", p, v), p


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_prompt_compression_and_step(dtype):
    from paper_2508_02751_amd import pipeline as P
    from paper_2508_02751_amd import smallkv as S
    gen = torch.Generator().manual_seed(5)
    B, n_cap = 2, 192
    shapes = {"s": (2, 4, 2, 64), "l": (2, 8, 2, 128)}  # layers, Hq, Hkv, d
    half = R.HALF[dtype]
    caches, plain, scores = {}, {}, {}
    for m, (L, hq, hk, d) in shapes.items():
        freq, amp = S.rope_freqs(d, 10000.0, S.ROPE_BANDS, 4.0, 1.0, 4.0, 128)
        caches[m] = P.ModelCache(B, L, hq, hk, d, n_cap, S.RopeSpec(freq, S.ROPE_HALF, amp), dtype,
                                 DEV, keep_scores=m == "s")
        plain[m] = [Plain(B, dtype) for _ in range(L)]
        scores[m] = torch.zeros(B, L * hk, n_cap, dtype=torch.float64)

    def chunk(m, cache, new):
        """One chunk through every layer; the turned queries of each layer."""
        L, hq, hk, d = shapes[m]
        at = [t for t in cache.tokens]
        T = cache.begin(new)
        qs = []
        for layer in range(L):
            qkv = torch.randn(T, hq + 2 * hk, d, generator=gen).to(dtype)
            x = qkv.to(DEV)
            log(f"[pipeline] {m} layer {layer} {new}")
            out, q = cache.layer(layer, x[:, :hq], x[:, hq: hq + hk], x[:, hq + hk:])
            torch.cuda.synchronize()
            qs.append(q)
            if m == "s" and cache.row_pos is not None:
                continue  # (compressed: checked by the step below)
            i = 0
            for b, n in enumerate(new):
                pos = torch.arange(at[b], at[b] + n)
                rows = slice(i, i + n)
                i += n
                if n == 0:
                    continue
                pl = plain[m][layer]
                # the reference goes on from what the kernel stored: a rounding that
                # falls the other way there is no error here
                turned = rotated(qkv[rows, hq: hq + hk], pos, cache.rope.freq, cache.rope.amplitude)
                got = cache.k[b, layer, :, at[b]: at[b] + n].transpose(0, 1).cpu().double()
                assert bool(((got - turned).abs() <= 1.01 * half * turned.abs() + 2.0 ** -19).all())
                assert torch.equal(cache.v[b, layer, :, at[b]: at[b] + n].transpose(0, 1).cpu(), qkv[rows, hq + hk:])
                pl.k[b].append(got)
                pl.v[b].append(qkv[rows, hq + hk:].double())
                want, p = pl.attend(b, q[rows].cpu().double(), P.softmax_scale(d))
                # values of size up to 5: P's rounding and the output's in bf16, in fp32
                # logits of size 10 and sums over up to 200 rows
                tol = 5 * 2.02 * half if dtype == torch.bfloat16 else 2.0 ** -14
                assert float((out[rows].cpu().double() - want).abs().max()) <= tol
                if m == "s":
                    total = p.sum(1).view(hk, hq // hk, -1).sum(1)
                    scores[m][b, layer * hk: (layer + 1) * hk, : total.shape[1]] += total
        return qs

    for new in ([64, 50], [70, 0], [16, 47]):  # prompts of 150 and 97 tokens in three chunks
        for m in shapes:
            chunk(m, caches[m], new)
    small = caches["s"]
    for b, n in enumerate(small.rows):
        # every weight is right to about 2^-18 (logits and lse of size 10 in fp32)
        assert torch.allclose(small.scores[b, :, :n].cpu().double(), scores["s"][b, :, :n], rtol=2.0 ** -16)
    keep, recent, sinks = [60, 41], [8, 5], 2
    packed = small.compress(keep, recent, sinks, n_rows=64)
    torch.cuda.synchronize()
    L, hq, hk, d = shapes["s"]
    for b in range(B):
        assert packed.rows == keep and packed.tokens == [150, 97]
        for layer in range(L):
            for h in range(hk):
                f = small.scores[b, layer * hk + h].cpu()
                rows = R.kept_rows(f.tolist(), small.rows[b], keep[b], recent[b], sinks, 64)
                assert packed.row_pos[b, layer, h, : keep[b]].cpu().tolist() == rows
                assert torch.equal(packed.k[b, layer, h, : keep[b]], small.k[b, layer, h, rows])
                assert torch.equal(packed.v[b, layer, h, : keep[b]], small.v[b, layer, h, rows])
                assert torch.equal(packed.scores[b, layer * hk + h, : keep[b]].cpu(), f[rows])

    # the next token: appended to the compressed small cache and the full large one
    s_q, l_q = chunk("s", packed, [1, 1]), chunk("l", caches["l"], [1, 1])
    for b in range(B):
        assert packed.row_pos[b, :, :, keep[b]].cpu().eq([150, 97][b]).all()
    hm = torch.randint(0, 8, (16,), generator=gen).int()
    x = dict(packed.small_inputs(), s_q=torch.stack(s_q, 1), l_q=torch.stack(l_q, 1),
             l_k=caches["l"].k, l_v=caches["l"].v, n_cap=n_cap, head_map=hm.to(DEV),
             seq_len=torch.tensor([151, 98], dtype=torch.int32, device=DEV),
             k_crit=torch.tensor([20, 15], dtype=torch.int32, device=DEV),
             k_marg=torch.tensor([25, 30], dtype=torch.int32, device=DEV), kc_cap=20, km_cap=30)
    log(f"[pipeline] step {dtype}")
    ps = P.prepare_step(x)
    ps.run()
    torch.cuda.synchronize()
    e = compare_step(ps.buf, oracle_step(x, 0), x, dtype, "step over the compressed cache")
    log(f"[pipeline] {e}")
    # a second compression, from the compressed cache with its positions
    again = packed.compress([30, 30], [4, 4], 1)
    torch.cuda.synchronize()
    for b in range(B):
        for layer in range(L):
            for h in range(hk):
                f = packed.scores[b, layer * hk + h].cpu()
                rows = R.kept_rows(f.tolist(), packed.rows[b], 30, 4, 1, 30)
                pos = packed.row_pos[b, layer, h].cpu()[rows]
                assert torch.equal(again.row_pos[b, layer, h, :30].cpu(), pos)
                assert bool((pos[1:] > pos[:-1]).all())


def test_scores_start_the_accumulated_selection():
    """The decode step's running scores, started by the prompt: one layer of acc_score at
    a time, per query head, and the next step ranks by them."""
    from paper_2508_02751_amd import pipeline as P
    from paper_2508_02751_amd import smallkv as S
    from paper_2508_02751_amd import workloads as W
    w = W.Workload(190, "accum-prompt", 2, 300, "bf16", W.ModelShape(2, 8, 2, 64),
                   W.ModelShape(2, 8, 2, 128), ("pct", 8), ("pct", 15), ragged_min=200, select=2)
    x = W.make_step_inputs(w, DEV)
    ps = P.prepare_step(x)
    lens = [int(n) for n in x["seq_len"]]
    prompt = [n - 1 for n in lens]  # the last row is the step's own token
    gen = torch.Generator().manual_seed(3)
    start = torch.tensor([0, prompt[0], sum(prompt)], dtype=torch.int32, device=DEV)
    chunk = S.ChunkSpec(start, torch.tensor(prompt, dtype=torch.int32, device=DEV), sum(prompt),
                        max(prompt), w.n_cap)
    scale = P.softmax_scale(64)
    want = torch.zeros(2, 16, w.n_cap, dtype=torch.float64)
    for layer in range(2):
        q = torch.randn(sum(prompt), 8, 64, generator=gen).to(torch.bfloat16)
        cache = S.CacheSpec(x["s_k"][:, layer], x["s_v"][:, layer])
        log(f"[accum] layer {layer}")
        att = S.prepare_chunk_attn(chunk, cache, q.to(DEV), scale)
        att.run()
        S.prepare_chunk_scores(chunk, cache, q.to(DEV), att.lse, scale,
                               ps.buf.acc_score[:, 8 * layer: 8 * layer + 8]).run()
        torch.cuda.synchronize()
        for b, n in enumerate(prompt):
            k = x["s_k"][b, layer, :, :n].cpu().double().repeat_interleave(4, 0)
            rows = q[int(start[b]): int(start[b]) + n].double()
            s = torch.einsum("nhd,hrd->hnr", rows, k) * scale
            s = s.masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), -math.inf)
            want[b, 8 * layer: 8 * layer + 8, :n] = torch.softmax(s, -1).sum(1)
    got = ps.buf.acc_score.cpu().double()
    assert torch.allclose(got, want, rtol=2.0 ** -15, atol=1e-30)
    before = ps.buf.acc_score.clone()
    ps.run()
    torch.cuda.synchronize()
    for b, n in enumerate(lens):
        p = torch.exp(ps.buf.logits[b, :, :n].double() - ps.buf.row_max[b, :, None].double()) / \
            ps.buf.row_sum[b, :, None].double()
        grown = before[b, :, :n].double() + p
        assert torch.allclose(ps.buf.acc_score[b, :, :n].double(), grown, rtol=2.0 ** -18)
        acc = ps.buf.acc_score[b, :, :n].cpu().numpy()
        crit = ps.buf.crit_idx[b].cpu().numpy()
        for j in range(16):
            k = int(x["k_crit"][b])
            order = np.lexsort((np.arange(n), -acc[j].astype(np.float64)))[:k]
            assert sorted(order.tolist()) == crit[j][:k].tolist()


def test_no_new_tokens():
    """A chunk without tokens leaves a cache, its scores and its lengths as they were."""
    from paper_2508_02751_amd import pipeline as P
    from paper_2508_02751_amd import smallkv as S
    freq, amp = S.rope_freqs(64, 10000.0)
    c = P.ModelCache(2, 1, 4, 2, 64, 40, S.RopeSpec(freq, S.ROPE_HALF, amp), torch.bfloat16, DEV,
                     keep_scores=True)
    g = torch.Generator().manual_seed(3)

    def step(*new):
        T = c.begin(new)
        x = [torch.randn(T, h, 64, generator=g).to(DEV, torch.bfloat16) for h in (4, 2, 2)]
        return c.layer(0, *x)
    log("[pipeline] no new tokens")
    step(20, 9)
    before = c.k.clone(), c.v.clone(), c.scores.clone()
    out, q = step(0, 0)
    assert out.shape == (0, 4, 64) and q.shape == (0, 4, 64)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(before, (c.k, c.v, c.scores)))
    step(0, 1)
    torch.cuda.synchronize()
    assert c.rows == [20, 10] and torch.equal(c.scores[0], before[2][0])


def test_begin_refuses():
    from paper_2508_02751_amd import pipeline as P
    from paper_2508_02751_amd import smallkv as S
    freq, amp = S.rope_freqs(64, 10000.0)
    c = P.ModelCache(2, 1, 2, 1, 64, 8, S.RopeSpec(freq), device=DEV)
    for bad in ([1], [1, -1], [9, 0]):
        with pytest.raises(ValueError):
            c.begin(bad)
    with pytest.raises(ValueError):
        c.layer(0, None, None, None)
    with pytest.raises(ValueError):
        c.compress([1, 1])
