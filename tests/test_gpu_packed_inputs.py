"""A decode step over a packed ModelCache, prepared once and run again after each chunk: its inputs
brought up to date in place, against a step prepared anew."""
from __future__ import annotations

import pytest
import torch

import packed_ref as P
from parity import log
from test_gpu_packed_ops import NAMES, lib

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16 = torch.bfloat16


@pytest.mark.parametrize("positions", [False, True])
@pytest.mark.parametrize("fmt", [None, P.MXFP8, P.MXFP4], ids=lambda f: NAMES.get(f, "plain"))
def test_a_step_prepared_once_finds_later_rows(fmt, positions):
    from paper_2508_02751_amd import pipeline as L
    S = lib()
    log(f"[packed inputs] {fmt} {positions}")
    g = torch.Generator().manual_seed(7)
    B, n_cap, layers = 2, 128, 2
    caches = {}
    for m, (hq, hk, d, packed) in dict(s=(4, 2, 64, fmt), l=(8, 2, 128, None)).items():
        freq, amp = S.rope_freqs(d, 10000.0)
        caches[m] = L.ModelCache(B, layers, hq, hk, d, n_cap, S.RopeSpec(freq, S.ROPE_HALF, amp),
                                 positions=positions and m == "s", packed=packed)

    def fill(new):
        """The chunk through both models; the queries of each sequence's last token."""
        last = torch.tensor(new).cumsum(0) - 1
        got = []
        for c in caches.values():
            T, qs = c.begin(new), []
            for layer in range(layers):
                x = [torch.randn(T, h, c.head_dim, generator=g).to(DEV, BF16)
                     for h in (c.q_heads, c.kv_heads, c.kv_heads)]
                qs.append(c.layer(layer, *x)[1][last.to(DEV)])
            got.append(torch.stack(qs, 1))
        return got

    def lengths():
        return torch.tensor(caches["s"].tokens, dtype=torch.int32, device=DEV)
    s, hm = caches["s"], torch.randint(0, 8, (16,), generator=g).int().to(DEV)
    s_q, l_q = fill([60, 41])
    budget = dict(k_crit=torch.tensor([12, 9], dtype=torch.int32, device=DEV),
                  k_marg=torch.tensor([20, 15], dtype=torch.int32, device=DEV), kc_cap=12, km_cap=20)

    def step(x, s_q, l_q):
        return L.prepare_step(dict(x, s_q=s_q.clone(), l_q=l_q.clone(), l_k=caches["l"].k, l_v=caches["l"].v,
                                   n_cap=n_cap, head_map=hm, seq_len=lengths(), **budget))
    x = s.small_inputs()
    once = step(x, s_q, l_q)
    once.run()
    for new in ([1, 1], [3, 1], [1, 2]):
        begin = list(s.rows)
        s_q, l_q = fill(new)
        old = x["s_k"].clone()
        assert s.small_inputs(x, begin) is x
        torch.cuda.synchronize()
        if fmt is not None:  # the new rows only
            for b in range(B):
                assert torch.equal(x["s_k"][b, :, :, : begin[b]], old[b, :, :, : begin[b]])
                assert not torch.equal(x["s_k"][b, :, :, begin[b]: s.rows[b]], old[b, :, :, begin[b]: s.rows[b]])
        anew = s.small_inputs()
        assert set(anew) == set(x) and all(torch.equal(x[n], anew[n]) for n in x)
        once.with_query(s_q, l_q, lengths(), budget["k_crit"], budget["k_marg"])
        once.run()
        fresh = step(anew, s_q, l_q)
        fresh.run()
        torch.cuda.synchronize()
        for n in ("small_out", "large_out"):
            a, b = getattr(once.buf, n), getattr(fresh.buf, n)
            assert torch.equal(a, b), n
