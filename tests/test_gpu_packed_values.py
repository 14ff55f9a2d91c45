"""Values at the edges of packed caches and of the queries over them, against the plain forms in 64
bits: NaN of every payload."""
from __future__ import annotations

import pytest
import torch

import cache_ref as R
import packed_ref as P
from parity import log
from test_gpu_packed_ops import NAMES, lib, within

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
