"""Appending to packed caches where a finite key turns past what fp32 holds: codes and scales bit by
bit against the plain form in 64 bits."""
from __future__ import annotations

import math

import pytest
import torch

import packed_ref as P
from parity import log
from test_gpu_packed_ops import NAMES, run_append

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
FORMATS = [P.MXFP8, P.MXFP4]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("rot,layout", [(64, 0), (32, 0), (22, 0), (64, 1)])
def test_finite_keys_that_turn_past_fp32_are_cut_to_the_largest_code(rot, layout, fmt, dtype):
    """Keys of 3e38 turn to up to sqrt(2) times that, 2.5 times with the amplitude: finite in 64
    bits, so their blocks are, at the largest scale.  Infinite ones stay NaN blocks."""
    log(f"[packed append] past fp32 {rot} {layout} {NAMES[fmt]} {dtype}")
    g = torch.Generator().manual_seed(17)
    T = 24
    x = torch.randn(T, 1, 64, generator=g) * 1e30
    sign = torch.where(torch.rand(T, 1, 64, generator=g) < 0.5, -1.0, 1.0)
    x[:16, :, :rot] = (sign * 3e38)[:16, :, :rot]
    x[8:16, :, 1:rot:3] = torch.randn(8, 1, len(range(1, rot, 3)), generator=g) * 1e36
    x[20, 0, 5] = math.inf
    x = x.to(dtype)
    assert torch.isfinite(x[:20]).all()
    for amp in (1.0, 2.5):
        c = P.Case([(T, T)], 1, 1, 64, dtype, fmt, 0, seed=2)
        run_append(c, rot, layout, far=3, amp=amp, new_k=x, new_v=x.flip(0))
