"""Appending to packed caches where a thread packs several items of a token, where the queries
turn in place in part, and where a finite key turns past what fp32 holds: codes and scales bit by
bit against the plain form in 64 bits."""
from __future__ import annotations

import math

import pytest
import torch

import cache_ref as R
import packed_ref as P
from parity import log
from test_gpu_packed_ops import NAMES, lib, run_append, same, within

pytestmark = pytest.mark.gpu

DEV = "cuda"
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


def append_many(c, rot, layout, far, in_place):
    """run_append for many tokens: the rows' places found at once."""
    S = lib()
    T, hk, d = c.T, c.hk, c.d
    k, v = (torch.randn(T, hk, d, generator=c.gen).to(c.dtype) for _ in range(2))
    seqs = torch.repeat_interleave(torch.arange(c.B), torch.tensor([new for _, new in c.lens]))
    rows = torch.cat([torch.arange(n - new, n) for n, new in c.lens])
    pos = (rows + far).int()
    freq = 10000.0 ** (-torch.arange(0, max(rot, 2), 2, dtype=torch.float64) / max(rot, 2))[: rot // 2]
    chunk, cache, q = c.to(DEV)
    want = [t.cpu().clone() for t in cache.tensors[:4]]
    call = S.prepare_append(chunk, cache, S.RopeSpec(freq.to(DEV), layout), q, k.to(DEV), v.to(DEV),
                            positions=pos.to(DEV), q_out=q if in_place else None)
    call.run()
    torch.cuda.synchronize()
    angle = pos.double()[:, None] * freq
    turned, size = R.turned(c.q, angle, 1.0, rot, layout == S.ROPE_INTERLEAVED)
    within(call.q_out, turned, R.HALF[c.dtype] * turned.abs() + 16 * R.U * size, "q_out")
    if in_place:
        assert call.q_out.data_ptr() == q.data_ptr()
    tk, _ = R.turned(k, angle, 1.0, rot, layout == S.ROPE_INTERLEAVED)
    page, at = (seqs, rows) if c.table is None else (c.table[seqs, rows // c.page].long(), rows % c.page)
    for x, codes, scales in ((tk, 0, 2), (v, 1, 3)):
        want[codes][page, :, at], want[scales][page, :, at] = P.pack(x, c.fmt)
    for t, w, what in zip(cache.tensors, want, ("k", "v", "k_scale", "v_scale")):
        same(t, w, what)


# sequences, hq, hk, d, dtype, page, rows_first, rot, layout, far, in place; the items of a token
# (8 elements of a head each)
MANY = [
    ([(700, 512), (300, 3)], 14, 2, 64, BF16, 16, False, 64, 0, 0, False),    # 144
    ([(600, 600)], 14, 2, 64, F32, 0, False, 32, 0, 5, True),
    ([(600, 513)], 28, 4, 128, BF16, 0, False, 128, 0, 1000003, True),        # 576
    ([(520, 520)], 28, 4, 128, F32, 64, True, 128, 1, 0, True),
    ([(530, 512), (1, 1)], 64, 8, 128, F32, 32, True, 96, 0, 0, True),        # 1280
    ([(530, 530)], 64, 8, 128, BF16, 16, False, 50, 0, 131072, True),
    ([(512, 512)], 64, 8, 128, BF16, 0, False, 96, 1, 0, False),
    ([(515, 515)], 64, 8, 128, F32, 128, False, 0, 0, 0, False),
    ([(515, 515)], 30, 6, 64, BF16, 8, False, 22, 0, 0, True),                # 336
    ([(900, 515)], 30, 6, 64, F32, 8, False, 48, 0, 17, True),
    ([(40, 1)] * 512, 32, 8, 64, BF16, 16, False, 64, 0, 0, True),            # 384
]


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("case", MANY, ids=[f"{i}" for i in range(len(MANY))])
def test_append_of_many_tokens(case, fmt):
    lens, hq, hk, d, dtype, page, rows_first, rot, layout, far, in_place = case
    log(f"[packed append] many {len(lens)} {case[1:]} {NAMES[fmt]}")
    append_many(P.Case(lens, hq, hk, d, dtype, fmt, page, rows_first, seed=13), rot, layout, far, in_place)


# fewer tokens, an item a thread: partial turns in place, tokens in several workgroups
FEW = [(14, 2, 64, BF16, 32, 0), (14, 2, 64, F32, 22, 0), (64, 8, 128, BF16, 96, 0), (64, 8, 128, F32, 50, 0),
       (64, 8, 128, BF16, 128, 0), (28, 4, 128, F32, 62, 1), (3, 1, 64, BF16, 0, 0)]


@pytest.mark.parametrize("fmt", FORMATS, ids=NAMES.get)
@pytest.mark.parametrize("case", FEW, ids=[str(c[:3] + c[4:]) for c in FEW])
def test_partial_turns_in_place(case, fmt):
    hq, hk, d, dtype, rot, layout = case
    log(f"[packed append] in place {case} {NAMES[fmt]}")
    append_many(P.Case([(90, 70), (33, 1)], hq, hk, d, dtype, fmt, 16, seed=14), rot, layout, 9, True)
