"""The packed cache's host side: what its calls refuse before touching the GPU, the binding's
checks, and the plain packing that the GPU tests compare with (no GPU needed)."""
import ctypes as C
import math

import pytest
import torch

import packed_ref as R
from paper_2508_02751_amd import pipeline as L
from paper_2508_02751_amd import smallkv as S
from test_cache_abi import P, append, cache, chunk, evict, queries


def packed(**over):
    c = S.Packed(P, P + (1 << 20), P + 4, P + 8, S.MXFP8, S.BF16, 128, 4, 16, 100, 8, 4 * 16 * 128, 16 * 128, 128,
                 4 * 16 * 4, 16 * 4, 4, P)
    for k, v in over.items():
        setattr(c, k, v)
    return c


def other(**over):
    return packed(**dict(dict(k=P + 4096, v=P + 8192, k_scale=P + 64, v_scale=P + 128), **over))


def calls(p):
    """The status of every call on the packed cache p, by name."""
    lib, n = S.lib(), C.c_size_t()
    got = {}
    hq = 28 if 28 % max(p.n_heads, 1) == 0 else max(p.n_heads, 1)
    ch, q, a, e = chunk(), queries(n_heads=hq), append(n_q_heads=hq), evict(n_score_heads=hq)
    got["size"] = lib.smallkv_chunk_attn_packed_workspace_size(C.byref(ch), C.byref(p), C.byref(q), C.byref(n))
    if got["size"]:  # (nothing is launched)
        got["attn"] = lib.smallkv_chunk_attn_packed(C.byref(ch), C.byref(p), C.byref(q), None, 0, None)
        got["scores"] = lib.smallkv_chunk_scores_packed(C.byref(ch), C.byref(p), C.byref(q), hq, None, P, 128,
                                                        1 << 40, None)
        got["append"] = lib.smallkv_append_packed(C.byref(ch), C.byref(p), C.byref(a), None)
        to = cache(k=P + (1 << 30), v=P + (1 << 31), n_heads=p.n_heads, head_dim=p.head_dim)
        if to.head_dim in (64, 128) and 0 < to.n_heads < 1 << 24:
            got["read"] = lib.smallkv_read_packed(C.byref(p), C.byref(to), 2, 128, None, P, None)
        same = dict(format=p.format, n_heads=p.n_heads, head_dim=p.head_dim, dtype=p.dtype)
        got["from"] = lib.smallkv_evict_packed_workspace_size(C.byref(e), C.byref(p), C.byref(other(**same)),
                                                              C.byref(n))
        got["evict"] = lib.smallkv_evict_packed(C.byref(e), C.byref(p), C.byref(other(**same)), P, 1 << 40, None)
    return got


BAD = [
    (dict(k=None), S.EINVAL), (dict(v=None), S.EINVAL), (dict(k_scale=None), S.EINVAL), (dict(v_scale=None), S.EINVAL),
    (dict(k=P + 8), S.EINVAL), (dict(v=P + 4), S.EINVAL), (dict(k_scale=P + 2), S.EINVAL),
    (dict(v_scale=P + 1, head_dim=64), S.EINVAL), (dict(format=2), S.EINVAL), (dict(format=-1), S.EINVAL),
    (dict(dtype=2), S.EINVAL), (dict(n_heads=0), S.EINVAL), (dict(page_rows=0), S.EINVAL),
    (dict(page_rows=24), S.EINVAL), (dict(n_pages=0), S.EINVAL), (dict(table_width=0), S.EINVAL),
    (dict(row_stride=-16), S.EINVAL), (dict(row_stride=136), S.EINVAL), (dict(head_stride=8), S.EINVAL),
    (dict(page_stride=24), S.EINVAL), (dict(scale_row_stride=2), S.EINVAL), (dict(scale_head_stride=-4), S.EINVAL),
    (dict(scale_page_stride=3), S.EINVAL), (dict(head_dim=96), S.EUNSUPPORTED), (dict(head_dim=256), S.EUNSUPPORTED),
    (dict(page_stride=1 << 40), S.EUNSUPPORTED), (dict(scale_page_stride=1 << 40), S.EUNSUPPORTED),
    (dict(page_rows=1 << 20, table_width=1 << 12), S.EUNSUPPORTED), (dict(n_heads=1 << 24), S.EUNSUPPORTED),
    (dict(page_table=None, table_width=0, n_pages=1), S.EINVAL),
]


@pytest.mark.parametrize("over,status", BAD, ids=[str(b[0]) for b in BAD])
def test_every_call_rejects_a_bad_cache(over, status):
    got = calls(packed(**over))
    if over.get("n_heads") == 1 << 24:
        got = {k: got[k] for k in ("size", "attn", "scores")}
    assert set(got.values()) == {status}, got


def test_good_caches():
    for over in (dict(), dict(format=S.MXFP4), dict(dtype=S.F32), dict(row_stride=0, scale_row_stride=0),
                 dict(head_dim=64, scale_row_stride=2, k_scale=P + 2), dict(page_table=None, table_width=0)):
        assert calls(packed(**over)) == {"size": S.OK}, over


def test_the_tokens_side_is_checked_as_on_a_plain_cache():
    lib, n = S.lib(), C.c_size_t()
    for ch, q, status in ((chunk(batch=0), queries(), S.EINVAL), (chunk(max_new=0), queries(), S.EINVAL),
                          (chunk(max_len=(1 << 30) + 1), queries(), S.EUNSUPPORTED),
                          (chunk(), queries(scale=0.0), S.EINVAL), (chunk(), queries(scale=math.nan), S.EINVAL),
                          (chunk(), queries(n_heads=27), S.EINVAL), (chunk(), queries(out=None), S.EINVAL),
                          (chunk(), queries(q=P + 4), S.EINVAL),
                          (chunk(batch=1 << 22, n_tokens=1 << 22, max_new=1), queries(), S.EUNSUPPORTED)):
        p = packed()
        assert lib.smallkv_chunk_attn_packed_workspace_size(C.byref(ch), C.byref(p), C.byref(q), C.byref(n)) == status
        assert lib.smallkv_chunk_attn_packed(C.byref(ch), C.byref(p), C.byref(q), None, 0, None) == status
    ch, p, q = chunk(max_len=20000, batch=2), packed(table_width=2000), queries()
    assert lib.smallkv_chunk_attn_packed_workspace_size(C.byref(ch), C.byref(p), C.byref(q), C.byref(n)) == S.OK
    assert n.value > 0
    assert lib.smallkv_chunk_attn_packed(C.byref(ch), C.byref(p), C.byref(q), P, n.value - 1, None) == S.EWORKSPACE
    assert lib.smallkv_chunk_attn_packed(C.byref(ch), C.byref(p), C.byref(q), P + 8, n.value, None) == S.EINVAL
    assert lib.smallkv_chunk_attn_packed_workspace_size(C.byref(ch), None, C.byref(q), C.byref(n)) == S.EINVAL
    assert lib.smallkv_chunk_attn_packed_workspace_size(None, C.byref(p), C.byref(q), C.byref(n)) == S.EINVAL
    assert lib.smallkv_chunk_attn_packed_workspace_size(C.byref(ch), C.byref(p), C.byref(q), None) == S.EINVAL
    for args, status in (((14, None, P, 20000, 1 << 40), S.EINVAL), ((28, None, None, 20000, 1 << 40), S.EINVAL),
                         ((28, None, P, 19999, 1 << 40), S.EINVAL), ((28, None, P, 20000, 28 * 20000 - 1), S.EINVAL)):
        assert lib.smallkv_chunk_scores_packed(C.byref(ch), C.byref(p), C.byref(q), *args, None) == status


def test_written_rows_do_not_share_memory():
    lib, n = S.lib(), C.c_size_t()
    ch, a, e = chunk(), append(), evict()
    for over in (dict(row_stride=0), dict(row_stride=112), dict(scale_row_stride=0), dict(head_stride=16),
                 dict(scale_head_stride=0), dict(page_stride=0), dict(scale_page_stride=0)):
        p = packed(**over)
        assert lib.smallkv_append_packed(C.byref(ch), C.byref(p), C.byref(a), None) == S.EINVAL, over
        t = other(**over)
        assert lib.smallkv_evict_packed_workspace_size(C.byref(e), C.byref(packed()), C.byref(t),
                                                       C.byref(n)) == S.EINVAL, over
    to = cache(k=P + (1 << 30), v=P + (1 << 31), row_stride=0)
    assert lib.smallkv_read_packed(C.byref(packed()), C.byref(to), 2, 128, None, P, None) == S.EINVAL
    # half the bytes are enough in 4 bits
    p = packed(format=S.MXFP4, row_stride=64)
    bad = append(q=None)
    assert lib.smallkv_append_packed(C.byref(ch), C.byref(p), C.byref(bad), None) == S.EINVAL


def test_read_and_evict_need_caches_that_fit():
    lib, n = S.lib(), C.c_size_t()
    p = packed()

    def read(to=None, batch=2, max_len=128, length=P, frm=p):
        to = to or cache(k=P + (1 << 30), v=P + (1 << 31))
        return lib.smallkv_read_packed(C.byref(frm), C.byref(to), batch, max_len, None, length, None)
    far = dict(k=P + (1 << 30), v=P + (1 << 31))
    for kw, status in ((dict(batch=0), S.EINVAL), (dict(max_len=0), S.EINVAL), (dict(length=None), S.EINVAL),
                       (dict(to=cache(**far, head_dim=64)), S.EINVAL), (dict(to=cache(**far, n_heads=2)), S.EINVAL),
                       (dict(to=cache(k=P, v=P + (1 << 31))), S.EINVAL), (dict(to=cache(**far, dtype=7)), S.EINVAL),
                       (dict(batch=1 << 20), S.EUNSUPPORTED), (dict(max_len=(1 << 30) + 1), S.EUNSUPPORTED)):
        assert read(**kw) == status, kw
    assert lib.smallkv_read_packed(None, C.byref(cache()), 2, 128, None, P, None) == S.EINVAL
    assert lib.smallkv_read_packed(C.byref(p), None, 2, 128, None, P, None) == S.EINVAL
    e = evict()

    def size(frm=p, to=None, e=e):
        return lib.smallkv_evict_packed_workspace_size(C.byref(e), C.byref(frm), C.byref(to or other()), C.byref(n))
    assert size() == S.OK and n.value == 2 * 4 * 64 * 4
    for to in (other(format=S.MXFP4), other(head_dim=64), other(n_heads=2), other(k=P), other(k_scale=P + 4),
               other(v_scale=P + 8)):
        assert size(to=to) == S.EINVAL
    assert size(e=evict(keep=None)) == S.EINVAL and size(e=evict(score_rows=127)) == S.EINVAL
    assert lib.smallkv_evict_packed(C.byref(e), C.byref(p), C.byref(other()), P, n.value - 1, None) == S.EWORKSPACE


# ---------------------------------------------------------------- binding --

def spec(fmt=S.MXFP8, d=64, **kw):
    return S.PackedSpec.empty(3, 2, 16, d, fmt, device="cpu", **kw)


def test_specs():
    for fmt, width in ((S.MXFP8, 64), (S.MXFP4, 32)):
        c = spec(fmt)
        assert c.head_dim == 64 and c.capacity == 16 and c.k.shape == (3, 2, 16, width)
        d = c.c(3, S.F32)
        assert (d.format, d.dtype, d.head_dim, d.row_stride, d.scale_row_stride) == (fmt, S.F32, 64, width, 2)
    t = torch.zeros(2, 4, dtype=torch.int32)
    assert spec(page_table=t).capacity == 64
    with pytest.raises(ValueError, match="page per sequence"):
        spec().c(4)
    with pytest.raises(ValueError, match="page_table"):
        spec(page_table=t).c(3)
    with pytest.raises(ValueError, match="MXFP8 or MXFP4"):
        spec(7)
    c = spec()
    for name, value, match in (("v", c.v[:, :, :15], "one shape"), ("k_scale", c.k_scale[..., :1], "scales a row"),
                               ("k", c.k.int(), "uint8"), ("format", 5, "format"),
                               ("v", torch.zeros(3, 2, 32, 64, dtype=torch.uint8)[:, :, ::2], "strides"),
                               ("v_scale", c.v_scale[0], "4-d")):
        bad = spec()
        setattr(bad, name, value)
        with pytest.raises(ValueError, match=match):
            bad.c(3)


def test_calls_need_matching_tensors():
    c = spec()
    ch = S.ChunkSpec(torch.tensor([0, 2], dtype=torch.int32), torch.tensor([2], dtype=torch.int32), 2, 2, 16)
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="on a GPU"):
        S.prepare_chunk_attn(ch, c, q, 0.1)
    with pytest.raises(ValueError, match="head_dim"):
        S.prepare_chunk_attn(ch, c, q[..., :32], 0.1)
    with pytest.raises(ValueError, match="dtype"):
        S.prepare_chunk_attn(ch, c, q.half(), 0.1)
    with pytest.raises(ValueError, match="k must be"):
        S.prepare_append(ch, c, S.RopeSpec(torch.zeros(32, dtype=torch.float64)), q, q[:, :2].float(), q[:, :2])
    plain = S.CacheSpec(torch.zeros(3, 2, 16, 64), torch.zeros(3, 2, 16, 64))
    one = torch.ones(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="both"):
        S.prepare_evict(c, plain, one, one, torch.zeros(1, 2, 16))
    with pytest.raises(ValueError, match="PackedSpec"):
        S.prepare_read(plain, plain, one)
    with pytest.raises(ValueError, match="length"):
        S.prepare_read(c, plain, one.long())
    with pytest.raises(ValueError, match="on a GPU"):
        S.prepare_read(c, plain, one)


def test_a_packed_model_cache_counts_rows_as_a_plain_one():
    freq, amp = S.rope_freqs(64, 10000.0, device="cpu")
    rope = S.RopeSpec(freq, S.ROPE_HALF, amp)
    c = L.ModelCache(2, 3, 4, 2, 64, 40, rope, device="cpu", packed=S.MXFP4)
    assert c.k.shape == (2, 3, 2, 40, 32) and c.k_scale.shape == (2, 3, 2, 40, 2) and c.n_rows == 40
    T = c.begin([20, 9])
    x = [torch.zeros(T, h, 64, dtype=torch.bfloat16) for h in (4, 2, 2)]
    with pytest.raises(ValueError, match="on a GPU"):
        c.layer(0, *x)
    with pytest.raises(ValueError, match="queries of"):
        c.layer(0, *(t.float() for t in x))
    assert c.rows == [0, 0]
    with pytest.raises(ValueError, match="keep_scores"):
        c.compress([1, 1])
    with pytest.raises(ValueError, match="MXFP8 or MXFP4"):
        L.ModelCache(2, 3, 4, 2, 64, 40, rope, device="cpu", packed=3)
    plain = L.ModelCache(2, 3, 4, 2, 64, 40, rope, device="cpu")
    with pytest.raises(ValueError, match="packed"):
        plain.read_back()


# ------------------------------------------------------- the plain packing --

@pytest.mark.parametrize("fmt", [R.MXFP8, R.MXFP4])
def test_packing_is_within_half_a_step(fmt):
    g = torch.Generator().manual_seed(1)
    x = torch.randn(300, 64, generator=g).double() * torch.exp(6 * torch.randn(300, 1, generator=g))
    codes, scales = R.pack(x, fmt)
    y = R.unpack(codes, scales, fmt)
    e = (scales.double() - 127).repeat_interleave(32, -1)
    least, bits = (-6, 3) if fmt == R.MXFP8 else (0, 1)
    binade = torch.floor(torch.log2(x.abs())).clamp_min(0.0 * e + least + e)
    assert ((x - y).abs() <= 2.0 ** (binade - bits - 1)).all()
    # packed again it stays: what a row stands for is its own nearest
    c2, s2 = R.pack(y, fmt)
    assert torch.equal(R.unpack(c2, s2, fmt), y)
    assert torch.equal(y, y.to(torch.bfloat16).double())


def test_code_values():
    assert R.code_values(R.MXFP4).tolist()[:8] == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    v = R.code_values(R.MXFP8)
    assert v[0x7E] == 448 and v[1] == 2.0 ** -9 and v[0x38] == 1 and v[0xB8] == -1 and math.isnan(v[0x7F])
