"""The cache operators' host side: what they refuse before touching the GPU, the
binding's checks of tensors, and the rotary frequencies (no GPU needed)."""
import ctypes as C
import math

import pytest
import torch

import cache_ref as R
from paper_2508_02751_amd import smallkv as S

P = 0x1000


def cache(**over):
    c = S.Cache(P, P, S.BF16, 128, 4, 16, 100, 8, 4 * 16 * 128, 16 * 128, 128, P)
    for k, v in over.items():
        setattr(c, k, v)
    return c


def dense(**over):
    return cache(**dict(dict(page_table=None, table_width=0, page_rows=37, n_pages=2), **over))


def chunk(**over):
    c = S.Chunk(2, 50, 40, 128, P, P)
    for k, v in over.items():
        setattr(c, k, v)
    return c


def queries(**over):
    q = S.Queries(28, 0.088, P, 28 * 128, 128, P, 28 * 128, 128, P)
    for k, v in over.items():
        setattr(q, k, v)
    return q


def append(**over):
    a = S.Append(P, P, P, 28 * 128, 128, 4 * 128, 128, 4 * 128, 128, 28, P + 4096, 28 * 128, 128,
                 None, P, 128, 0, 1.0, None, 0, 0)
    for k, v in over.items():
        setattr(a, k, v)
    return a


def evict(frm=None, to=None, **over):
    e = S.Evict(2, 128, P, P, None, 4, frm or cache(), to or cache(k=P + 4096, v=P + 8192), 28, P,
                128, None, 0, 64, None, P, P)
    for k, v in over.items():
        setattr(e, k, v)
    return e


def try_attn(ch, ca, q):
    n = C.c_size_t()
    rc = S.lib().smallkv_chunk_attn_workspace_size(C.byref(ch), C.byref(ca), C.byref(q), C.byref(n))
    if rc:  # (nothing is launched)
        assert S.lib().smallkv_chunk_attn(C.byref(ch), C.byref(ca), C.byref(q), None, 0, None) == rc
    return rc


BAD_CACHES = [
    (dict(k=None), S.EINVAL), (dict(v=None), S.EINVAL), (dict(k=P + 8), S.EINVAL),
    (dict(v=P + 2), S.EINVAL), (dict(dtype=2), S.EINVAL), (dict(n_heads=0), S.EINVAL),
    (dict(page_rows=0), S.EINVAL), (dict(page_rows=24), S.EINVAL), (dict(n_pages=0), S.EINVAL),
    (dict(table_width=0), S.EINVAL), (dict(row_stride=-8), S.EINVAL), (dict(row_stride=132), S.EINVAL),
    (dict(head_stride=4), S.EINVAL), (dict(page_stride=12), S.EINVAL), (dict(head_dim=96), S.EUNSUPPORTED),
    (dict(head_dim=256), S.EUNSUPPORTED), (dict(page_stride=1 << 40), S.EUNSUPPORTED),
    (dict(page_rows=1 << 20, table_width=1 << 12), S.EUNSUPPORTED),
    (dict(n_heads=1 << 24), S.EUNSUPPORTED),
]


@pytest.mark.parametrize("over,status", BAD_CACHES)
def test_every_call_rejects_a_bad_cache(over, status):
    hq = over.get("n_heads", 4) or 4
    assert try_attn(chunk(), cache(**over), queries(n_heads=hq)) == status
    q = queries(n_heads=hq)
    L = S.lib()
    assert L.smallkv_chunk_scores(C.byref(chunk()), C.byref(cache(**over)), C.byref(q), hq, None, P, 128,
                                  1 << 40, None) == status
    assert L.smallkv_append(C.byref(chunk()), C.byref(cache(**over)), C.byref(append()), None) == status
    n = C.c_size_t()
    for e in (evict(frm=cache(**over)), evict(to=cache(**dict(dict(k=P + 4096, v=P + 8192), **over)))):
        if over.get("n_heads") == 1 << 24:
            continue  # (and not the other cache's heads)
        assert L.smallkv_evict_workspace_size(C.byref(e), C.byref(n)) == status
        assert L.smallkv_evict(C.byref(e), P, 1 << 40, None) == status


@pytest.mark.parametrize("over,status", [
    (dict(batch=0), S.EINVAL), (dict(n_tokens=-1), S.EINVAL), (dict(max_new=0), S.EINVAL),
    (dict(max_len=0), S.EINVAL), (dict(start=None), S.EINVAL), (dict(len=None), S.EINVAL),
    (dict(max_len=(1 << 30) + 1), S.EUNSUPPORTED), (dict(max_new=1 << 28), S.EUNSUPPORTED),
])
def test_bad_chunks(over, status):
    assert try_attn(chunk(**over), cache(), queries()) == status
    ca, q = cache(), queries()
    assert S.lib().smallkv_chunk_scores(C.byref(chunk(**over)), C.byref(ca), C.byref(q), 28, None, P, 1 << 31,
                                        1 << 40, None) == status


@pytest.mark.parametrize("over,status", [
    (dict(q=None), S.EINVAL), (dict(q=P + 4), S.EINVAL), (dict(out=None), S.EINVAL),
    (dict(out=P + 8), S.EINVAL), (dict(n_heads=0), S.EINVAL), (dict(n_heads=27), S.EINVAL),
    (dict(scale=0.0), S.EINVAL), (dict(scale=-1.0), S.EINVAL), (dict(scale=math.inf), S.EINVAL),
    (dict(scale=math.nan), S.EINVAL), (dict(token_stride=-128), S.EINVAL),
    (dict(token_stride=3), S.EINVAL), (dict(head_stride=130), S.EINVAL),
    (dict(out_token_stride=4), S.EINVAL), (dict(out_token_stride=0), S.EINVAL),
    (dict(out_head_stride=0), S.EINVAL),
])
def test_bad_queries(over, status):
    assert try_attn(chunk(), cache(), queries(**over)) == status


def test_a_scale_stays_finite_in_log2_units():
    assert try_attn(chunk(), cache(), queries(scale=3e38)) == S.EINVAL
    assert try_attn(chunk(), cache(), queries(scale=1e37)) == S.OK


def test_a_dense_cache_has_a_page_per_sequence():
    assert try_attn(chunk(), dense(), queries()) == S.OK
    assert try_attn(chunk(), dense(n_pages=1), queries()) == S.EINVAL
    assert try_attn(chunk(batch=3), dense(), queries()) == S.EINVAL


def test_launches_stay_below_their_limits():
    """Calls whose workgroups a launch cannot count are refused on the host."""
    L = S.lib()
    n = C.c_size_t()
    big = dict(batch=1 << 22, n_tokens=1 << 22, max_new=1)
    assert try_attn(chunk(**big), cache(), queries()) == S.EUNSUPPORTED
    assert try_attn(chunk(**dict(big, batch=(1 << 22) - 1)), cache(), queries()) == S.OK
    many = chunk(batch=1, n_tokens=1 << 30, max_new=1 << 24)  # 7 query heads a kv head
    assert try_attn(many, cache(), queries()) == S.OK         # 2^24 * 7 / 128 tiles * 4
    assert try_attn(chunk(batch=8, n_tokens=1 << 27, max_new=1 << 24), cache(), queries()) == S.EUNSUPPORTED
    ca, q = cache(table_width=1 << 20), queries()
    ch = chunk(batch=1 << 10, max_len=1 << 24)
    assert L.smallkv_chunk_scores(C.byref(ch), C.byref(ca), C.byref(q), 28, None, P, 1 << 24, 1 << 40,
                                  None) == S.EUNSUPPORTED
    ch, a = chunk(n_tokens=1 << 24), append()
    assert L.smallkv_append(C.byref(ch), C.byref(cache()), C.byref(a), None) == S.EUNSUPPORTED
    e = evict(batch=1 << 20)
    assert L.smallkv_evict_workspace_size(C.byref(e), C.byref(n)) == S.EUNSUPPORTED
    e = evict(batch=(1 << 20) - 1)
    assert L.smallkv_evict_workspace_size(C.byref(e), C.byref(n)) == S.OK


def test_attention_needs_its_workspace():
    n = C.c_size_t()
    ch, ca, q = chunk(batch=1, n_tokens=1, max_new=1, max_len=100000), cache(table_width=6250), queries()
    L = S.lib()
    assert L.smallkv_chunk_attn_workspace_size(C.byref(ch), C.byref(ca), C.byref(q), C.byref(n)) == S.OK
    assert n.value > 0
    args = (C.byref(ch), C.byref(ca), C.byref(q))
    assert L.smallkv_chunk_attn(*args, None, n.value, None) == S.EWORKSPACE
    assert L.smallkv_chunk_attn(*args, P, n.value - 1, None) == S.EWORKSPACE
    assert L.smallkv_chunk_attn(*args, P + 4, n.value, None) == S.EINVAL
    assert L.smallkv_chunk_attn_workspace_size(*args, None) == S.EINVAL


def test_no_tokens_is_no_work():
    ch, ca, q, a = chunk(n_tokens=0), cache(), queries(), append()
    L = S.lib()
    n = C.c_size_t()
    assert L.smallkv_chunk_attn_workspace_size(C.byref(ch), C.byref(ca), C.byref(q), C.byref(n)) == S.OK
    assert L.smallkv_chunk_attn(C.byref(ch), C.byref(ca), C.byref(q), P, n.value, None) == S.OK
    assert L.smallkv_append(C.byref(ch), C.byref(ca), C.byref(a), None) == S.OK
    # and no operands of the tokens
    q, a = queries(q=None, out=None, lse=None), append(q=None, k=None, v=None, q_out=None)
    assert L.smallkv_chunk_attn_workspace_size(C.byref(ch), C.byref(ca), C.byref(q), C.byref(n)) == S.OK
    assert L.smallkv_chunk_attn(C.byref(ch), C.byref(ca), C.byref(q), P, n.value, None) == S.OK
    assert L.smallkv_append(C.byref(ch), C.byref(ca), C.byref(a), None) == S.OK


def test_scores_refusals():
    L = S.lib()
    ch, ca = chunk(), cache()

    def call(q, heads=28, out=P, rows=128, seq=28 * 128):
        return L.smallkv_chunk_scores(C.byref(ch), C.byref(ca), C.byref(q), heads, None, out, rows, seq,
                                      None)
    assert call(queries(lse=None)) == S.EINVAL
    assert call(queries(), out=None) == S.EINVAL
    assert call(queries(), rows=127) == S.EINVAL
    assert call(queries(), seq=28 * 128 - 1) == S.EINVAL
    assert call(queries(token_stride=1 << 31)) == S.EUNSUPPORTED
    assert call(queries(), heads=14) == S.EINVAL
    assert call(queries(n_heads=27), heads=27) == S.EINVAL
    assert call(queries(scale=0.0)) == S.EINVAL


@pytest.mark.parametrize("over,status", [
    (dict(q=None), S.EINVAL), (dict(k=None), S.EINVAL), (dict(v=None), S.EINVAL),
    (dict(q_out=None), S.EINVAL), (dict(k=P + 2), S.EINVAL), (dict(q_out=P + 8), S.EINVAL),
    (dict(v_token_stride=129), S.EINVAL), (dict(k_head_stride=-128), S.EINVAL),
    (dict(q_out_token_stride=0), S.EINVAL), (dict(q_out_head_stride=0), S.EINVAL),
    (dict(n_q_heads=0), S.EINVAL), (dict(n_q_heads=30), S.EINVAL), (dict(rot_dim=-2), S.EINVAL),
    (dict(rot_dim=31), S.EINVAL), (dict(rot_dim=130), S.EINVAL), (dict(freq=None), S.EINVAL),
    (dict(layout=2), S.EINVAL), (dict(amplitude=math.nan), S.EINVAL),
    (dict(row_pos=P, pos_rows=0), S.EINVAL), (dict(row_pos=P, pos_rows=9, pos_seq_stride=35), S.EINVAL),
    (dict(q_out=P, q_out_token_stride=128, q_out_head_stride=50 * 128), S.EINVAL),  # in place, other strides
])
def test_append_refusals(over, status):
    ch, ca, a = chunk(), cache(), append(**over)
    assert S.lib().smallkv_append(C.byref(ch), C.byref(ca), C.byref(a), None) == status


@pytest.mark.parametrize("over", [dict(row_stride=0), dict(head_stride=0), dict(page_stride=0)])
def test_broadcast_caches_are_read_but_not_written(over):
    ch, ca, a = chunk(), cache(**over), append()
    assert S.lib().smallkv_append(C.byref(ch), C.byref(ca), C.byref(a), None) == S.EINVAL
    assert try_attn(ch, ca, queries()) == S.OK
    n = C.c_size_t()
    to = cache(**dict(over, k=P + 4096, v=P + 8192))
    assert S.lib().smallkv_evict_workspace_size(C.byref(evict(to=to)), C.byref(n)) == S.EINVAL


@pytest.mark.parametrize("over,status", [
    (dict(batch=0), S.EINVAL), (dict(max_len=0), S.EINVAL), (dict(sinks=-1), S.EINVAL),
    (dict(out_rows=0), S.EINVAL), (dict(len=None), S.EINVAL), (dict(keep=None), S.EINVAL),
    (dict(scores=None), S.EINVAL), (dict(out_pos=None), S.EINVAL), (dict(held=None), S.EINVAL),
    (dict(n_score_heads=0), S.EINVAL), (dict(n_score_heads=30), S.EINVAL),
    (dict(score_rows=127), S.EINVAL), (dict(row_pos=2 * P, pos_rows=127), S.EINVAL),
    (dict(row_pos=P, pos_rows=128), S.EINVAL),            # its own output
    (dict(out_scores=P), S.EINVAL),
    (dict(to=cache()), S.EINVAL),                          # the same cache
    (dict(to=cache(k=P + 4096, v=P + 8192, head_dim=64)), S.EINVAL),
    (dict(to=cache(k=P + 4096, v=P + 8192, dtype=S.F32)), S.EINVAL),
    (dict(to=cache(k=P + 4096, v=P + 8192, n_heads=2)), S.EINVAL),
    (dict(n_score_heads=4 * 65), S.EUNSUPPORTED),
    (dict(max_len=(1 << 20) + 1, score_rows=1 << 21), S.EUNSUPPORTED),
])
def test_evict_refusals(over, status):
    n = C.c_size_t()
    e = evict(**over)
    assert S.lib().smallkv_evict_workspace_size(C.byref(e), C.byref(n)) == status
    assert S.lib().smallkv_evict(C.byref(e), P, 1 << 40, None) == status


def test_evict_needs_its_workspace():
    n = C.c_size_t()
    e = evict()
    L = S.lib()
    assert L.smallkv_evict_workspace_size(C.byref(e), C.byref(n)) == S.OK and n.value > 0
    assert L.smallkv_evict(C.byref(e), None, 0, None) == S.EWORKSPACE
    assert L.smallkv_evict(C.byref(e), P, n.value - 1, None) == S.EWORKSPACE
    assert L.smallkv_evict(C.byref(e), P + 4, n.value, None) == S.EINVAL
    assert L.smallkv_evict_workspace_size(C.byref(e), None) == S.EINVAL
    assert L.smallkv_evict(None, P, n.value, None) == S.EINVAL


# ------------------------------------------------------------- frequencies --

def test_rope_freqs():
    f, amp = S.rope_freqs(8, 10000.0, device="cpu")
    assert amp == 1.0 and torch.allclose(f, torch.tensor([1.0, 0.1, 0.01, 0.001]).double(), rtol=1e-15)
    f, _ = S.rope_freqs(8, 10000.0, S.ROPE_LINEAR, 4.0, device="cpu")
    assert torch.allclose(f, torch.tensor([0.25, 0.025, 0.0025, 0.00025]).double(), rtol=1e-15)
    f, amp = S.rope_freqs(64, 10000.0, S.ROPE_BASE, 8.0, device="cpu")
    # the slowest pair is slowed by the factor itself, the fastest not at all
    assert f[0] == 1.0 and amp == 1.0
    assert math.isclose(f[31], 10000.0 ** (-62 / 64) / 8.0, rel_tol=1e-12)
    f, amp = S.rope_freqs(128, 500000.0, S.ROPE_RAMP, 16.0, low=1.0, high=32.0, orig_len=8192, device="cpu")
    plain, _ = S.rope_freqs(128, 500000.0, device="cpu")
    assert math.isclose(amp, 0.1 * math.log(16.0) + 1.0, rel_tol=1e-7)
    turns = 8192 * plain / (2 * math.pi)
    ratio = plain / f
    assert bool((ratio[turns > 40] == 1).all())
    assert torch.allclose(ratio[turns < 0.8], torch.tensor(16.0).double(), rtol=1e-12)
    assert bool((ratio[1:] >= ratio[:-1] - 1e-12).all())
    f, amp = S.rope_freqs(128, 500000.0, S.ROPE_BANDS, 8.0, low=1.0, high=4.0, orig_len=8192, device="cpu")
    share = ((turns - 1) / 3).clamp(0, 1)
    assert amp == 1.0 and torch.allclose(f, plain / 8 * (1 - share) + plain * share, rtol=1e-13)
    f, _ = S.rope_freqs(2, 10000.0, S.ROPE_BASE, 8.0, device="cpu")
    assert f.tolist() == [1.0]


@pytest.mark.parametrize("args", [
    (0, 1e4), (7, 1e4), (-2, 1e4), (8, 1.0), (8, math.nan), (8, math.inf), (8, 1e4, 5), (8, 1e4, -1),
    (8, 1e4, S.ROPE_LINEAR, 0.5), (8, 1e4, S.ROPE_LINEAR, math.nan), (8, 1e4, S.ROPE_RAMP, 4.0, 0.0, 32.0, 4096),
    (8, 1e4, S.ROPE_RAMP, 4.0, 2.0, 1.0, 4096), (8, 1e4, S.ROPE_BANDS, 4.0, 1.0, 32.0, 0),
    (8, 1e4, S.ROPE_BANDS, 4.0, 1.0, math.inf, 4096),
])
def test_rope_freqs_refusals(args):
    with pytest.raises(S.SmallKVError) as e:
        S.rope_freqs(*args, device="cpu")
    assert e.value.status == S.EINVAL


# ------------------------------------------------- the binding's own checks --

def specs(**kw):
    c = R.Case([(20, 4), (7, 7)], 8, 2, 64, torch.bfloat16, 8, **kw)
    chunk, cache, q = c.to("cpu")
    return c, chunk, cache, q


def refuses(match, f, *args, **kw):
    with pytest.raises(ValueError, match=match):
        f(*args, **kw)


def test_binding_checks_attention():
    c, ch, ca, q = specs()
    f = S.prepare_chunk_attn
    refuses("on a GPU", f, ch, ca, q, 0.1, out=torch.empty_like(q), lse=False)
    refuses("q must be", f, ch, ca, q[:-1], 0.1)
    refuses("q must be", f, ch, ca, q.float(), 0.1)
    refuses("q must be", f, ch, ca, q[..., :32], 0.1)
    refuses("last dimension", f, ch, ca, torch.empty(11, 64, 8, dtype=torch.bfloat16).transpose(1, 2), 0.1)
    refuses("out must be", f, ch, ca, q, 0.1, out=q[:, :4])
    refuses("lse must be", f, ch, ca, q, 0.1, lse=torch.empty(11, 7))
    refuses("lse must be", f, ch, ca, q, 0.1, lse=torch.empty(11, 8, dtype=torch.bfloat16))
    refuses("length", f, S.ChunkSpec(ch.start, ch.length.long(), 11, 7, 20), ca, q, 0.1)
    refuses("start", f, S.ChunkSpec(ch.start[:-1], ch.length, 11, 7, 20), ca, q, 0.1)
    refuses("4-d", f, ch, S.CacheSpec(ca.k, ca.v[:-1], ca.page_table), q, 0.1)
    refuses("page_table", f, ch, S.CacheSpec(ca.k, ca.v, ca.page_table[:1]), q, 0.1)
    refuses("page_table", f, ch, S.CacheSpec(ca.k, ca.v, ca.page_table.long()), q, 0.1)
    refuses("page per sequence", f, ch, S.CacheSpec(ca.k[:1], ca.v[:1]), q, 0.1)
    strided = ca.v.transpose(1, 2).contiguous().transpose(1, 2)
    refuses("same strides", f, ch, S.CacheSpec(ca.k, strided, ca.page_table), q, 0.1)
    refuses("unsupported dtype", f, ch, S.CacheSpec(ca.k.half(), ca.v.half(), ca.page_table), q.half(), 0.1)


def test_binding_checks_scores_append_and_evict():
    c, ch, ca, q = specs()
    lse = torch.zeros(11, 8)
    out = torch.zeros(2, 8, 24)
    refuses("on a GPU", S.prepare_chunk_scores, ch, ca, q, lse, 0.1, out)
    refuses("lse must be", S.prepare_chunk_scores, ch, ca, q, lse[:-1], 0.1, out)
    refuses("out must be", S.prepare_chunk_scores, ch, ca, q, lse, 0.1, out[:1])
    refuses("before must be", S.prepare_chunk_scores, ch, ca, q, lse, 0.1, out, before=out[:, :2])
    refuses("out's strides", S.prepare_chunk_scores, ch, ca, q, lse, 0.1, out,
            before=torch.zeros(2, 16, 24)[:, :8])
    refuses("contiguous", S.prepare_chunk_scores, ch, ca, q, lse, 0.1, out.transpose(1, 2)[:, :8, :8])
    refuses("overlap", S.prepare_chunk_scores, ch, ca, q, lse, 0.1, out[:1].expand(2, 8, 24))
    rope = S.RopeSpec(torch.zeros(32, dtype=torch.float64))
    kv = torch.zeros(11, 2, 64, dtype=torch.bfloat16)
    refuses("on a GPU", S.prepare_append, ch, ca, rope, q, kv, kv)
    refuses("k must be", S.prepare_append, ch, ca, rope, q, kv[:, :1], kv)
    refuses("v must be", S.prepare_append, ch, ca, rope, q, kv, kv.float())
    refuses("positions must be", S.prepare_append, ch, ca, rope, q, kv, kv, positions=torch.zeros(11))
    refuses("freq must be", S.prepare_append, ch, ca, S.RopeSpec(torch.zeros(32)), q, kv, kv)
    refuses("row_pos must be", S.prepare_append, ch, ca, rope, q, kv, kv,
            row_pos=torch.zeros(2, 3, 9, dtype=torch.int32))
    n = torch.tensor([20, 7], dtype=torch.int32)
    sc = torch.zeros(2, 4, 24)
    to = S.CacheSpec(torch.zeros(2, 2, 9, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 9, 64, dtype=torch.bfloat16))
    refuses("on a GPU", S.prepare_evict, ca, to, n, n, sc)
    refuses("keep must be", S.prepare_evict, ca, to, n, n[:1], sc)
    refuses("scores must be", S.prepare_evict, ca, to, n, n, sc[:, :3])
    refuses("recent must be", S.prepare_evict, ca, to, n, n, sc, recent=n.long())
    refuses("row_pos must be", S.prepare_evict, ca, to, n, n, sc, row_pos=torch.zeros(2, 4, 24, dtype=torch.int32))
