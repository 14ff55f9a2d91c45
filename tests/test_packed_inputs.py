"""ModelCache.small_inputs: what it hands out, and what it refuses to bring up to date (no GPU
needed)."""
import pytest
import torch

from paper_2508_02751_amd import pipeline as L
from paper_2508_02751_amd import smallkv as S


def cache(**kw):
    freq, amp = S.rope_freqs(64, 10000.0, device="cpu")
    return L.ModelCache(2, 3, 4, 2, 64, 40, S.RopeSpec(freq, S.ROPE_HALF, amp), device="cpu", **kw)


def test_a_plain_caches_inputs_are_its_own_and_held_is_brought_up_to_date():
    c = cache(positions=True)
    x = c.small_inputs()
    assert x["s_k"] is c.k and x["s_v"] is c.v and x["s_row_pos"] is c.row_pos
    c.rows = [5, 2]
    held = x["s_held"]
    y = c.small_inputs(dict(x, seq_len=None), begin=[0, 0])
    assert y["s_k"] is c.k and y["s_held"] is held and held.tolist() == [5, 2] and "seq_len" in y
    plain = cache()
    x = plain.small_inputs()
    assert plain.small_inputs(x) is x and set(x) == {"s_k", "s_v"}


def test_inputs_of_another_cache_are_refused():
    for kw in (dict(), dict(positions=True), dict(packed=S.MXFP8, positions=True)):
        a, b = cache(**kw), cache(**kw)
        k = torch.zeros(2, 3, 2, 40, 64, dtype=torch.bfloat16)
        x = {"s_k": k, "s_v": k.clone()} if kw.get("packed") is not None else b.small_inputs()
        if a.row_pos is not None:
            x.update(s_held=torch.zeros(2, dtype=torch.int32), s_row_pos=b.row_pos)
        before = {n: t.clone() for n, t in x.items()}
        with pytest.raises(ValueError, match="small_inputs"):
            a.small_inputs(x)
        assert all(torch.equal(x[n], t) for n, t in before.items())
        for bad in ({}, {"s_k": a.k}, dict(x, s_row_pos=a.row_pos) if a.row_pos is None else {"s_k": k, "s_v": k}):
            with pytest.raises(ValueError, match="small_inputs"):
                a.small_inputs(bad)
    c = cache(packed=S.MXFP4)
    k = torch.zeros(2, 3, 2, 39, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="out must be"):
        c.small_inputs({"s_k": k, "s_v": k})
    with pytest.raises(ValueError, match="on a GPU"):
        c.small_inputs()
