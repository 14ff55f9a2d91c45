"""pipeline.ModelCache's own bookkeeping (no GPU needed: a cache in host memory, whose
layers refuse to run)."""
import pytest
import torch

from paper_2508_02751_amd import pipeline as P
from paper_2508_02751_amd import smallkv as S


def cache(**kw):
    freq, amp = S.rope_freqs(64, 10000.0, device="cpu")
    return P.ModelCache(2, 3, 4, 2, 64, 40, S.RopeSpec(freq, S.ROPE_HALF, amp), device="cpu", **kw)


def tokens(c, T):
    return [torch.zeros(T, h, 64, dtype=torch.bfloat16) for h in (4, 2, 2)]


@pytest.mark.parametrize("keep_scores", [False, True])
def test_a_refused_layer_leaves_no_rows(keep_scores):
    c = cache(keep_scores=keep_scores)
    T = c.begin([20, 9])
    for layer in (0, -1, 2):
        with pytest.raises(ValueError, match="on a GPU"):
            c.layer(layer, *tokens(c, T))
        assert c.rows == [0, 0] and c.tokens == [0, 0]
    # the next chunk replaces it: 40 rows fit
    assert c.begin([40, 1]) == 41
    with pytest.raises(ValueError, match="must be"):
        c.layer(0, *tokens(c, 29))
    assert c.rows == [0, 0] and c.tokens == [0, 0]
    with pytest.raises(ValueError, match="do not fit"):
        c.begin([41, 0])


@pytest.mark.parametrize("layer", [3, -4, 100])
def test_layers_out_of_range(layer):
    c = cache(keep_scores=True)
    T = c.begin([1, 1])
    with pytest.raises(IndexError, match="layer"):
        c.layer(layer, *tokens(c, T))
