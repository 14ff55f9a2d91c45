"""What the cache operators refuse on the host, at the limits themselves (no GPU needed)."""
import ctypes as C

import pytest

from paper_2508_02751_amd import smallkv as S
from test_cache_abi import append, cache, chunk, queries, try_attn


@pytest.mark.parametrize("batch,heads", [(1 << 24, 1), (1 << 23, 2), (1, 1 << 24)])
def test_a_launch_counts_fewer_than_2_to_the_24_workgroups(batch, heads):
    """2^24 pairs of a sequence and a kv head, a workgroup of 256 threads each, are 2^32
    threads: refused, for a decode step's scores as for the others."""
    L, q = S.lib(), queries(n_heads=heads)
    ch, ca = chunk(batch=batch, n_tokens=0, max_new=1), cache(n_heads=heads)
    assert L.smallkv_chunk_scores(C.byref(ch), C.byref(ca), C.byref(q), heads, None, 0x1000, 128, 1 << 40,
                                  None) == S.EUNSUPPORTED
    assert try_attn(ch, ca, q) == S.EUNSUPPORTED
    a = append(n_q_heads=heads)
    assert L.smallkv_append(C.byref(ch), C.byref(ca), C.byref(a), None) == S.EUNSUPPORTED


def test_a_ramp_over_slow_pairs_only():
    """A length over which no pair turns `low` times: all of them are slow, the first too."""
    plain, _ = S.rope_freqs(64, 10000.0, device="cpu")
    f, _ = S.rope_freqs(64, 10000.0, S.ROPE_RAMP, 4.0, low=1.0, high=32.0, orig_len=1, device="cpu")
    assert (plain / f).tolist() == [4.0] * 32
    # and as few as none are slow where all turn `high` times
    f, _ = S.rope_freqs(64, 1.001, S.ROPE_RAMP, 4.0, low=1.0, high=32.0, orig_len=8192, device="cpu")
    plain, _ = S.rope_freqs(64, 1.001, device="cpu")
    assert (plain / f).tolist() == [1.0] * 32


def test_a_base_that_overflows_is_refused():
    with pytest.raises(S.SmallKVError) as e:
        S.rope_freqs(64, 1e200, S.ROPE_BASE, 1e150, device="cpu")
    assert e.value.status == S.EINVAL
