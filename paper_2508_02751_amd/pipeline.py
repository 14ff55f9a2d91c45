"""Wiring of one decode step's tensors to the C ABI (marshalling only).

`prepare_step` turns the dict produced by workloads.make_step_inputs (or any
dict with the same keys) into BatchSpec/ModelSpec objects, allocates the
caller-owned intermediates and the workspace, and builds the C step
descriptor; `run` enqueues smallkv_step on the current stream.

`ModelCache` holds the caches that a step reads: a prompt's chunks and decoded
tokens fill them layer by layer (smallkv_append, smallkv_chunk_attn), the
attention they spend is kept per cached row (smallkv_chunk_scores), and
`compress` keeps the rows that received most of it (smallkv_evict).
"""
from __future__ import annotations

import dataclasses
import math
from typing import Optional, Sequence

import torch

from . import smallkv as S


MATCH_MIN, MATCH_MAX = 100, 200  # prompt tokens the matching uses ("Method Details")


def match_window(prompt_len: int) -> Optional[int]:
    """Window of the prefill matching for a prompt: None (delay the matching
    until the context reaches MATCH_MIN tokens) below MATCH_MIN, else the
    first min(prompt_len, MATCH_MAX) tokens (a longer prompt is truncated)."""
    if prompt_len < MATCH_MIN:
        return None
    return min(prompt_len, MATCH_MAX)


def prepare_match(x: dict, scores: bool = True, top_bits: bool = True) -> S.MatchCall:
    """smallkv_match over the window operands produced by workloads.match_inputs."""
    return S.prepare_match(x["win_len"], x["top_k"], x["l_q"], x["l_k"],
                           softmax_scale(x["l_q"].shape[-1]), x["s_q"], x["s_k"],
                           softmax_scale(x["s_q"].shape[-1]), scores, top_bits)


def softmax_scale(head_dim: int) -> float:
    return float(torch.tensor(1.0 / math.sqrt(head_dim), dtype=torch.float32))


@dataclasses.dataclass
class PreparedStep:
    batch: S.BatchSpec
    small: S.ModelSpec
    large: S.ModelSpec
    head_map: torch.Tensor
    mode: int
    buf: S.StepBuffers
    desc: S.Step
    inputs: dict

    def run(self, stream=None):
        S.smallkv_step(self.desc, self.buf.ws, stream)

    def with_query(self, s_q: torch.Tensor, l_q: torch.Tensor, seq_len=None, k_crit=None,
                   k_marg=None, k_recent=None):
        """Point the descriptor at new queries/lengths (same shapes; for multi-step runs)."""
        self.small.q.copy_(s_q)
        self.large.q.copy_(l_q)
        if seq_len is not None:
            self.batch.seq_len.copy_(seq_len)
            self.batch.k_crit.copy_(k_crit)
            self.batch.k_marg.copy_(k_marg)
        if k_recent is not None:
            self.batch.k_recent.copy_(k_recent)


def prepare_step(x: dict, mode: int = S.NORM_REMAINING,
                 k_slot: Optional[torch.Tensor] = None,
                 v_slot: Optional[torch.Tensor] = None,
                 l_k: Optional[torch.Tensor] = None,
                 l_v: Optional[torch.Tensor] = None,
                 select: Optional[int] = None) -> PreparedStep:
    """`select` defaults to x["select"] when present, else per-head selection."""
    if select is None:
        select = x.get("select", S.SELECT_HEAD)
    s_q, s_k, s_v = x["s_q"], x["s_k"], x["s_v"]
    l_q = x["l_q"]
    l_k = x["l_k"] if l_k is None else l_k
    l_v = x["l_v"] if l_v is None else l_v
    n_cap = x["n_cap"] if "n_cap" in x else s_k.shape[3]
    kr = x.get("k_recent")
    batch = S.BatchSpec(x["seq_len"].contiguous(), x["k_crit"].contiguous(),
                        x["k_marg"].contiguous(), n_cap, int(x["kc_cap"]), int(x["km_cap"]),
                        kr.contiguous() if kr is not None else None)
    small = S.ModelSpec(s_q.contiguous(), s_k, s_v, torch.empty_like(s_q),
                        softmax_scale(s_q.shape[-1]), held=x.get("s_held"),
                        row_pos=x.get("s_row_pos"))
    large = S.ModelSpec(l_q.contiguous(), l_k, l_v, torch.empty_like(l_q),
                        softmax_scale(l_q.shape[-1]), k_slot, v_slot)
    hm = x["head_map"].contiguous()
    ws_bytes = S.smallkv_workspace_size(batch, small, large, hm, select)
    buf = S.alloc_step_buffers(batch, s_q, l_q, ws_bytes, select, l_k.shape[2])
    buf.small_out = small.out
    buf.large_out = large.out
    # accumulated scores: the running state, zero before the first step
    acc = (torch.zeros((batch.seq_len.numel(), buf.logits.shape[1], n_cap), dtype=torch.float32,
                       device=s_q.device) if select == S.SELECT_ACCUM else None)
    buf.acc_score = acc
    desc = S.make_step(batch, small, large, hm, mode, buf.logits, buf.row_max, buf.row_sum,
                       buf.crit_idx, buf.marg_idx, buf.marg_prob, buf.mass, select, acc)
    return PreparedStep(batch, small, large, hm, mode, buf, desc, x)


class ModelCache:
    """One model's keys and values [B][layers][Hkv][n_rows][d], filled a chunk of new
    tokens at a time:

        cache.begin([new tokens of each sequence])
        for layer in range(layers):
            out, turned_q = cache.layer(layer, q, k, v)   # packed [T][heads][d]

    rows[b]: rows in use; tokens[b]: the sequence's length (more than its rows once
    the cache is compressed: row_pos [B][layers][Hkv][n_rows] then names the rows'
    positions).  Both count a chunk from the first layer that has taken it: a chunk
    whose first layer() raised is not part of the cache, and the next begin() replaces
    it.  With keep_scores, scores [B][layers * Hkv][n_rows] sum the
    attention each row has received, over queries and the query heads of a kv head.
    packed (smallkv.MXFP8 or MXFP4): k and v hold the rows' codes, k_scale and v_scale their
    blocks' scales (see smallkv.PackedSpec); read_back gives the rows as the step takes them,
    and small_inputs a copy of them, to be brought up to date after later chunks; everything
    else is the same.
    Everything runs on the current stream.
    """

    def __init__(self, batch: int, layers: int, q_heads: int, kv_heads: int, head_dim: int,
                 n_rows: int, rope: S.RopeSpec, dtype=torch.bfloat16, device="cuda",
                 keep_scores: bool = False, positions: bool = False, packed: Optional[int] = None):
        def new(*shape, dt=dtype):
            return torch.zeros(shape, dtype=dt, device=device)
        self.layers, self.q_heads, self.kv_heads, self.rope = layers, q_heads, kv_heads, rope
        self.head_dim, self.dtype, self.packed = head_dim, dtype, packed
        rows = (batch, layers, kv_heads, n_rows)
        if packed is None:
            self.k, self.v = new(*rows, head_dim), new(*rows, head_dim)
        else:
            empty = S.PackedSpec.empty(batch, layers * kv_heads, n_rows, head_dim, packed, device=device)
            self.k, self.v, self.k_scale, self.v_scale = (
                t.view(*rows, -1) for t in (empty.k, empty.v, empty.k_scale, empty.v_scale))
        self.scores = new(batch, layers * kv_heads, n_rows, dt=torch.float32) if keep_scores else None
        self.row_pos = new(batch, layers, kv_heads, n_rows, dt=torch.int32) if positions else None
        self.rows, self.tokens = [0] * batch, [0] * batch
        self._chunk = self._taken = None

    @property
    def n_rows(self) -> int:
        return self.k.shape[3]

    def _rows(self, at):
        """The layers' rows as a cache: `at` takes [B][layers][Hkv][rows][...] to
        [B][heads][rows][...]."""
        if self.packed is None:
            return S.CacheSpec(at(self.k), at(self.v))
        return S.PackedSpec(*(at(t) for t in (self.k, self.v, self.k_scale, self.v_scale)),
                            self.packed)

    def _ints(self, v) -> torch.Tensor:
        return torch.tensor(v, dtype=torch.int32, device=self.k.device)

    def _stream(self) -> Optional[int]:
        return torch._C._cuda_getCurrentRawStream(self.k.device.index) if self.k.is_cuda else None

    def begin(self, new: Sequence[int]) -> int:
        """Announce new[b] more tokens per sequence (packed in this order); their number.
        The layers then take them one by one."""
        if len(new) != len(self.rows) or min(new) < 0:
            raise ValueError("begin() takes the number of new tokens of every sequence")
        rows = [r + n for r, n in zip(self.rows, new)]
        if max(rows) > self.n_rows:
            raise ValueError(f"{max(rows)} rows do not fit a cache of {self.n_rows}")
        start = [0]
        for n in new:
            start.append(start[-1] + n)
        pos = [t + i for t, n in zip(self.tokens, new) for i in range(n)]
        self._positions = self._ints(pos)
        self._chunk = S.ChunkSpec(self._ints(start), self._ints(rows), start[-1],
                                  max(max(new), 1), max(max(rows), 1))
        self._taken = rows, [t + n for t, n in zip(self.tokens, new)]
        self._home = self._stream()
        return start[-1]

    def layer(self, layer: int, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor):
        """The chunk's queries, keys and values in one layer (negative: from the last):
        (attention output, turned queries), [T][Hq][d] both.  What is refused is refused
        before anything is written."""
        if self._chunk is None:
            raise ValueError("begin() first")
        if not -self.layers <= layer < self.layers:
            raise IndexError(f"layer {layer} of {self.layers}")
        layer %= self.layers
        if self.packed is not None and q.dtype != self.dtype:
            raise ValueError(f"queries of {q.dtype} for a cache of {self.dtype}")
        cache = self._rows(lambda t: t[:, layer])
        scale = softmax_scale(self.head_dim)
        pos = None if self.row_pos is None else self.row_pos[:, layer]
        add = S.prepare_append(self._chunk, cache, self.rope, q, k, v, positions=self._positions,
                               row_pos=pos)
        attn = S.prepare_chunk_attn(self._chunk, cache, add.q_out, scale)
        calls = [add, attn]
        if self.scores is not None:
            h = slice(layer * self.kv_heads, (layer + 1) * self.kv_heads)
            calls.append(S.prepare_chunk_scores(self._chunk, cache, add.q_out, attn.lse, scale,
                                                self.scores[:, h], before=self.scores[:, h]))
        for call in calls:
            call.run()
        if self._stream() != self._home:  # the chunk's tensors, which the next begin() drops
            for t in (self._chunk.start, self._chunk.length, self._positions):
                t.record_stream(torch.cuda.current_stream(self.k.device))
        self.rows, self.tokens = self._taken
        return attn.out, add.q_out

    def compress(self, keep: Sequence[int], recent: Optional[Sequence[int]] = None, sinks: int = 0,
                 n_rows: Optional[int] = None) -> "ModelCache":
        """A cache of n_rows rows (default: the largest keep) that holds keep[b] of each
        sequence's rows: the first `sinks`, the last recent[b], and those that
        received most attention.  Needs keep_scores."""
        if self.scores is None:
            raise ValueError("compress() needs a cache with keep_scores")
        B, L, H = self.k.shape[:3]
        to = ModelCache(B, L, self.q_heads, H, self.head_dim, n_rows or max(max(keep), 1), self.rope,
                        self.dtype, self.k.device, keep_scores=True, positions=True,
                        packed=self.packed)
        pos = None if self.row_pos is None else self.row_pos.view(B, L * H, -1)
        def all_layers(t):
            return t.flatten(1, 2)
        S.prepare_evict(self._rows(all_layers), to._rows(all_layers), self._ints(self.rows),
                        self._ints(keep), self.scores,
                        recent=None if recent is None else self._ints(recent), sinks=sinks,
                        row_pos=pos, out_pos=to.row_pos.view(B, L * H, -1), out_scores=to.scores,
                        max_len=max(max(self.rows), 1)).run()
        to.rows = [max(0, min(k, r, to.n_rows)) for k, r in zip(keep, self.rows)]
        to.tokens = list(self.tokens)
        return to

    def read_back(self, out: Optional[tuple] = None, begin: Optional[Sequence[int]] = None):
        """A packed cache's rows as plain keys and values (k, v) [B][layers][Hkv][n_rows][d]; out:
        such a pair to write into (None: a new one, 0 where there are no rows), begin[b]: the
        first row of each sequence to read (the others of `out` stay as they are)."""
        if self.packed is None:
            raise ValueError("read_back() is for packed caches")
        if out is None:
            out = tuple(torch.zeros((*self.k.shape[:4], self.head_dim), dtype=self.dtype,
                                    device=self.k.device) for _ in range(2))
        k, v = out
        if not tuple(k.shape) == tuple(v.shape) == (*self.k.shape[:4], self.head_dim):
            raise ValueError("out must be two tensors [B][layers][Hkv][n_rows][d]")
        S.prepare_read(self._rows(lambda t: t.flatten(1, 2)),
                       S.CacheSpec(k.view(k.shape[0], -1, *k.shape[3:]), v.view(v.shape[0], -1, *v.shape[3:])),
                       self._ints(self.rows), None if begin is None else self._ints(begin),
                       max_len=max(max(self.rows), 1)).run()
        return k, v

    def small_inputs(self, into: Optional[dict] = None, begin: Optional[Sequence[int]] = None) -> dict:
        """The small model's entries of a step's inputs (see prepare_step).  A plain cache's rows
        and the positions are the cache's own tensors, which later chunks reach.  A packed
        cache's rows are read back, and s_held is counted, as of this call.  into: what an
        earlier call returned (other entries may be beside it), which is brought up to date in
        place and returned, so that a step prepared from it finds the present rows; begin[b]: the
        first row of each sequence that it does not hold yet (None: every row is read again)."""
        if into is None:
            k, v = (self.k, self.v) if self.packed is None else self.read_back()
            x = {"s_k": k, "s_v": v}
            if self.row_pos is not None:
                x.update(s_held=self._ints(self.rows), s_row_pos=self.row_pos)
            return x
        own = self.packed is not None or (into.get("s_k") is self.k and into.get("s_v") is self.v)
        if not own or "s_k" not in into or "s_v" not in into or \
                into.get("s_row_pos") is not self.row_pos or ("s_held" in into) != (self.row_pos is not None):
            raise ValueError("into must be what small_inputs() of this cache returned")
        if self.packed is not None:
            self.read_back((into["s_k"], into["s_v"]), begin)
        if self.row_pos is not None:
            into["s_held"].copy_(self._ints(self.rows))
        return into
