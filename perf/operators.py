"""The cache operators as cases that can be timed and compared.

Kinds of a case:
  append  the new tokens' queries and keys turned by their rotary positions,
          keys and values written into the cache
  attn    attention of the new tokens over a paged or dense cache
  scores  the attention weight that the new tokens give every cached row,
          added to the rows' running scores
  evict   the rows of largest score kept, the others dropped: a compact cache
          with its rows' positions and scores

`own` chooses who computes a pass: elementary torch operations in 32 bits, or
the library's calls.  Head counts are those of the model pairs that the
library's workloads name.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}

# (query heads, kv heads, head dim)
SHAPES = {"qwen2-0.5b": (14, 2, 64), "qwen2-7b": (28, 4, 128), "qwen2-72b": (64, 8, 128),
          "llama3-8b": (32, 8, 128), "llama3.2-1b": (32, 8, 64)}

# batch sequences of n_lo..n cached rows each (n_lo 0: all n), of which
# new_lo..new are new; the last `singles` sequences have one new token.
# page 0: a dense cache; rows_first: pages hold [row][head] instead of [head][row].
BASE = dict(shape="qwen2-7b", dtype="bf16", batch=1, n=8192, n_lo=0, new=1, new_lo=0, singles=0,
            page=16, rows_first=False)


def case(kind, name=None, **kw):
    c = dict(BASE, kind=kind, **kw)
    if kind == "append":
        for k, v in (("layout", "half"), ("rot", SHAPES[c["shape"]][2]), ("scaling", "none"),
                     ("far", 0)):
            c.setdefault(k, v)
    if kind == "scores":
        c.setdefault("per_kv", False)
    if kind == "evict":
        for k, v in (("layers", 1), ("keep", 20), ("recent", 5), ("sinks", 4), ("group", 1)):
            c.setdefault(k, v)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one decode step of a batch of chats: a token each, latency counts
        case("append", "append-step", batch=64, n=4096, n_lo=1024),
        # a batch of prompts on a model stretched to a longer context, part of
        # each head turned, neighbours paired
        case("append", "append-prompts", shape="llama3-8b", batch=4, n=8192, n_lo=5000, new=8192,
             new_lo=4096, layout="interleaved", rot=64, scaling="ramp", far=100000, page=64),
        # a long prompt's chunk in 32 bits, an odd number of tokens
        case("append", "append-chunk-f32", shape="qwen2-0.5b", dtype="f32", n=20011, new=5003,
             scaling="bands", page=0),
        # the smallest attention: one token of one sequence, 32 bits
        case("attn", "attn-token-f32", dtype="f32", n=512, page=0),
        # one decode step of a batch of reasoning traces of mixed lengths
        case("attn", "attn-step", batch=64, n=4096, n_lo=1024),
        # a serving step of the small model: prompt chunks among single tokens
        case("attn", "attn-mixed", shape="qwen2-0.5b", batch=20, n=6007, n_lo=900, new=517,
             new_lo=130, singles=16, page=32),
        # long prompts taken in chunks of 4096 tokens
        case("attn", "attn-prompts", shape="llama3-8b", batch=2, n=32768, new=4096, page=64),
        # scores of a decode step over the small model's cache
        case("scores", "scores-step", shape="qwen2-0.5b", batch=16, n=8192, n_lo=2000, per_kv=True),
        # scores of a long prompt's chunk, per query head
        case("scores", "scores-chunk", shape="llama3.2-1b", n=16384, new=2048, page=64),
        # one layer of a short chat in 32 bits
        case("evict", "evict-layer-f32", shape="qwen2-0.5b", dtype="f32", n=1237, keep=40),
        # every layer of the small model after a prompt, kept to 40%
        case("evict", "evict-prompt", shape="qwen2-0.5b", layers=24, n=8192, keep=40, group=7,
             page=0),
        # a batch of long contexts of another pair's small model
        case("evict", "evict-batch", shape="llama3.2-1b", layers=16, batch=4, n=32768, n_lo=20000,
             page=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attn", "attn", "attn", "scores", "scores", "evict", "evict"])
    shape = rng.choice(list(SHAPES))
    hq, hk, d = SHAPES[shape]
    c = dict(shape=shape, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]),
             page=rng.choice([0, 8, 16, 32, 64, 128, 256]), rows_first=rng.random() < 0.3)
    n = _log_int(rng, 1, 32768)
    batch = _log_int(rng, 1, 64)
    if kind == "evict":
        layers = rng.choice([1, 1, 4, 16, 24])
        while batch * layers * hk * n * d > 1 << 30:
            batch = max(1, batch // 2)
            n = n * 3 // 4
        c.update(layers=layers, keep=rng.choice([5, 10, 20, 40, 75]), recent=rng.choice([0, 2, 10]),
                 sinks=rng.choice([0, 1, 4]), group=rng.choice([1, 1, hq // hk]))
        return case(kind, batch=batch, n=n, n_lo=rng.choice([0, max(1, n // 4)]), **c)
    new = 1 if rng.random() < 0.35 else _log_int(rng, 1, 4096)
    new = min(new, n)
    while batch * n * hk * d > 1 << 28:  # the cache
        batch = max(1, batch // 2)
        n = max(1, n * 3 // 4)
        new = min(new, n)
    # pairs of a query row and a cached row; 32-bit products cost more
    limit = (4e9 if kind == "attn" else 1.2e9) / (4 if c["dtype"] == "f32" else 1)
    while batch * new * n * hq * (d / 128) > limit:
        if batch > 1:
            batch = max(1, batch // 2)
        else:
            new = max(1, new // 2)
    c.update(batch=batch, n=n, new=new, n_lo=rng.choice([0, max(1, n // 4)]),
             new_lo=rng.choice([0, 0, max(1, new // 3)]),
             singles=rng.choice([0, 0, batch // 2]) if new > 1 else 0)
    if kind == "append":
        c.update(layout=rng.choice(["half", "interleaved"]),
                 rot=rng.choice([d, d, d // 2, d // 4, 2 * rng.randint(1, d // 2)]),
                 scaling=rng.choice(["none", "linear", "base", "ramp", "bands"]),
                 far=rng.choice([0, 0, 1000, 131072, 1000003]))
    if kind == "scores":
        c.update(per_kv=rng.random() < 0.5)
    return case(kind, **c)


# ------------------------------------------------------------------ inputs --

def _spread(lo, hi, i):
    """The i-th of values spread over [lo, hi] (lo 0: all hi)."""
    return hi if lo == 0 else lo + int((hi - lo) * ((0.5 + i * 0.6180339887498949) % 1.0) + 0.5)


def lengths(c):
    """(cached rows, new tokens) of every sequence."""
    out = []
    for b in range(c["batch"]):
        new = 1 if b >= c["batch"] - c["singles"] else _spread(c["new_lo"], c["new"], b)
        out.append((max(_spread(c["n_lo"], c["n"], b), new), new))
    return out


def _frequencies(rot, scaling):
    """Angles per position of the rot/2 pairs, in 64 bits, and the factor on
    the turned elements: positions of a model of 8192 tokens stretched by 4."""
    base, factor, orig = 1e6, 4.0, 8192
    i = torch.arange(0, rot, 2, dtype=torch.float64)
    amp = 1.0
    if scaling == "base":
        if rot > 2:
            base *= factor ** (rot / (rot - 2))
    f = base ** (-i / rot)
    if scaling == "linear":
        f = f / factor
    elif scaling == "ramp":
        def pair(turns):
            return rot * math.log(orig / (turns * 2 * math.pi)) / (2 * math.log(base))
        lo, hi = max(math.floor(pair(32.0)), 0), min(math.ceil(pair(1.0)), rot - 1)
        t = ((i / 2 - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
        f = f / factor * t + f * (1 - t)
        amp = 0.1 * math.log(factor) + 1.0
    elif scaling == "bands":
        t = ((orig * f / (2 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0, 1)
        f = f / factor * (1 - t) + f * t
    return f.to(DEV), amp


def _generator(c, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) & ((1 << 62) - 1))
    return g


def _cache(c, heads, d, rows, g, fill=True):
    """Pools of keys and values seen as [page][head][row][d] and the page table
    (None: dense, a page per sequence), for sequences of up to `rows` rows."""
    dt, page = DTYPES[c["dtype"]], c["page"] or rows
    width = (rows + page - 1) // page
    pages = c["batch"] * width + (3 if c["page"] else 0)
    shape = (pages, page, heads, d) if c["rows_first"] else (pages, heads, page, d)
    pools = []
    for _ in range(2):
        t = torch.zeros(shape, dtype=dt, device=DEV)
        if fill:
            for p in range(0, pages, max(1, (1 << 26) // max(1, page * heads * d))):
                q = p + max(1, (1 << 26) // max(1, page * heads * d))
                t[p:q] = torch.randn(t[p:q].shape, device=DEV, generator=g).to(dt)
        pools.append(t.transpose(1, 2) if c["rows_first"] else t)
    table = None
    if c["page"]:
        perm = torch.randperm(pages, device=DEV, generator=g)[: c["batch"] * width]
        table = perm.view(c["batch"], width).to(torch.int32).contiguous()
    return pools[0], pools[1], table


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def prepare(c, seed):
    hq, hk, d = SHAPES[c["shape"]]
    dt, g, lens = DTYPES[c["dtype"]], _generator(c, seed), lengths(c)
    rows = max(n for n, _ in lens)
    s = {"c": c, "lens": lens, "rows": rows, "length": _ints([n for n, _ in lens])}
    if c["kind"] == "evict":
        _prepare_evict(c, s, g, hk * c["layers"], d)
        return s
    start = [0]
    for _, new in lens:
        start.append(start[-1] + new)
    T = start[-1]
    s.update(starts=start, start=_ints(start), new=max(new for _, new in lens))
    s["k"], s["v"], s["table"] = _cache(c, hk, d, rows, g)
    # queries and keys as a projection leaves them, one row per token
    qkv = torch.randn((T, (hq + 2 * hk) * d), device=DEV, generator=g).to(dt)
    s["q"] = qkv[:, : hq * d].view(T, hq, d)
    if c["kind"] == "append":
        s["new_k"] = qkv[:, hq * d: (hq + hk) * d].view(T, hk, d)
        s["new_v"] = qkv[:, (hq + hk) * d:].view(T, hk, d)
        s["freq"], s["amp"] = _frequencies(c["rot"], c["scaling"])
        row = torch.cat([torch.arange(n - new, n) for n, new in lens])
        s["pos"] = (row + c["far"]).to(torch.int32).to(DEV)
        s["row"] = row.to(DEV)  # each token's cached row and sequence
        s["seq"] = torch.repeat_interleave(torch.arange(c["batch"]),
                                           torch.tensor([new for _, new in lens])).to(DEV)
        s["q_out"] = torch.zeros((T, hq, d), dtype=dt, device=DEV)
    else:
        s["scale"] = 1.0 / math.sqrt(d)
        # the first rows draw most of the attention
        for b, (n, _) in enumerate(lens):
            for r in range(min(4, n)):
                p, o = (b, r) if s["table"] is None else (s["table"][b, r // c["page"]].long(),
                                                          r % c["page"])
                s["k"][p, :, o] *= 2.5
    if c["kind"] == "scores":
        s["lse"] = _plain_attn(s, need_out=False)["lse"]
        heads = hk if c["per_kv"] else hq
        s["before"] = torch.rand((c["batch"], heads, rows), device=DEV, generator=g)
        s["after"] = torch.zeros_like(s["before"])
    if own:
        from paper_2508_02751_amd import smallkv as S
        chunk = S.ChunkSpec(s["start"], s["length"], T, s["new"], rows)
        cache = S.CacheSpec(s["k"], s["v"], s["table"])
        if c["kind"] == "append":
            rope = S.RopeSpec(s["freq"], S.ROPE_HALF if c["layout"] == "half" else
                              S.ROPE_INTERLEAVED, s["amp"])
            s["call"] = S.prepare_append(chunk, cache, rope, s["q"], s["new_k"], s["new_v"],
                                         positions=s["pos"], q_out=s["q_out"])
        elif c["kind"] == "attn":
            s["call"] = S.prepare_chunk_attn(chunk, cache, s["q"], s["scale"])
        else:
            s["call"] = S.prepare_chunk_scores(chunk, cache, s["q"], s["lse"], s["scale"],
                                               s["after"], before=s["before"])
    return s


def _budgets(c, lens):
    return [(max(1, n * c["keep"] // 100), n * c["recent"] // 100) for n, _ in lens]


def _prepare_evict(c, s, g, heads, d):
    s["k"], s["v"], s["table"] = _cache(c, heads, d, s["rows"], g)
    budgets = _budgets(c, s["lens"])
    s["budgets"] = budgets
    s["keep"], s["recent"] = _ints([k for k, _ in budgets]), _ints([r for _, r in budgets])
    kept = max(k for k, _ in budgets)
    # running scores: heavy-tailed, larger for older rows, some rows never
    # attended (equal to the last bit)
    sh = (c["batch"], heads * c["group"], s["rows"])
    t = torch.exp(2.0 * torch.randn(sh, device=DEV, generator=g))
    t /= torch.arange(s["rows"], 0, -1, device=DEV).flip(0) + 16.0
    t[torch.rand(sh, device=DEV, generator=g) < 0.02] = 0.0
    s["before"] = t
    # the rows of a cache that was compacted before: positions with gaps
    gaps = torch.randint(1, 4, (c["batch"], heads, s["rows"]), device=DEV, generator=g)
    s["row_pos"] = (gaps.cumsum(2) - 1).to(torch.int32)
    dense = dict(c, page=0, rows_first=False)
    s["out_k"], s["out_v"], _ = _cache(dense, heads, d, kept, g, fill=False)
    s["out_pos"] = torch.zeros((c["batch"], heads, kept), dtype=torch.int32, device=DEV)
    s["after"] = torch.zeros((c["batch"], heads * c["group"], kept), device=DEV)
    s["held"] = torch.zeros(c["batch"], dtype=torch.int32, device=DEV)
    if own:
        from paper_2508_02751_amd import smallkv as S
        s["call"] = S.prepare_evict(S.CacheSpec(s["k"], s["v"], s["table"]),
                                    S.CacheSpec(s["out_k"], s["out_v"]), s["length"], s["keep"],
                                    s["before"], recent=s["recent"], sinks=c["sinks"],
                                    row_pos=s["row_pos"], out_pos=s["out_pos"],
                                    out_scores=s["after"], held=s["held"])


# --------------------------------------------------------------- one pass --

def run(state):
    kind = state["c"]["kind"]
    if own:
        call = state["call"]
        call.run()
        if kind == "append":
            return {"q": call.q_out, "k": state["k"], "v": state["v"]}
        if kind == "attn":
            return {"out": call.out, "lse": call.lse}
        if kind == "scores":
            return {"scores": state["after"]}
        return {"k": state["out_k"], "v": state["out_v"], "pos": state["out_pos"],
                "scores": state["after"], "held": state["held"]}
    return {"append": _plain_append, "attn": _plain_attn, "scores": _plain_scores,
            "evict": _plain_evict}[kind](state)


def _slots(s, b, lo, hi):
    """(pages, rows in them) of the sequence's rows lo..hi-1."""
    r = torch.arange(lo, hi, device=DEV)
    if s["table"] is None:
        return torch.full_like(r, b), r
    page = s["c"]["page"]
    return s["table"][b].long()[r // page], r % page


def _turn(x, cos, sin, rot, layout):
    """x [T][heads][d] in 32 bits; cos, sin [T][1][rot/2]."""
    y = x.clone()
    if layout == "half":
        a, b = x[..., : rot // 2], x[..., rot // 2: rot]
        y[..., : rot // 2] = a * cos - b * sin
        y[..., rot // 2: rot] = a * sin + b * cos
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2] = a * cos - b * sin
        y[..., 1:rot:2] = a * sin + b * cos
    return y


def _plain_append(s):
    c = s["c"]
    dt = DTYPES[c["dtype"]]
    angle = s["pos"].double()[:, None, None] * s["freq"]
    cos, sin = (s["amp"] * torch.cos(angle)).float(), (s["amp"] * torch.sin(angle)).float()
    s["q_out"].copy_(_turn(s["q"].float(), cos, sin, c["rot"], c["layout"]).to(dt))
    k = _turn(s["new_k"].float(), cos, sin, c["rot"], c["layout"]).to(dt)
    pages, rows = s["seq"], s["row"]
    if s["table"] is not None:
        pages, rows = s["table"].long()[s["seq"], s["row"] // c["page"]], s["row"] % c["page"]
    s["k"][pages, :, rows] = k
    s["v"][pages, :, rows] = s["new_v"]
    return {"q": s["q_out"], "k": s["k"], "v": s["v"]}


def _gather(s, pool, b, n):
    pages, rows = _slots(s, b, 0, n)
    return pool[pages, :, rows].transpose(0, 1).float().contiguous()  # [heads][n][d]


def _logits(s, b, t0, t1, kt):
    """Logits of the sequence's new tokens t0..t1-1: [kv heads][g*(t1-t0)][n],
    query heads outermost, the rows after a token's own at -inf."""
    n, new = s["lens"][b]
    hk, d = kt.shape[0], kt.shape[1]
    q = s["q"][s["starts"][b] + t0: s["starts"][b] + t1].float()
    g = q.shape[1] // hk
    q = q.view(t1 - t0, hk, g, d).permute(1, 2, 0, 3).reshape(hk, g * (t1 - t0), d)
    x = torch.matmul(q, kt) * s["scale"]
    own_row = torch.arange(n - new + t0, n - new + t1, device=DEV).repeat(g)
    return x.masked_fill_(torch.arange(n, device=DEV) > own_row[:, None], -math.inf)


def _blocks(n, new, heads):
    step = max(1, (1 << 29) // max(1, n * heads))  # logits of at most 2 GiB
    return [(t, min(t + step, new)) for t in range(0, new, step)]


def _plain_attn(s, need_out=True):
    q = s["q"]
    T, hq, d = q.shape
    out = torch.empty_like(q, memory_format=torch.contiguous_format)
    lse = torch.empty((T, hq), dtype=torch.float32, device=DEV)
    for b, (n, new) in enumerate(s["lens"]):
        kt = _gather(s, s["k"], b, n).transpose(1, 2).contiguous()
        v = _gather(s, s["v"], b, n) if need_out else None
        for t0, t1 in _blocks(n, new, hq):
            x = _logits(s, b, t0, t1, kt)
            m = x.amax(-1, keepdim=True)
            x = x.sub_(m).exp_()
            z = x.sum(-1, keepdim=True)
            hk, rows = kt.shape[0], slice(s["starts"][b] + t0, s["starts"][b] + t1)
            if need_out:
                o = (torch.matmul(x, v) / z).view(hk, hq // hk, t1 - t0, d)
                out[rows] = o.permute(2, 0, 1, 3).reshape(t1 - t0, hq, d).to(out.dtype)
            lse[rows] = (m + z.log()).view(hq, t1 - t0).t()
    return {"out": out, "lse": lse}


def _plain_scores(s):
    c = s["c"]
    hq, hk, _ = SHAPES[c["shape"]]
    for b, (n, new) in enumerate(s["lens"]):
        kt = _gather(s, s["k"], b, n).transpose(1, 2).contiguous()
        f = torch.zeros((hq, n), device=DEV)
        for t0, t1 in _blocks(n, new, hq):
            lse = s["lse"][s["starts"][b] + t0: s["starts"][b] + t1].t().reshape(hk, -1, 1)
            x = _logits(s, b, t0, t1, kt).sub_(lse).exp_()
            f += x.view(hq, t1 - t0, n).sum(1)
        if c["per_kv"]:
            f = f.view(hk, hq // hk, n).sum(1)
        f[:, : n - new] += s["before"][b, :, : n - new]
        s["after"][b, :, :n] = f
    return {"scores": s["after"]}


def _plain_evict(s):
    c = s["c"]
    for b, ((n, _), (keep, recent)) in enumerate(zip(s["lens"], s["budgets"])):
        kept = min(keep, n)
        r = min(recent, kept)
        first = min(c["sinks"], kept - r)
        top = kept - r - first
        heads = s["out_k"].shape[1]
        x = s["before"][b, :, :n].view(heads, c["group"], n)
        f = x[:, 0]
        for i in range(1, c["group"]):
            f = f + x[:, i]
        order = torch.sort(f[:, first: n - r], dim=1, descending=True, stable=True).indices
        chosen = torch.zeros((heads, n), dtype=torch.bool, device=DEV)
        chosen[:, :first] = True
        chosen[:, n - r:] = True
        chosen.scatter_(1, order[:, :top] + first, True)
        rows = torch.nonzero(chosen)[:, 1].view(heads, kept)
        h = torch.arange(heads, device=DEV)[:, None]
        if s["table"] is None:
            pages, at = torch.full_like(rows, b), rows
        else:
            pages, at = s["table"][b].long()[rows // c["page"]], rows % c["page"]
        s["out_k"][b, :, :kept] = s["k"][pages, h, at]
        s["out_v"][b, :, :kept] = s["v"][pages, h, at]
        s["out_pos"][b, :, :kept] = s["row_pos"][b].gather(1, rows)
        s["after"][b, :, :kept] = s["before"][b].gather(
            1, rows.repeat_interleave(c["group"], 0))
        s["held"][b] = kept
    return {"k": s["out_k"], "v": s["out_v"], "pos": s["out_pos"], "scores": s["after"],
            "held": s["held"]}


# -------------------------------------------------------------------- work --

def work(c):
    hq, hk, d = SHAPES[c["shape"]]
    e = 4 if c["dtype"] == "f32" else 2
    lens = lengths(c)
    T, rows = sum(new for _, new in lens), sum(n for n, _ in lens)
    # a new token attends to the rows up to its own
    pairs = sum(new * (n - new) + new * (new + 1) // 2 for n, new in lens)
    if c["kind"] == "append":
        return {"bytes": 2 * T * (hq + 2 * hk) * d * e + 4 * T,
                "flops": 3 * T * (hq + hk) * c["rot"]}
    if c["kind"] == "attn":
        return {"bytes": 2 * rows * hk * d * e + T * hq * (2 * d * e + 4),
                "flops": 4 * pairs * hq * d}
    if c["kind"] == "scores":
        heads = hk if c["per_kv"] else hq
        old = sum(n - new for n, new in lens)
        return {"bytes": rows * hk * d * e + T * hq * (d * e + 4) + 4 * heads * (old + rows),
                "flops": 2 * pairs * hq * d}
    heads, kept = hk * c["layers"], sum(k for k, _ in _budgets(c, lens))
    return {"bytes": heads * (4 * c["group"] * rows + kept * (4 * d * e + 8 + 4 * c["group"])),
            "flops": heads * c["group"] * rows}


# ------------------------------------------------------- the same in 64 bits --

def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] == "append":
        return _exact_append(s)
    if c["kind"] == "evict":
        return _exact_evict(s)
    lens, q = s["lens"], s["q"]
    hq, hk, d = SHAPES[c["shape"]]
    g = hq // hk
    if c["kind"] == "attn":
        out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
        lse = torch.zeros(q.shape[:2], dtype=torch.float64, device=DEV)
    else:
        acc = torch.zeros(s["after"].shape, dtype=torch.float64, device=DEV)
    for b, (n, new) in enumerate(lens):
        a = torch.arange(n, device=DEV)
        at = (torch.full_like(a, b), a) if s["table"] is None else (
            torch.index_select(s["table"][b], 0, a // c["page"]).long(), a % c["page"])
        step = max(1, (1 << 27) // (n * g))
        for h in range(hk):
            K = s["k"][at[0], h, at[1]].double()
            V = s["v"][at[0], h, at[1]].double()
            for j in range(g if c["kind"] == "scores" else 1):
                # one query head at a time where sums over rows are kept per head
                js = slice(j, j + 1) if c["kind"] == "scores" else slice(0, g)
                f = torch.zeros(n, dtype=torch.float64, device=DEV)
                for t0 in range(0, new, step):
                    t1 = min(t0 + step, new)
                    i = slice(s["starts"][b] + t0, s["starts"][b] + t1)
                    heads_of = slice(h * g + js.start, h * g + js.stop)
                    x = q[i, heads_of].double().reshape(-1, d) @ K.t().contiguous()
                    x = (x * s["scale"]).view(t1 - t0, -1, n)
                    seen = a[None, :] <= (n - new + torch.arange(t0, t1, device=DEV))[:, None]
                    x = torch.where(seen[:, None], x, torch.tensor(-math.inf, device=DEV,
                                                                   dtype=torch.float64))
                    if c["kind"] == "attn":
                        lse[i, heads_of] = torch.logsumexp(x, -1)
                        w = torch.softmax(x, -1)
                        out[i, heads_of] = (w.reshape(-1, n) @ V).view(t1 - t0, -1, d)
                    else:
                        f += torch.exp(x - s["lse"][i, heads_of].double()[..., None]).sum((0, 1))
                if c["kind"] == "scores":
                    acc[b, h if c["per_kv"] else h * g + j, :n] += f
        if c["kind"] == "scores":
            acc[b, :, : n - new] += s["before"][b, :, : n - new].double()
    return {"out": out, "lse": lse} if c["kind"] == "attn" else {"scores": acc}


def _exact_append(s):
    c, lens = s["c"], s["lens"]
    rot = c["rot"]
    th = s["pos"].to(torch.float64).unsqueeze(1) * s["freq"].unsqueeze(0)  # [T][rot/2]
    turn = torch.polar(torch.full_like(th, s["amp"]), th).unsqueeze(1)

    def turned(x):
        x = x.double()
        head = x[..., :rot]
        if c["layout"] == "half":
            z = torch.complex(head[..., : rot // 2].contiguous(), head[..., rot // 2:].contiguous())
            z = z * turn
            head = torch.cat([z.real, z.imag], -1)
        else:
            z = torch.view_as_complex(head.reshape(*head.shape[:-1], rot // 2, 2).contiguous())
            head = torch.view_as_real(z * turn).flatten(-2)
        return torch.cat([head, x[..., rot:]], -1)

    out = {"q": turned(s["q"]), "k": s["k"].double(), "v": s["v"].double()}
    k, v = turned(s["new_k"]), s["new_v"].double()
    i = 0
    for b, (n, new) in enumerate(lens):
        r = n - new + torch.arange(new, device=DEV)
        page = c["page"] or s["rows"]
        p = s["table"][b].long().index_select(0, r // page) if c["page"] else r * 0 + b
        out["k"][p, :, r % page] = k[i: i + new]
        out["v"][p, :, r % page] = v[i: i + new]
        i += new
    return out


def _exact_evict(s):
    """Moved values: the rows by their rank, counted instead of sorted (None
    where that takes long)."""
    c, lens = s["c"], s["lens"]
    heads = s["out_k"].shape[1]
    if sum(heads * n * n for n, _ in lens) > 1 << 40:
        return None
    out = {"k": s["out_k"].double(), "v": s["out_v"].double(), "pos": s["out_pos"].clone(),
           "scores": s["after"].double(), "held": s["held"].clone()}
    for b, ((n, _), (keep, recent)) in enumerate(zip(lens, s["budgets"])):
        kept = min(keep, n)
        r = min(recent, kept)
        first = min(c["sinks"], kept - r)
        idx = torch.arange(n, device=DEV)
        for h in range(heads):
            x = s["before"][b, h * c["group"]: (h + 1) * c["group"], :n]
            f = x[0].clone()
            for i in range(1, c["group"]):
                f += x[i]  # in 32 bits: the sum that ranks the rows is defined so
            fixed = (idx < first) | (idx >= n - r)
            f = torch.where(fixed, torch.full_like(f, math.inf), f)
            rank = torch.zeros(n, dtype=torch.int64, device=DEV)
            for j in range(0, n, 4096):
                o, oi = f[j: j + 4096, None], idx[j: j + 4096, None]
                rank += ((o > f) | ((o == f) & (oi < idx))).sum(0)
            rows = idx[rank < kept]
            page = c["page"] or s["rows"]
            p = s["table"][b].long()[rows // page] if c["page"] else rows * 0 + b
            out["k"][b, h, :kept] = s["k"][p, h, rows % page].double()
            out["v"][b, h, :kept] = s["v"][p, h, rows % page].double()
            out["pos"][b, h, :kept] = s["row_pos"][b, h, rows]
            out["scores"][b, h * c["group"]: (h + 1) * c["group"], :kept] = \
                s["before"][b, h * c["group"]: (h + 1) * c["group"], rows].double()
        out["held"][b] = kept
    return out
