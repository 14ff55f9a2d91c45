"""The packed cache's operators as cases that can be timed and compared.

A packed cache holds keys and values in 8 or 4 bits: blocks of 32 elements of a
row share a power of two, an element is a small float times it.

  mxfp8  1 sign, 4 exponent and 3 mantissa bits, up to 448
  mxfp4  1 sign, 2 exponent and 1 mantissa bit, up to 6, two to a byte

Kinds of a case:
  append  the new tokens' queries and keys turned by their rotary positions, keys
          and values packed and written into the cache
  read    packed rows read back into the dense cache that a decode step reads;
          where the case has new tokens they are appended first, and their rows read
  attn    attention of the new tokens over a packed cache
  scores  the attention weight that the new tokens give every packed row, added
          to the rows' running scores
  evict   the packed rows of largest score kept, the others dropped

`own` chooses who computes a pass: elementary torch operations in 32 bits (64
where a value is next to a border of two codes), or the library's calls.  Head
counts are those of the model pairs that the library's workloads name.
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
BASE = dict(shape="qwen2-7b", dtype="bf16", format="mxfp8", batch=1, n=8192, n_lo=0, new=1, new_lo=0,
            singles=0, page=16, rows_first=False)


def case(kind, name=None, **kw):
    c = dict(BASE, kind=kind, **kw)
    if kind in ("append", "read"):
        for k, v in (("layout", "half"), ("rot", SHAPES[c["shape"]][2]), ("far", 0)):
            c.setdefault(k, v)
    if kind == "scores":
        c.setdefault("per_kv", False)
    if kind == "evict":
        c["new"] = 0
        for k, v in (("keep", 20), ("recent", 5), ("sinks", 4), ("group", 1)):
            c.setdefault(k, v)
    if kind in ("read", "evict"):
        c.setdefault("layers", 1)  # without new tokens: of layers * kv heads
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one decode step of a batch of chats: a token each, latency counts
        case("append", "append-step", batch=64, n=4096, n_lo=1024),
        # a batch of prompts, part of each head turned, neighbours paired
        case("append", "append-prompts", shape="llama3-8b", batch=3, n=12011, n_lo=7000, new=9000,
             new_lo=5000, layout="interleaved", rot=96, far=100000, page=64),
        # a chunk of a 32-bit model, an odd number of tokens: packed, and its rows read
        # back as the next step of the compensated attention sees them
        case("read", "read-chunk-f32", shape="qwen2-0.5b", dtype="f32", format="mxfp4", batch=2,
             n=9011, new=1501, page=32),
        # every layer of a batch of long contexts, read back for a decode step
        case("read", "read-batch", shape="llama3.2-1b", layers=4, batch=4, n=32768, n_lo=20000, new=0,
             page=64),
        # the smallest attention: one token of one sequence, 32 bits
        case("attn", "attn-token-f32", dtype="f32", n=512, page=0),
        # one decode step of a batch of reasoning traces of mixed lengths
        case("attn", "attn-step", batch=64, n=4096, n_lo=1024),
        # a decode step over a few very long contexts
        case("attn", "attn-long", shape="llama3-8b", format="mxfp4", batch=4, n=131072, n_lo=90001,
             page=64, rows_first=True),
        # prompts taken in chunks
        case("attn", "attn-prompts", shape="llama3-8b", batch=2, n=16384, new=2048, page=64),
        # scores of a decode step over the small model's cache
        case("scores", "scores-step", shape="qwen2-0.5b", format="mxfp4", batch=16, n=8192, n_lo=2000,
             per_kv=True),
        # scores of a prompt's chunk, per query head
        case("scores", "scores-chunk", shape="llama3.2-1b", n=16384, new=1024, page=64),
        # one layer of a short chat
        case("evict", "evict-layer", shape="qwen2-0.5b", n=1237, keep=40),
        # layers of a batch of long contexts
        case("evict", "evict-batch", shape="llama3.2-1b", layers=8, batch=4, n=32768, n_lo=20000,
             page=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "read", "attn", "attn", "attn", "scores", "evict"])
    shape = rng.choice(list(SHAPES))
    hq, hk, d = SHAPES[shape]
    c = dict(shape=shape, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]),
             format=rng.choice(["mxfp8", "mxfp4"]) if kind in ("read", "attn", "scores") else "mxfp8",
             page=rng.choice([0, 8, 16, 32, 64, 128, 256]), rows_first=rng.random() < 0.3)
    n = _log_int(rng, 1, 131072 if kind == "attn" else 32768)
    batch = _log_int(rng, 1, 64)
    new = 1 if rng.random() < 0.35 else _log_int(rng, 1, 4096)
    if kind == "evict" or (kind == "read" and rng.random() < 0.5):
        layers = rng.choice([1, 1, 4, 16, 24])
        while batch * layers * hk * n * d > 1 << (28 if kind == "evict" else 27):
            batch = max(1, batch // 2)
            n = n * 3 // 4
        c.update(layers=layers, new=0)
        if kind == "evict":
            c.update(keep=rng.choice([5, 10, 20, 40, 75]), recent=rng.choice([0, 2, 10]),
                     sinks=rng.choice([0, 1, 4]), group=rng.choice([1, 1, hq // hk]))
        return case(kind, batch=batch, n=n, n_lo=rng.choice([0, max(1, n // 4)]), **c)
    new = min(new, n)
    while batch * n * hk * d > 1 << 28:  # the cache
        batch = max(1, batch // 2)
        n = max(1, n * 3 // 4)
        new = min(new, n)
    # pairs of a query row and a cached row; 32-bit products cost more
    limit = (2e9 if kind == "attn" else 2.5e8) / (4 if c["dtype"] == "f32" else 1)
    while batch * new * n * hq * (d / 128) > limit and kind in ("attn", "scores"):
        if batch > 1:
            batch = max(1, batch // 2)
        else:
            new = max(1, new // 2)
    while batch * new * (hq + 2 * hk) * d > 1 << (26 if c["dtype"] == "f32" else 27):
        batch = max(1, batch // 2)
    c.update(batch=batch, n=n, new=new, n_lo=rng.choice([0, max(1, n // 4)]),
             new_lo=rng.choice([0, 0, max(1, new // 3)]),
             singles=rng.choice([0, 0, batch // 2]) if new > 1 else 0)
    if kind in ("append", "read"):
        c.update(layout=rng.choice(["half", "interleaved"]),
                 rot=rng.choice([d, d, d // 2, d // 4, 2 * rng.randint(1, d // 2)]),
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
    got = []
    for b in range(c["batch"]):
        new = 1 if b >= c["batch"] - c["singles"] else _spread(c["new_lo"], c["new"], b)
        got.append((max(_spread(c["n_lo"], c["n"], b), new), new))
    return got


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _row_bytes(c, d):
    """Bytes of a row's codes."""
    return d if c["format"] == "mxfp8" else d // 2


def _pools(c, heads, d, rows, g, fill=True):
    """Codes and block scales of keys and values seen as [page][head][row][bytes], and
    the page table (None: dense, a page per sequence), for sequences of up to `rows`
    rows.  Filled with packed normal values, the first rows of a page's keys larger."""
    page = c["page"] or rows
    width = (rows + page - 1) // page
    pages = c["batch"] * width + (3 if c["page"] else 0)
    pools = []
    for which in range(2):
        lead = (pages, page, heads) if c["rows_first"] else (pages, heads, page)
        codes = torch.zeros((*lead, _row_bytes(c, d)), dtype=torch.uint8, device=DEV)
        scales = torch.zeros((*lead, d // 32), dtype=torch.uint8, device=DEV)
        step = max(1, (1 << 23) // (page * heads * d))
        for p in range(0, pages if fill else 0, step):
            x = torch.randn((min(step, pages - p), *lead[1:], d), device=DEV, generator=g)
            if which == 0:  # a few channels of keys stand out, as trained models have them
                x[..., :: d // 4] *= 6.0
            codes[p: p + step], scales[p: p + step] = _packed(x.double(), c["format"])
        if c["rows_first"]:
            codes, scales = codes.transpose(1, 2), scales.transpose(1, 2)
        pools += [codes, scales]
    table = None
    if c["page"]:
        perm = torch.randperm(pages, device=DEV, generator=g)[: c["batch"] * width]
        table = perm.view(c["batch"], width).to(torch.int32).contiguous()
    return dict(k=pools[0], k_scale=pools[1], v=pools[2], v_scale=pools[3], table=table)


def _spec(c, s, p):
    from paper_2508_02751_amd import smallkv as S
    return S.PackedSpec(p["k"], p["v"], p["k_scale"], p["v_scale"],
                        S.MXFP8 if c["format"] == "mxfp8" else S.MXFP4, p["table"])


def prepare(c, seed):
    hq, hk, d = SHAPES[c["shape"]]
    lens = lengths(c)
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) & ((1 << 62) - 1))
    rows, new = max(n for n, _ in lens), max(m for _, m in lens)
    heads = hk * c.get("layers", 1)
    s = {"c": c, "lens": lens, "rows": rows, "new": new, "heads": heads,
         "length": _ints([n for n, _ in lens]), "first": _ints([n - m for n, m in lens])}
    s["from"] = _pools(c, heads, d, rows, g, fill=c["kind"] != "append")
    if c["kind"] == "evict":
        _prepare_evict(c, s, g, heads, d)
    elif new:
        _prepare_tokens(c, s, g, lens, (hq, hk, d))
    if c["kind"] == "read":
        _prepare_read(c, s, heads, d)
    if own:
        s["calls"] = _calls(c, s)
    return s


def _prepare_tokens(c, s, g, lens, shape):
    hq, hk, d = shape
    start = [0]
    for _, m in lens:
        start.append(start[-1] + m)
    T = start[-1]
    s.update(T=T, start=_ints(start), scale=1.0 / math.sqrt(d))
    # each token's sequence, its number in it and its cached row; and, for batches padded
    # to the longest chunk, the token at [sequence][number]
    count = torch.tensor([m for _, m in lens], device=DEV)
    s["seq"] = torch.repeat_interleave(torch.arange(c["batch"], device=DEV), count)
    s["number"] = torch.arange(T, device=DEV) - s["start"].long()[s["seq"]]
    s["row"] = s["first"].long()[s["seq"]] + s["number"]
    numbers = torch.arange(s["new"], device=DEV)
    s["padded"] = (s["start"].long()[:-1, None] + numbers).clamp_max(T - 1)
    s["padded_row"] = s["first"].long()[:, None] + numbers
    # queries and keys as a projection leaves them, one row per token
    qkv = torch.randn((T, (hq + 2 * hk) * d), device=DEV, generator=g).to(DTYPES[c["dtype"]])
    s["q"] = qkv[:, : hq * d].view(T, hq, d)
    if c["kind"] in ("append", "read"):
        s["new_k"] = qkv[:, hq * d: (hq + hk) * d].view(T, hk, d)
        s["new_v"] = qkv[:, (hq + hk) * d:].view(T, hk, d)
        s["freq"] = 1e6 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64) / c["rot"]).to(DEV)
        s["pos"] = (s["row"] + c["far"]).to(torch.int32)
        s["q_out"] = torch.zeros((T, hq, d), dtype=s["q"].dtype, device=DEV)
    if c["kind"] == "scores":
        s["lse"] = _plain_attn(s, need_out=False)["lse"]
        shape = (c["batch"], hk if c["per_kv"] else hq, s["rows"])
        s["before"] = torch.rand(shape, device=DEV, generator=g)
        s["after"] = torch.zeros_like(s["before"])


def _prepare_read(c, s, heads, d):
    """The dense cache that is read into, and the rows of each sequence."""
    s["begin"] = s["first"] if s["new"] else torch.zeros_like(s["first"])
    shape = (c["batch"], heads, s["rows"], d)
    s["out_k"] = torch.zeros(shape, dtype=DTYPES[c["dtype"]], device=DEV)
    s["out_v"] = torch.zeros_like(s["out_k"])


def _prepare_evict(c, s, g, heads, d):
    budgets = [(max(1, n * c["keep"] // 100), n * c["recent"] // 100) for n, _ in s["lens"]]
    s["budgets"] = budgets
    s["keep"], s["recent"] = _ints([k for k, _ in budgets]), _ints([r for _, r in budgets])
    kept = max(k for k, _ in budgets)
    # running scores: heavy-tailed, larger for older rows, some rows never
    # attended (equal to the last bit)
    t = torch.exp(2.0 * torch.randn((c["batch"], heads * c["group"], s["rows"]), device=DEV, generator=g))
    t /= torch.arange(s["rows"], 0, -1, device=DEV).flip(0) + 16.0
    t[torch.rand(t.shape, device=DEV, generator=g) < 0.02] = 0.0
    s["before"] = t
    s["to"] = _pools(dict(c, page=0, rows_first=False), heads, d, kept, g, fill=False)
    s["out_pos"] = torch.zeros((c["batch"], heads, kept), dtype=torch.int32, device=DEV)
    s["after"] = torch.zeros((c["batch"], heads * c["group"], kept), device=DEV)
    s["held"] = torch.zeros(c["batch"], dtype=torch.int32, device=DEV)


def _calls(c, s):
    """The library's calls, as a program that runs them over and over prepares them."""
    from paper_2508_02751_amd import smallkv as S
    cache = _spec(c, s, s["from"])
    if c["kind"] == "evict":
        return [S.prepare_evict(cache, _spec(c, s, s["to"]), s["length"], s["keep"], s["before"],
                                recent=s["recent"], sinks=c["sinks"], out_pos=s["out_pos"],
                                out_scores=s["after"], held=s["held"])]
    calls = []
    if s["new"]:
        chunk = S.ChunkSpec(s["start"], s["length"], s["T"], s["new"], s["rows"])
    if c["kind"] in ("append", "read") and s["new"]:
        rope = S.RopeSpec(s["freq"], S.ROPE_HALF if c["layout"] == "half" else S.ROPE_INTERLEAVED)
        calls.append(S.prepare_append(chunk, cache, rope, s["q"], s["new_k"], s["new_v"],
                                      positions=s["pos"], q_out=s["q_out"]))
    if c["kind"] == "read":
        calls.append(S.prepare_read(cache, S.CacheSpec(s["out_k"], s["out_v"]), s["length"],
                                    begin=s["begin"]))
    if c["kind"] == "attn":
        calls.append(S.prepare_chunk_attn(chunk, cache, s["q"], s["scale"]))
    if c["kind"] == "scores":
        calls.append(S.prepare_chunk_scores(chunk, cache, s["q"], s["lse"], s["scale"], s["after"],
                                            before=s["before"]))
    return calls


# --------------------------------------------------------------- one pass --

def run(state):
    kind = state["c"]["kind"]
    if own:
        for call in state["calls"]:
            call.run()
        if kind == "attn":
            return {"out": state["calls"][0].out, "lse": state["calls"][0].lse}
    elif kind == "attn":
        return _plain_attn(state)
    else:
        {"append": _plain_append, "read": _plain_read, "scores": _plain_scores,
         "evict": _plain_evict}[kind](state)
    if kind == "append":
        return dict(_values(state["from"]), q=state["q_out"])
    if kind == "read":
        got = {"k": state["out_k"], "v": state["out_v"]}
        return dict(got, q=state["q_out"]) if state["new"] else got
    if kind == "scores":
        return {"scores": state["after"]}
    return dict(_values(state["to"]), pos=state["out_pos"], scores=state["after"], held=state["held"])


def _values(p):
    """Codes of 8 bits and their scales, as the numbers that they are."""
    return {"k": p["k"].view(torch.float8_e4m3fn), "v": p["v"].view(torch.float8_e4m3fn),
            "k_scale": p["k_scale"].view(torch.float8_e8m0fnu),
            "v_scale": p["v_scale"].view(torch.float8_e8m0fnu)}


def _power(e):
    """2^e in 64 bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _packed(x, fmt):
    """Codes and block scales of x [...][d] in 64 bits.  The scale is the smallest power of
    two, 2^-100 at least, with which the largest element is at most half a step above the
    format's largest value; elements round to the nearest, ties to even."""
    most, limit, least, bits = (448.0, 464.0, -6, 3) if fmt == "mxfp8" else (6.0, 7.0, 0, 1)
    b = x.view(*x.shape[:-1], -1, 32)
    mantissa, e = torch.frexp(b.abs().amax(-1, keepdim=True) / limit)
    e = torch.where(mantissa == 0.5, e - 1, e).clamp_min(-100)
    e = torch.where(mantissa == 0, torch.full_like(e, -100), e)
    y = b * _power(-e)
    size = y.abs().clamp_max(most)
    top = (torch.frexp(size)[1] - 1).clamp_min(least)
    steps = torch.round(size * _power(bits - top))
    code = ((top - least) << bits) + steps.long() + (torch.signbit(y).long() << (7 if fmt == "mxfp8" else 3))
    code = code.view(x.shape)
    if fmt == "mxfp4":
        code = code[..., 0::2] + (code[..., 1::2] << 4)
    return code.to(torch.uint8), (e.squeeze(-1) + 127).to(torch.uint8)


def _unpacked(codes, scales, fmt):
    """The values in 32 bits, which hold them exactly."""
    if fmt == "mxfp8":
        x = codes.contiguous().view(torch.float8_e4m3fn).float()
    else:
        x = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
        size = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=codes.device)
        x = size[(x & 7).int()] * (1.0 - (x >> 3).float() * 2.0)
    scale = (scales.int() << 23).view(torch.float32)
    return (x.view(*x.shape[:-1], -1, 32) * scale[..., None]).flatten(-2)


def _place(s, seq, row):
    """Pages and rows in them of the sequences' rows."""
    table, page = s["from"]["table"], s["c"]["page"]
    return (seq, row) if table is None else (table[seq, row // page].long(), row % page)


def _all_rows(s, codes, scales):
    """[batch][head][row][d] in 32 bits; a sequence's rows past its last are some others."""
    seq = torch.arange(s["c"]["batch"], device=DEV)[:, None]
    row = torch.minimum(torch.arange(s["rows"], device=DEV), s["length"].long()[:, None] - 1)
    page, at = _place(s, seq, row)
    x = _unpacked(codes[page, :, at], scales[page, :, at], s["c"]["format"])
    return x.transpose(1, 2).contiguous()


def _turn(x, cos, sin, rot, layout):
    y = x.clone()
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2),
                                                                              slice(1, rot, 2))
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., a] * sin + x[..., b] * cos
    return y


def _plain_append(s):
    c, p = s["c"], s["from"]
    angle = s["pos"].double()[:, None, None] * s["freq"]
    cos, sin = torch.cos(angle), torch.sin(angle)
    s["q_out"].copy_(_turn(s["q"].float(), cos.float(), sin.float(), c["rot"], c["layout"]))
    page, at = _place(s, s["seq"], s["row"])
    # (in 64 bits: a code goes by which side of a border the turned key is on)
    k = _packed(_turn(s["new_k"].double(), cos, sin, c["rot"], c["layout"]), c["format"])
    v = _packed(s["new_v"].double(), c["format"])
    p["k"][page, :, at], p["k_scale"][page, :, at] = k
    p["v"][page, :, at], p["v_scale"][page, :, at] = v


def _plain_read(s):
    p = s["from"]
    if s["new"]:
        _plain_append(s)
        page, at = _place(s, s["seq"], s["row"])
        for out, codes, scales in ((s["out_k"], p["k"], p["k_scale"]), (s["out_v"], p["v"], p["v_scale"])):
            x = _unpacked(codes[page, :, at], scales[page, :, at], s["c"]["format"])
            out[s["seq"], :, s["row"]] = x.to(out.dtype)
        return
    there = (torch.arange(s["rows"], device=DEV) < s["length"][:, None])[:, None, :, None]
    for out, codes, scales in ((s["out_k"], p["k"], p["k_scale"]), (s["out_v"], p["v"], p["v_scale"])):
        out.copy_(torch.where(there, _all_rows(s, codes, scales).to(out.dtype), out))


def _logits(s, k):
    """[batch][kv head][query head of it, number of the token][row]; rows that a token does
    not see at -inf.  Chunks shorter than the longest repeat some token."""
    B, hk, n, d = k.shape
    q = s["q"].float()[s["padded"]].view(B, s["new"], hk, -1, d).permute(0, 2, 3, 1, 4)
    g = q.shape[2]
    x = torch.matmul(q.reshape(B, hk, -1, d), k.transpose(2, 3).contiguous()).mul_(s["scale"])
    seen = torch.arange(n, device=DEV) <= s["padded_row"][:, :, None]
    x = x.view(B, hk, g, s["new"], n)
    return x.masked_fill_(~seen[:, None, None], -math.inf)


def _tokens(s, x):
    """[batch][kv head][query head of it][number][...] as packed [token][query head][...]."""
    x = x[s["seq"], :, :, s["number"]]
    return x.flatten(1, 2)


def _plain_attn(s, need_out=True):
    p = s["from"]
    x = _logits(s, _all_rows(s, p["k"], p["k_scale"]))
    m = x.amax(-1, keepdim=True)
    x = x.sub_(m).exp_()
    z = x.sum(-1, keepdim=True)
    got = {"lse": _tokens(s, (m + z.log()).squeeze(-1)).contiguous()}
    if need_out:
        B, hk, g, M, n = x.shape
        v = _all_rows(s, p["v"], p["v_scale"])
        there = torch.arange(n, device=DEV) < s["length"][:, None]
        v = v * there[:, None, :, None]
        o = torch.matmul(x.view(B, hk, g * M, n), v).view(B, hk, g, M, -1) / z
        got["out"] = _tokens(s, o).to(s["q"].dtype)
    return got


def _plain_scores(s):
    c, p = s["c"], s["from"]
    x = _logits(s, _all_rows(s, p["k"], p["k_scale"]))
    B, hk, g, M, n = x.shape
    lse = s["lse"][s["padded"]].view(B, M, hk, g).permute(0, 2, 3, 1)
    x = x.sub_(lse[..., None]).exp_()
    numbers = torch.arange(M, device=DEV) < (s["length"] - s["first"])[:, None]
    x = x.mul_(numbers[:, None, None, :, None])
    f = x.sum((2, 3)) if c["per_kv"] else x.sum(3).view(B, hk * g, n)
    row = torch.arange(n, device=DEV)
    f += torch.where(row < s["first"][:, None, None], s["before"], torch.zeros_like(s["before"]))
    s["after"].copy_(torch.where(row < s["length"][:, None, None], f, s["after"]))


def _plain_evict(s):
    c, to = s["c"], s["to"]
    B, H, g, n = c["batch"], s["heads"], c["group"], s["rows"]
    x = s["before"].view(B, H, g, n)
    f = x[:, :, 0]
    for i in range(1, g):
        f = f + x[:, :, i]  # (the order is part of what ranks the rows)
    row = torch.arange(n, device=DEV)
    length, kept = s["length"][:, None, None], s["keep"][:, None, None]
    last = torch.minimum(s["recent"][:, None, None], kept)
    first = (kept - last).clamp_max(c["sinks"])
    # rows that stay come first, then the others by score, then those that are not there
    f = torch.where((row < first) | (row >= length - last), torch.full_like(f, math.inf), f)
    f = torch.where(row < length, f, torch.full_like(f, -math.inf))
    rank = torch.sort(f, dim=2, descending=True, stable=True).indices
    place = torch.arange(n, device=DEV) < kept
    rows = torch.where(place, rank, torch.full_like(rank, n)).sort(2).values[..., : s["out_pos"].shape[2]]
    there = rows < n
    b, h, i = torch.nonzero(there, as_tuple=True)
    r = rows[b, h, i]
    page, at = _place(s, b, r)
    for name in ("k", "v", "k_scale", "v_scale"):
        to[name][b, h, i] = s["from"][name][page, h, at]
    s["out_pos"][b, h, i] = r.to(torch.int32)
    s["after"].view(B, H, g, -1)[b, h, :, i] = x[b, h, :, r]
    s["held"].copy_(s["keep"])


# -------------------------------------------------------------------- work --

def work(c):
    hq, hk, d = SHAPES[c["shape"]]
    e = 4 if c["dtype"] == "f32" else 2
    lens = lengths(c)
    T, rows = sum(m for _, m in lens), sum(n for n, _ in lens)
    packed = _row_bytes(c, d) + d // 32
    heads = hk * c.get("layers", 1)
    # a new token attends to the rows up to its own
    pairs = sum(m * (n - m) + m * (m + 1) // 2 for n, m in lens)
    append = {"bytes": T * (2 * hq + 2 * hk) * d * e + 2 * T * hk * packed + 4 * T,
              "flops": T * (3 * (hq + hk) * c.get("rot", 0) + 6 * hk * d)}
    if c["kind"] == "append":
        return append
    if c["kind"] == "read":
        if T:  # the new rows, packed and read back
            return {"bytes": append["bytes"] + 2 * T * hk * (packed + d * e),
                    "flops": append["flops"] + 2 * T * hk * d}
        return {"bytes": 2 * rows * heads * (packed + d * e), "flops": 2 * rows * heads * d}
    if c["kind"] == "attn":
        return {"bytes": 2 * rows * hk * packed + T * hq * (2 * d * e + 4), "flops": 4 * pairs * hq * d}
    if c["kind"] == "scores":
        n_scores = hk if c["per_kv"] else hq
        return {"bytes": rows * hk * packed + T * hq * (d * e + 4) + 4 * n_scores * (2 * rows - T),
                "flops": 2 * pairs * hq * d}
    kept = sum(max(1, n * c["keep"] // 100) for n, _ in lens)
    return {"bytes": heads * (4 * c["group"] * rows + kept * (4 * packed + 4 + 4 * c["group"])),
            "flops": heads * c["group"] * rows}


# ------------------------------------------------------- the same in 64 bits --

def _table(fmt):
    """What every code stands for, from the bits of the format."""
    e_bits, m_bits, bias = (4, 3, 7) if fmt == "mxfp8" else (2, 1, 1)
    vals = []
    for code in range(1 << (1 + e_bits + m_bits)):
        m, e = code & ((1 << m_bits) - 1), (code >> m_bits) & ((1 << e_bits) - 1)
        x = (m / (1 << m_bits)) * 2.0 ** (1 - bias) if e == 0 else (1 + m / (1 << m_bits)) * 2.0 ** (e - bias)
        vals.append(-x if code >> (e_bits + m_bits) else x)
    if fmt == "mxfp8":
        vals[0x7F] = vals[0xFF] = math.nan
    return torch.tensor(vals, dtype=torch.float64, device=DEV)


def _nearest(x, fmt):
    """x [...][d] packed and read back: the block's power of two by trying them, each element
    the nearest of the format's values, of two as near the one with an even code."""
    vals = _table(fmt)[: 127 if fmt == "mxfp8" else 8]
    most = float(vals[-1] + (vals[-1] - vals[-2]) / 2)
    b = x.unflatten(-1, (-1, 32))
    size = b.abs().max(-1, keepdim=True).values
    e = torch.floor(torch.log2(size.clamp_min(1e-300) / most)).clamp_min(-100)
    for _ in range(2):
        e = torch.where(size > most * torch.exp2(e), e + 1, e)
    y = b.abs() / torch.exp2(e)
    hi = torch.searchsorted(vals, y.contiguous()).clamp(1, len(vals) - 1)
    lo = hi - 1
    up, down = vals[hi] - y, y - vals[lo]
    pick = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return torch.copysign(vals[pick], b).flatten(-2), torch.exp2(e).squeeze(-1)


def _decoded(codes, scales, fmt):
    t = _table(fmt)
    i = codes.int()
    x = t[i] if fmt == "mxfp8" else torch.stack([t[i % 16], t[i // 16]], -1).flatten(-2)
    return x * torch.exp2(scales.double() - 127.0).repeat_interleave(32, -1)


def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] == "evict":
        return _exact_evict(s)
    if c["kind"] in ("append", "read"):
        return _exact_rows(s)
    p, lens, q = s["from"], s["lens"], s["q"]
    hq, hk, d = SHAPES[c["shape"]]
    g = hq // hk
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(q.shape[:2], dtype=torch.float64, device=DEV)
    acc = torch.zeros(s["after"].shape, dtype=torch.float64, device=DEV) if c["kind"] == "scores" else None
    t0 = 0
    for b, (n, new) in enumerate(lens):
        r = torch.arange(n, device=DEV)
        page, at = (r * 0 + b, r) if p["table"] is None else (p["table"][b].long()[r // c["page"]],
                                                              r % c["page"])
        limit = max(1, (1 << 27) // (n * g))
        for h in range(hk):
            K = _decoded(p["k"][page, h, at], p["k_scale"][page, h, at], c["format"])
            V = _decoded(p["v"][page, h, at], p["v_scale"][page, h, at], c["format"])
            per_head = torch.zeros((g, n), dtype=torch.float64, device=DEV)
            for i in range(0, new, limit):
                j = slice(t0 + i, t0 + min(i + limit, new))
                m = j.stop - j.start
                hs = slice(h * g, h * g + g)
                x = (q[j, hs].double().reshape(m * g, d) @ K.t().contiguous()).view(m, g, n) * s["scale"]
                blind = r[None, :] > (n - new + i + torch.arange(m, device=DEV))[:, None]
                x.masked_fill_(blind[:, None], -math.inf)
                if c["kind"] == "attn":
                    lse[j, hs] = torch.logsumexp(x, -1)
                    out[j, hs] = (torch.softmax(x, -1).view(m * g, n) @ V).view(m, g, d)
                else:
                    per_head += torch.exp(x - s["lse"][j, hs].double()[..., None]).sum(0)
            if acc is not None:
                if c["per_kv"]:
                    acc[b, h, :n] = per_head.sum(0)
                else:
                    acc[b, h * g: h * g + g, :n] = per_head
        if acc is not None:
            acc[b, :, : n - new] += s["before"][b, :, : n - new].double()
        t0 += new
    return {"out": out, "lse": lse} if c["kind"] == "attn" else {"scores": acc}


def _exact_rows(s):
    c, p, rot = s["c"], s["from"], s["c"]["rot"]
    got = {}
    if c["kind"] == "append":
        t = _table("mxfp8")
        got = {x: t[p[x].int()] for x in ("k", "v")}
        got.update({x: torch.exp2(p[x].double() - 127.0) for x in ("k_scale", "v_scale")})
    else:
        got = {"k": s["out_k"].double(), "v": s["out_v"].double()}
    if s["new"]:
        th = s["pos"].double().unsqueeze(1) * s["freq"].unsqueeze(0)
        turn = torch.polar(torch.ones_like(th), th).unsqueeze(1)

        def turned(x):
            x = x.double()
            head = x[..., :rot]
            if c["layout"] == "half":
                z = torch.complex(head[..., : rot // 2].contiguous(), head[..., rot // 2:].contiguous()) * turn
                head = torch.cat([z.real, z.imag], -1)
            else:
                z = torch.view_as_complex(head.reshape(*head.shape[:-1], rot // 2, 2).contiguous()) * turn
                head = torch.view_as_real(z).flatten(-2)
            return torch.cat([head, x[..., rot:]], -1)

        got["q"] = turned(s["q"])
        for name, x in (("k", turned(s["new_k"])), ("v", s["new_v"].double())):
            y, scale = _nearest(x, c["format"])
            t0 = 0
            for b, (n, new) in enumerate(s["lens"]):
                r = torch.arange(n - new, n, device=DEV)
                if c["kind"] == "read":
                    z = y[t0: t0 + new] * scale[t0: t0 + new].repeat_interleave(32, -1)
                    got[name][b, :, r] = z.transpose(0, 1)
                else:
                    page = p["table"][b].long()[r // c["page"]] if c["page"] else r * 0 + b
                    at = r % c["page"] if c["page"] else r
                    got[name][page, :, at] = y[t0: t0 + new]
                    got[name + "_scale"][page, :, at] = scale[t0: t0 + new]
                t0 += new
        return got
    for b, (n, _) in enumerate(s["lens"]):
        r = torch.arange(n, device=DEV)
        page, at = (r * 0 + b, r) if p["table"] is None else (p["table"][b].long()[r // c["page"]],
                                                              r % c["page"])
        for h in range(s["heads"]):
            for name in ("k", "v"):
                got[name][b, h, :n] = _decoded(p[name][page, h, at], p[name + "_scale"][page, h, at],
                                               c["format"])
    return got


def _exact_evict(s):
    """Moved values: the rows by their rank, counted instead of sorted (None
    where that takes long)."""
    c, p, to, H = s["c"], s["from"], s["to"], s["heads"]
    if sum(H * n * n for n, _ in s["lens"]) > 1 << 40:
        return None
    t = _table("mxfp8")
    got = {x: t[to[x].int()] for x in ("k", "v")}
    got.update({x: torch.exp2(to[x].double() - 127.0) for x in ("k_scale", "v_scale")})
    got.update(pos=s["out_pos"].clone(), scores=s["after"].double(), held=s["held"].clone())
    g = c["group"]
    for b, ((n, _), (keep, recent)) in enumerate(zip(s["lens"], s["budgets"])):
        kept = min(keep, n)
        last = min(recent, kept)
        first = min(c["sinks"], kept - last)
        idx = torch.arange(n, device=DEV)
        for h in range(H):
            f = s["before"][b, h * g, :n].clone()
            for i in range(1, g):
                f += s["before"][b, h * g + i, :n]  # in 32 bits: the sum that ranks the rows is defined so
            f[(idx < first) | (idx >= n - last)] = math.inf
            rank = torch.zeros(n, dtype=torch.int64, device=DEV)
            for j in range(0, n, 4096):
                o, oi = f[j: j + 4096, None], idx[j: j + 4096, None]
                rank += ((o > f) | ((o == f) & (oi < idx))).sum(0)
            rows = idx[rank < kept]
            page, at = (rows * 0 + b, rows) if p["table"] is None else (
                p["table"][b].long()[rows // c["page"]], rows % c["page"])
            for name in ("k", "v"):
                got[name][b, h, :kept] = t[p[name][page, h, at].int()]
                name += "_scale"
                got[name][b, h, :kept] = torch.exp2(p[name][page, h, at].double() - 127.0)
            got["pos"][b, h, :kept] = rows.to(torch.int32)
            got["scores"][b, h * g: h * g + g, :kept] = s["before"][b, h * g: h * g + g, rows].double()
        got["held"][b] = kept
    return got
