"""Plain 64-bit forms of the cache operators and the bounds on what the kernels
may differ by, for the tests of them.  Half a unit in the last place: HALF."""
import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
U = 2.0 ** -24  # of fp32 arithmetic


class Case:
    """A cache and a batch of new tokens on `device`.  lens: (cached rows, new
    tokens) per sequence; rows that belong to nobody hold NaN.  page 0: dense."""

    def __init__(self, lens, hq, hk, d, dtype, page=0, rows_first=False, seed=0, extra_tokens=0,
                 device="cpu", cap=None, gap=0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.hq, self.hk, self.d, self.dtype, self.page = lens, hq, hk, d, dtype, page
        self.B = len(lens)
        rows = max(max(n for n, _ in lens), 1) + gap if cap is None else cap
        per = page or rows
        width = (rows + per - 1) // per
        pages = self.B * width + (2 if page else 0)
        shape = (pages, per, hk, d) if rows_first else (pages, hk, per, d)
        self.table = None
        if page:
            self.table = torch.randperm(pages, generator=g)[: self.B * width].view(self.B, width).int()
        self.rows = rows
        pools = []
        for _ in range(2):
            t = torch.full(shape, math.nan).to(dtype)
            t = t.transpose(1, 2) if rows_first else t
            for b, (n, _) in enumerate(lens):
                for r in range(min(max(n, 0), rows)):
                    p, i = self.slot(b, r)
                    t[p, :, i] = torch.randn(hk, d, generator=g).to(dtype)
            pools.append(t)
        self.k, self.v = pools
        starts = [0]
        for _, new in lens:
            starts.append(starts[-1] + new)
        self.starts, self.T = starts, starts[-1] + extra_tokens
        self.q = torch.randn(max(self.T, 1), hq, d, generator=g).to(dtype)[: self.T]
        self.gen = g
        self.max_new = max([new for _, new in lens] + [1])
        self.scale = 1.0 / math.sqrt(d)

    def slot(self, b, r):
        if self.table is None:
            return b, r
        return int(self.table[b, r // self.page]), r % self.page

    def to(self, device):
        """(ChunkSpec, CacheSpec, q) on the device; the originals stay."""
        from paper_2508_02751_amd import smallkv as S
        start = torch.tensor(self.starts, dtype=torch.int32, device=device)
        length = torch.tensor([n for n, _ in self.lens], dtype=torch.int32, device=device)
        chunk = S.ChunkSpec(start, length, self.T, self.max_new, self.rows)

        def dev(t):  # strides kept
            return t.transpose(1, 2).contiguous().to(device).transpose(1, 2) \
                if not t.is_contiguous() else t.to(device)
        cache = S.CacheSpec(dev(self.k), dev(self.v),
                            None if self.table is None else self.table.to(device))
        return chunk, cache, self.q.to(device)

    def gather(self, pool, b, n):
        """[hk][n][d] in 64 bits and which rows exist."""
        out = torch.zeros(self.hk, n, self.d, dtype=torch.float64)
        have = torch.zeros(n, dtype=torch.bool)
        for r in range(n):
            p, i = self.slot(b, r)
            if 0 <= p < pool.shape[0]:
                out[:, r] = pool[p, :, i].double()
                have[r] = True
        return out, have


def logits(c, b):
    """Per kv head h and query head j of its group: [hk][g][new][n] logits (-inf:
    not seen) and the bound on the fp32 logit's error."""
    n, new = c.lens[b]
    k, have = c.gather(c.k, b, max(n, 0))
    g = c.hq // c.hk
    q = c.q[c.starts[b]: c.starts[b] + new].double().view(new, c.hk, g, c.d).permute(1, 2, 0, 3)
    x = torch.einsum("hgnd,hrd->hgnr", q, k) * c.scale
    size = torch.einsum("hgnd,hrd->hgnr", q.abs(), torch.nan_to_num(k).abs()) * c.scale
    own = max(n, 0) - new + torch.arange(new)
    if n < 0:
        own = n - new + torch.arange(new)
    seen = (torch.arange(max(n, 0))[None, :] <= own[:, None]) & have[None, :]
    x = torch.where(seen, x, torch.tensor(-math.inf, dtype=torch.float64))
    # d products and sums, and the factors scale and log2(e) on the way to exp2
    return x, torch.where(seen, size, torch.zeros(())).nan_to_num() * (c.d + 4) * U


def attention(c):
    """out, lse in 64 bits and their bounds, [T][hq](...)."""
    out = torch.zeros(c.T, c.hq, c.d, dtype=torch.float64)
    lse = torch.full((c.T, c.hq), -math.inf, dtype=torch.float64)
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    for b, (n, new) in enumerate(c.lens):
        if new == 0 or n <= 0:
            continue
        i = slice(c.starts[b], c.starts[b] + new)
        x, dx = logits(c, b)
        v, _ = c.gather(c.v, b, n)
        e = torch.logsumexp(x, -1)
        p = torch.exp(x - torch.where(torch.isinf(e), torch.zeros(()).double(), e)[..., None])
        g = c.hq // c.hk

        def flat(t):  # [hk][g][new]... -> [new][hq]...
            return t.movedim(2, 0).reshape(new, c.hq, *t.shape[3:])
        # a key whose weight is 0 contributes nothing, whatever its values
        o = torch.zeros(c.hk, g, new, c.d, dtype=torch.float64)
        a = torch.zeros_like(o)
        for r in range(n) if not torch.isfinite(v).all() else []:
            w = p[..., r][..., None]
            o += torch.where(w > 0, w * v[:, r][:, None, None], torch.zeros(()).double())
        if torch.isfinite(v).all():
            o = torch.einsum("hgnr,hrd->hgnd", p, v)
        a = torch.einsum("hgnr,hrd->hgnd", p, torch.nan_to_num(v, 0.0, 0.0, 0.0).abs())
        d = dx.amax(-1)
        # each weight: its logit's error twice (the reference point's too), the
        # exponential; sums over n keys
        rel = 2 * d + (n + 64) * U
        out[i], lse[i] = flat(o), flat(e)
        h = HALF[c.dtype]
        t = a * rel[..., None]
        if c.dtype == torch.bfloat16:
            t = t + 1.01 * h * (a + o.abs().nan_to_num())  # P's rounding and the output's
        else:
            t = t + h * o.abs().nan_to_num()
        tol[i] = flat(t)
        ltol[i] = flat(d + (n + 64) * U + 8 * U * e.abs().nan_to_num(0, 0, 0) + 8 * U)
    return out, lse, tol, ltol


def scores(c, lse, before, per_kv):
    """Scores in 64 bits and their bound; lse [T][hq] as given to the kernel."""
    g = c.hq // c.hk
    out, tol = before.double().clone(), torch.zeros(before.shape, dtype=torch.float64)
    for b, (n, new) in enumerate(c.lens):
        if n <= 0:
            continue
        out[b, :, max(n - new, 0): n] = 0.0
        if new == 0:
            continue
        x, dx = logits(c, b)
        e = lse[c.starts[b]: c.starts[b] + new].double().view(new, c.hk, g).permute(1, 2, 0)[..., None]
        dead = torch.isinf(e)
        p = torch.where(dead | torch.isinf(x), torch.zeros(()).double(), torch.exp(x - torch.where(dead, 0.0, e)))
        # the exponent's products and differences round at the size of logit and lse
        arg = (torch.where(torch.isinf(x), 0.0, x).abs() + torch.where(dead, 0.0, e).abs() + 1) * 4 * U
        w = p * (dx + arg + 4 * U + (new * g + 64) * U)
        s, t = p.sum(2), w.sum(2)
        if per_kv:
            s, t = s.sum(1), t.sum(1)
        out[b, :, :n] += s.reshape(-1, n)
        tol[b, :, :n] = t.reshape(-1, n) + 2 * U * out[b, :, :n].abs()
    return out, tol


def turned(x, angle, amp, rot, interleaved):
    """x [T][heads][d] in 64 bits, angle [T][rot/2]; and the bound's scale."""
    x = x.double()
    y, size = x.clone(), torch.zeros_like(x)
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    a = slice(0, rot, 2) if interleaved else slice(0, rot // 2)
    b = slice(1, rot, 2) if interleaved else slice(rot // 2, rot)
    u, v = x[..., a], x[..., b]
    y[..., a], y[..., b] = amp * (u * cos - v * sin), amp * (u * sin + v * cos)
    size[..., a] = size[..., b] = abs(amp) * (u.abs() + v.abs())
    return y, size


def kept_rows(f, n, keep, recent, sinks, cap):
    """Ascending kept rows of the scores f (fp32, [n])."""
    kept = min(max(keep, 0), n, cap)
    last = min(max(recent, 0), kept)
    first = min(sinks, kept - last)
    order = sorted(range(first, n - last),
                   key=lambda r: (1, 0.0, r) if math.isnan(f[r]) else (0, -float(f[r]) + 0.0, r))
    return sorted(list(range(first)) + list(range(n - last, n)) + order[: kept - last - first])
