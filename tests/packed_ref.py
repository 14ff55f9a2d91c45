"""Plain 64-bit forms of packed rows for the tests of the packed cache: what codes stand
for, and how a block is packed, from the formats' definition; and cases over packed
caches."""
import math

import torch

import cache_ref as R

MXFP8, MXFP4 = 0, 1


def code_values(fmt):
    e_bits, m_bits, bias = (4, 3, 7) if fmt == MXFP8 else (2, 1, 1)
    got = []
    for c in range(1 << (1 + e_bits + m_bits)):
        m, e = c % (1 << m_bits), (c >> m_bits) % (1 << e_bits)
        x = math.ldexp(m, 1 - bias - m_bits) if e == 0 else math.ldexp(m + (1 << m_bits), e - bias - m_bits)
        got.append(-x if c >> (e_bits + m_bits) else x)
    if fmt == MXFP8:
        got[0x7F] = got[0xFF] = math.nan
    return torch.tensor(got, dtype=torch.float64)


def pack(x, fmt):
    """(codes [...][d or d / 2], scales [...][d / 32]) of x [...][d], uint8."""
    vals = code_values(fmt)[: 127 if fmt == MXFP8 else 8]
    limit, lo, hi = (464.0, -100, 119) if fmt == MXFP8 else (7.0, -100, 125)
    b = x.double().reshape(*x.shape[:-1], -1, 32)
    bad = ~torch.isfinite(b).all(-1, keepdim=True)
    size = torch.where(bad, torch.zeros(()).double(), b.abs()).amax(-1, keepdim=True)
    e = torch.full_like(size, lo)
    for k in range(lo, hi):  # the smallest power of two that is large enough
        e = torch.where((e == k) & (size > limit * 2.0 ** k), e + 1, e)
    y = torch.where(bad, torch.zeros(()).double(), b) * 2.0 ** -e
    mag = y.abs().clamp_max(float(vals[-1]))
    up = torch.searchsorted(vals, mag.contiguous()).clamp(1, len(vals) - 1)
    down = up - 1
    a, c = vals[up] - mag, mag - vals[down]
    code = torch.where((a < c) | ((a == c) & (up % 2 == 0)), up, down)
    code = code + torch.where(torch.signbit(y), 128 if fmt == MXFP8 else 8, 0)
    code = torch.where(bad, torch.zeros((), dtype=code.dtype), code).reshape(x.shape)
    if fmt == MXFP4:
        code = code[..., 0::2] + 16 * code[..., 1::2]
    scale = torch.where(bad, torch.full_like(e, 255.0), e + 127)
    return code.to(torch.uint8), scale.squeeze(-1).to(torch.uint8)


def unpack(codes, scales, fmt):
    """The values in 64 bits."""
    t, i = code_values(fmt), codes.long()
    x = t[i] if fmt == MXFP8 else torch.stack([t[i % 16], t[i // 16]], -1).flatten(-2)
    s = scales.double()
    s = torch.where(s == 255, torch.full_like(s, math.nan), torch.exp2(s - 127))
    return x * s.repeat_interleave(32, -1)


class Case(R.Case):
    """A packed cache and a batch of new tokens: R.Case packed, its k and v what the codes stand
    for (so that the plain forms of cache_ref are what the operators compute).  Rows that
    belong to nobody are NaN blocks."""

    def __init__(self, lens, hq, hk, d, dtype, fmt, *args, outliers=False, **kw):
        super().__init__(lens, hq, hk, d, dtype, *args, **kw)
        self.fmt = fmt
        if outliers:
            self.k[..., :: d // 4] *= 6
        self.pack()

    def pack(self):
        self.codes = [*pack(self.k, self.fmt), *pack(self.v, self.fmt)]
        self.refresh()

    def refresh(self):
        kc, ks, vc, vs = self.codes
        self.k = unpack(kc, ks, self.fmt).to(self.dtype)
        self.v = unpack(vc, vs, self.fmt).to(self.dtype)

    def to(self, device):
        from paper_2508_02751_amd import smallkv as S
        start = torch.tensor(self.starts, dtype=torch.int32, device=device)
        length = torch.tensor([n for n, _ in self.lens], dtype=torch.int32, device=device)
        chunk = S.ChunkSpec(start, length, self.T, self.max_new, self.rows)
        flipped = self.flipped

        def dev(t):
            return t.transpose(1, 2).contiguous().to(device).transpose(1, 2) if flipped else t.contiguous().to(device)
        kc, ks, vc, vs = map(dev, self.codes)
        cache = S.PackedSpec(kc, vc, ks, vs, self.fmt, None if self.table is None else self.table.to(device))
        return chunk, cache, self.q.to(device)

    @property
    def flipped(self):
        """Whether pages hold [row][head]."""
        return self._flipped

    def __setattr__(self, name, value):
        if name == "k" and "_flipped" not in self.__dict__:
            self.__dict__["_flipped"] = not value.is_contiguous()
        object.__setattr__(self, name, value)
