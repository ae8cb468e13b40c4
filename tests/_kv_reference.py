"""The paged 8-bit cache in 64 bits, from the definitions: lookup, rotation, quantisation, attention, with the bounds that the
kernels' roundings allow.  Everything on the host, sequence by sequence."""
import math

import torch

NAN_CODES = (0x7F, 0xFF)


def decode(codes):
    """e4m3 codes (uint8) -> float64."""
    c = codes.to(torch.int64)
    sign, e, m = torch.where(c >= 128, -1.0, 1.0).double(), (c >> 3) & 15, (c & 7).double()
    x = torch.where(e == 0, m * 2.0 ** -9, (8 + m) * torch.pow(2.0, (e - 10).double()))
    return sign * torch.where((c & 127) == 127, math.nan, x)


_VALUES = decode(torch.arange(127, dtype=torch.uint8))


def encode(x):
    """float64 -> e4m3 codes: nearest, ties to the even code, what is too large saturates, NaN stays NaN."""
    a = x.abs().clamp(max=448.0)
    hi = torch.searchsorted(_VALUES, a.nan_to_num(0.0).contiguous()).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    below, above = a - _VALUES[lo], _VALUES[hi] - a
    code = torch.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    code = torch.where(x.isnan(), 127, code)
    return (code + 128 * torch.signbit(x)).to(torch.uint8)


def scale_for(amax):
    """The smallest 2^e >= amax / 448, 2^-64 <= 2^e <= 2^64."""
    if amax == 0:
        return 2.0 ** -64
    e = math.frexp(amax / 448)[1]
    while e > -80 and amax <= 448 * 2.0 ** (e - 1):
        e -= 1
    return 2.0 ** max(-64, min(64, e))


def rotate(x, pos, inv_freq, interleaved):
    """x [n, heads, dim] float64 at positions pos [n]."""
    if inv_freq is None:
        return x
    angle = pos.double()[:, None] * inv_freq.double()[None]
    c, s, r = angle.cos()[:, None], angle.sin()[:, None], 2 * inv_freq.numel()
    y = x.clone()
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., :r // 2], x[..., r // 2:r])
    ya, yb = a * c - b * s, b * c + a * s
    if interleaved:
        y[..., 0:r:2], y[..., 1:r:2] = ya, yb
    else:
        y[..., :r // 2], y[..., r // 2:r] = ya, yb
    return y


class Pool:
    """A cache on the host: codes [pages, heads, page, dim] uint8, scales [pages, heads] fp32."""

    def __init__(self, pages, heads, page, dim, gen):
        x = torch.randn(pages, heads, page, dim, generator=gen, dtype=torch.float64)
        self.k, self.v = encode(x * 100), encode(torch.randn(pages, heads, page, dim, generator=gen, dtype=torch.float64) * 100)
        self.k_scale = torch.pow(2.0, torch.randint(-8, -5, (pages, heads), generator=gen).float())
        self.v_scale = torch.pow(2.0, torch.randint(-9, -4, (pages, heads), generator=gen).float())
        self.page = page

    def sequence(self, which, table_row, length):
        """values [heads, length, dim] float64 of one sequence."""
        codes, scale = (self.k, self.k_scale) if which == "k" else (self.v, self.v_scale)
        ids = table_row[:-(-length // self.page)].long()
        x = decode(codes[ids]) * scale[ids].double()[..., None, None]
        return x.transpose(0, 1).reshape(codes.shape[1], -1, codes.shape[3])[:, :length]

    def cuda(self, M, fp8=True):
        t = torch.float8_e4m3fn if fp8 else torch.uint8
        return M.KVCache(self.k.cuda().view(t), self.v.cuda().view(t), self.k_scale.cuda(), self.v_scale.cuda())


def tables(lens, page, gen, spare=2):
    """Page table int32 [B, width] over a pool in random order, and the number of pages."""
    need = [-(-n // page) for n in lens]
    total = sum(need) + spare
    order = torch.randperm(total, generator=gen).to(torch.int32)
    table = torch.full((len(lens), max(need + [1])), -7, dtype=torch.int32)       # (what is behind a sequence's end is not read)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, total


def offsets(new):
    return torch.tensor([0] + list(new)).cumsum(0).to(torch.int32)


def attend(q, pool, table, new, lens, scale, causal, window, terms=1):
    """(out, lse, bound of out's error before its last rounding, bound of lse's) of all rows, float64, q [N, heads, dim].

    Errors counted (u = 2^-24; tensor cores may truncate, so 2u an addition): a score is off by d = (dim + 8) 2u scale sum |q k| (q in
    11 * terms bits: for two terms 2u sum |q k| more, inside the 8) and by the rounding of its exponent, |s| up to 2^7: 2^-17; exp2 and the
    block scales' logarithms 2^-20; a weight is rounded to 11 * terms bits, and below 2^-14 to steps of 2^-24 where a row's largest is
    2^7 or more; sums of L terms are off by L 2u."""
    out, lse, eo, el = [], [], [], []
    at = 0
    for b, (n, l) in enumerate(zip(new, lens)):
        if n == 0:
            continue
        x = q[at:at + n].double()
        at += n
        k, v = pool.sequence("k", table[b], l), pool.sequence("v", table[b], l)
        group = q.shape[1] // k.shape[0]
        k, v = k.repeat_interleave(group, 0), v.repeat_interleave(group, 0)
        pos, key = torch.arange(l - n, l)[:, None], torch.arange(l)[None]
        seen = torch.ones(n, l, dtype=torch.bool)
        if causal:
            seen &= key <= pos
        if window:
            seen &= key > pos - window
        s = torch.einsum("nhd,hld->hnl", x, k) * scale
        s = s.masked_fill(~seen[None], -math.inf)
        z = torch.logsumexp(s, -1) if l else torch.full((q.shape[1], n), -math.inf, dtype=torch.float64)
        p = torch.where(seen[None], torch.exp(s - z[..., None]), 0.0)
        vv = torch.where(torch.isnan(v), 0.0, v)
        o = torch.einsum("hnl,hld->hnd", p, vv)
        pv = torch.einsum("hnl,hld->hnd", p, vv.abs())
        u2 = 2.0 ** -23
        d = ((q.shape[2] + 8) * u2 * scale * torch.einsum("nhd,hld->hnl", x.abs(), k.abs()).masked_fill(~seen[None], 0)).amax(-1) if l else torch.zeros_like(z)
        rel = (2 * d + 2.0 ** -16 + l * u2 * 2)[..., None]
        tiny = l * 2.0 ** -32 * 448 * (p.amax(-1, keepdim=True) if l else 0.0) * (float(pool.v_scale.max()) if terms == 1 else 0.0)
        eo.append(((2.0 ** (-11 * terms) + rel) * pv + rel * o.abs() + tiny).transpose(0, 1))
        el.append((d + l * u2 + 2.0 ** -16 + z.nan_to_num(0, 0, 0).abs() * 2.0 ** -22).transpose(0, 1))
        out.append(o.transpose(0, 1))
        lse.append(z.transpose(0, 1))
    return torch.cat(out), torch.cat(lse), torch.cat(eo), torch.cat(el)
