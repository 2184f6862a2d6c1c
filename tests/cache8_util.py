"""Inputs and float64 definitions of the 8-bit cache and of attention over a shared past (shared by their tests)."""
from __future__ import annotations

import math

import torch

from tests import cache_util as cu

# values of the e4m3 codes 0 .. 126 from their bits: 4 exponent bits of bias 7, 3 of the mantissa (127 is NaN)
CODES = [(8 + c % 8) * 2.0 ** (c // 8 - 10) if c >= 8 else c * 2.0 ** -9 for c in range(127)]


def quantised64(x):
    """Codes [..., hd] and exponent bytes [...] of heads x float64: the smallest exponent from -117 on that keeps the finite
    elements within 448, the nearest code (the even one of two); beyond 240 * 2^120 that value."""
    size = torch.where(torch.isfinite(x), x.abs(), 0).amax(-1)
    e = torch.full_like(size, -117)
    for step in range(-117, 121):
        e = torch.where(size > 448.0 * 2.0 ** step, step + 1.0, e)
    y = x * torch.exp2(-e)[..., None]
    top = torch.where(e == 120, 240.0, 448.0)[..., None]
    y = torch.where(torch.isfinite(x), torch.minimum(torch.maximum(y, -top), top), y)
    table = torch.tensor(CODES, dtype=torch.float64, device=x.device)
    mid = (table[1:] + table[:-1]) / 2
    at = torch.searchsorted(mid, y.abs().contiguous())           # midpoints below |y|
    tie = (at < 126) & (mid[at.clamp(max=125)] == y.abs())
    at = torch.where(tie & (at % 2 == 1), at + 1, at)
    code = torch.where(torch.isfinite(x), at + 128 * torch.signbit(x), 127)
    return code.to(torch.uint8), (e + 127).to(torch.uint8)


def values64(codes, byte):
    """What codes (uint8) and exponent bytes stand for."""
    table = torch.tensor(CODES + [math.nan], dtype=torch.float64, device=codes.device)
    x = table[(codes & 127).long()] * torch.where(codes >= 128, -1.0, 1.0)
    return x * torch.exp2(byte.double() - 127)[..., None]


def state8(dtype="bf16", *args, spread=0.7, **kw):
    """cache_util.state with the cache in codes (k8, v8, scale), and k and v as their values. Rows differ in size. Free
    slots hold NaN codes with the largest exponent byte."""
    s = cu.state(dtype, *args, **kw)
    g = torch.Generator().manual_seed(kw.get("seed", 0) + 1000)
    size = torch.exp(spread * torch.randn(s.mass.shape, generator=g)).to(s.k.device)[..., None]
    encode(s, s.k.double() * size, s.v.double() * size.flip(2))
    return s


def encode(s, k, v):
    """Puts float64 pools (NaN: free) into the state as codes."""
    free = torch.isnan(k).all(-1)
    (k8, ke), (v8, ve) = quantised64(k), quantised64(v)
    s.scale = torch.where(free[..., None], 255, torch.stack([ke, ve], -1)).to(torch.uint8).contiguous()
    s.k8, s.v8 = (torch.where(free[..., None], 127, x).to(torch.uint8).contiguous().view(torch.float8_e4m3fn) for x in (k8, v8))
    decode(s)


def decode(s):
    """The state's k and v: the values of its codes (exact in either type)."""
    s.k = values64(s.k8.view(torch.uint8), s.scale[..., 0]).to(s.td)
    s.v = values64(s.v8.view(torch.uint8), s.scale[..., 1]).to(s.td)


def cache8(wdc, s):
    return wdc.PagedCache8(s.k8, s.v8, s.scale)


class Past:
    """Groups of sequences of a state and their prefixes, as a call takes them and as the definition does."""

    def __init__(self, s, sizes, prefix, device="cuda:0"):
        self.first = [sum(sizes[:g]) for g in range(len(sizes) + 1)]
        self.sizes, self.prefix = list(sizes), list(prefix)
        self.group_start = torch.tensor(self.first, dtype=torch.int32, device=device)
        self.prefix_len = torch.tensor(self.prefix, dtype=torch.int32, device=device)
        self.keys, self.lead = [0] * len(s.kv), list(range(len(s.kv)))
        for g, p in enumerate(self.prefix):
            for b in range(self.first[g], self.first[g + 1]):
                self.lead[b] = self.first[g]
                self.keys[b] = min(p, s.kv[self.first[g]]) // s.page * s.page

    def desc(self, wdc, s, **kw):
        args = dict(max_prefix=max(self.prefix), max_own=max(max(n - p for n, p in zip(s.kv, self.keys)), 0))
        args.update(kw)
        return wdc.Prefix(self.group_start, self.prefix_len, **args)


def attention64(s, frame, past=None):
    """As cache_util.attention64, over the state's k and v: o, lse, sum p |v| and the largest sum |q k| / sqrt(hd). With a
    past the first keys of a group's sequences are those of its first one, and seen by all of its rows."""
    dev = s.k.device
    o = torch.zeros((s.rows, s.heads, s.hd), dtype=torch.float64, device=dev)
    lse = torch.full((s.rows, s.heads), -math.inf, dtype=torch.float64, device=dev)
    pv, qk = torch.zeros_like(o), torch.zeros_like(lse)
    grp, first = s.heads // s.kvh, 0
    for b, q in enumerate(s.q):
        p = past.keys[b] if past else 0
        pg, sl = cu.where(s, b)
        if past:
            lpg, lsl = cu.where(s, past.lead[b])
            pg, sl = torch.cat([lpg[:p], pg[p:]]), torch.cat([lsl[:p], sl[p:]])
        lim = cu.limits(s, b, frame).clamp(min=p)
        hidden = torch.arange(len(pg), device=dev) >= lim[:, None]
        for h in range(s.heads if q and len(pg) else 0):
            k, v = s.k[pg, h // grp, sl].double(), s.v[pg, h // grp, sl].double()
            x = s.x[first:first + q, h * s.hd:(h + 1) * s.hd].double()
            sc = (x @ k.T / math.sqrt(s.hd)).masked_fill(hidden, -math.inf)
            z = torch.logsumexp(sc, 1)
            w = torch.where(hidden, 0, torch.exp(sc - torch.where(z == -math.inf, 0, z)[:, None]))
            lse[first:first + q, h] = z
            # values of NaN count where they are seen, and only there
            nan = torch.isnan(v)
            bad = (~hidden).double() @ nan.double() > 0
            v = torch.where(nan, 0, v)
            o[first:first + q, h] = torch.where(bad, math.nan, w @ v)
            pv[first:first + q, h] = w @ v.abs()
            qk[first:first + q, h] = (x.abs() @ k.abs().T / math.sqrt(s.hd)).masked_fill(hidden, 0).nan_to_num(0, 0, 0).amax(1)
        first += q
    return o, lse, pv, qk
