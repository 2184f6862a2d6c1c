"""Inputs and float64 definitions of the paged cache operators (shared by their tests)."""
from __future__ import annotations

import math
from types import SimpleNamespace

import torch

ROPE = {64: (16, 24, 24), 128: (16, 56, 56)}


def config(dtype="bf16", heads=4, hd=64, qk_norm=True, rope=None):
    """A context configuration that describes an attention shape only (no blocks)."""
    return SimpleNamespace(name="cache", dtype=dtype, hidden=heads * hd, heads=heads, head_dim=hd, mlp_ratio=4, n_seq=0,
                           n_dual=0, n_single=0, cond_dim=0, cam_dim=0, text_tokens=0, text_dim=0, latent=(16, 1, 2, 2),
                           patch=(1, 2, 2), rope=ROPE[hd] if rope is None else rope, qk_norm=qk_norm, n_video=1)


def state(dtype="bf16", heads=4, kvh=4, hd=64, page=64, q=(1,), kv=(1,), seed=0, device="cuda:0", spare=3, tail_rows=0,
          fill=math.nan, scale=1.0):
    """A cache whose free slots and pages hold ``fill``, shuffled page tables (-1 past the end) and random rows."""
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator().manual_seed(seed)
    need = [-(-n // page) for n in kv]
    pages = sum(need) + spare
    order = torch.randperm(pages, generator=g)
    width = max(1, max(need))
    table = torch.full((len(kv), width), -1, dtype=torch.int32)
    k = torch.full((pages, kvh, page, hd), fill)
    v = torch.full((pages, kvh, page, hd), fill)
    mass = torch.full((pages, kvh, page), fill)
    at = 0
    for b, n in enumerate(kv):
        table[b, :need[b]] = order[at:at + need[b]].to(torch.int32)
        at += need[b]
        for j0 in range(0, n, page):
            m = min(page, n - j0)
            p = int(table[b, j0 // page])
            k[p, :, :m] = scale * torch.randn((kvh, m, hd), generator=g)
            v[p, :, :m] = torch.randn((kvh, m, hd), generator=g)
            mass[p, :, :m] = torch.exp(torch.randn((kvh, m), generator=g))
    rows = sum(q) + tail_rows
    s = SimpleNamespace(dtype=dtype, td=td, heads=heads, kvh=kvh, hd=hd, page=page, q=list(q), kv=list(kv), rows=rows,
                        pages=pages)
    s.table = table.to(device)
    s.q_start = torch.tensor([sum(q[:b]) for b in range(len(q) + 1)], dtype=torch.int32, device=device)
    s.kv_len = torch.tensor(list(kv), dtype=torch.int32, device=device)
    s.k, s.v, s.mass = k.to(td).to(device), v.to(td).to(device), mass.to(device)
    s.x = (scale * torch.randn((rows, heads * hd), generator=g)).to(td).to(device)
    s.qkv = torch.randn((rows, (heads + 2 * kvh) * hd), generator=g).to(td).to(device)
    return s


def chunks(wdc, s, **kw):
    args = dict(rows=s.rows, max_q=max(s.q), max_kv=max(s.kv))
    args.update(kw)
    return wdc.Chunks(s.q_start, s.kv_len, s.table, **args)


def where(s, b):
    """(pages, slots) of sequence b's keys."""
    j = torch.arange(s.kv[b], device=s.k.device)
    return s.table[b, torch.div(j, s.page, rounding_mode="floor")].long(), j % s.page


def limits(s, b, frame):
    """Keys seen by each row of sequence b."""
    q, n = s.q[b], s.kv[b]
    i = torch.arange(q, device=s.k.device)
    lim = torch.full((q,), n, device=s.k.device)
    if frame:
        lim = torch.clamp(n - q + (torch.div(i, frame, rounding_mode="floor") + 1) * frame, 0, n)
    return lim


def attention64(s, frame):
    """o [rows, H, hd], lse [rows, H], sum p |v|, and the largest sum |q k| / sqrt(hd) and key count of each row and head."""
    dev = s.k.device
    o = torch.zeros((s.rows, s.heads, s.hd), dtype=torch.float64, device=dev)
    lse = torch.full((s.rows, s.heads), -math.inf, dtype=torch.float64, device=dev)
    pv, qk = torch.zeros_like(o), torch.zeros_like(lse)
    grp, first = s.heads // s.kvh, 0
    for b, (q, n) in enumerate(zip(s.q, s.kv)):
        pg, sl = where(s, b)
        hidden = torch.arange(n, device=dev) >= limits(s, b, frame)[:, None]
        for h in range(s.heads if q and n else 0):
            k, v = s.k[pg, h // grp, sl].double(), s.v[pg, h // grp, sl].double()
            x = s.x[first:first + q, h * s.hd:(h + 1) * s.hd].double()
            sc = (x @ k.T / math.sqrt(s.hd)).masked_fill(hidden, -math.inf)
            ab = (x.abs() @ k.abs().T / math.sqrt(s.hd)).masked_fill(hidden, 0)
            z = torch.logsumexp(sc, 1)
            p = torch.where(hidden, 0, torch.exp(sc - torch.where(z == -math.inf, 0, z)[:, None]))
            lse[first:first + q, h] = z
            # a key that is not seen has no influence, whatever its value: 0 times its v is left out
            for r in torch.unique(limits(s, b, frame)).tolist():
                rows = limits(s, b, frame) == r
                o[first:first + q, h][rows] = p[rows, :r] @ v[:r]
                pv[first:first + q, h][rows] = p[rows, :r] @ v[:r].abs()
            qk[first:first + q, h] = ab.nan_to_num(0, 0, 0).amax(1)
        first += q
    return o, lse, pv, qk


def mass64(s, frame, lse, decay):
    """The masses [pages, kvh, page] (unwritten slots as they are), and for each the sum of its weights."""
    dev = s.k.device
    out = s.mass.double().clone()
    add = torch.zeros_like(out)
    grp, first = s.heads // s.kvh, 0
    for b, (q, n) in enumerate(zip(s.q, s.kv)):
        pg, sl = where(s, b)
        hidden = torch.arange(n, device=dev) >= limits(s, b, frame)[:, None]
        old = s.mass[pg, :, sl].double() * decay
        old[max(0, n - q):] = 0
        new = torch.zeros_like(old)
        for h in range(s.heads if q and n else 0):
            k = s.k[pg, h // grp, sl].double()
            x = s.x[first:first + q, h * s.hd:(h + 1) * s.hd].double()
            sc = x @ k.T / math.sqrt(s.hd)
            new[:, h // grp] += torch.where(hidden, 0, torch.exp(sc - lse[first:first + q, h, None].double())).sum(0)
        out[pg, :, sl] = old + new
        add[pg, :, sl] = new
        first += q
    return out, add


def evict64(s, mass, keep, sink, recent):
    """Plain eviction on the host: index [B][kvh] lists of former slots, in new slot order."""
    out = []
    for b, n in enumerate(s.kv):
        pg, sl = where(s, b)
        heads = []
        for h in range(s.kvh):
            if n <= keep:
                heads.append(list(range(n)))
                continue
            m = mass[pg, h, sl].double().cpu()
            m = torch.where(torch.isnan(m), torch.full_like(m, -math.inf), m).tolist()
            middle = sorted(range(sink, n - recent), key=lambda j: (-m[j], j))[:keep - sink - recent]
            kept = set(range(sink)) | set(range(n - recent, n)) | set(middle)
            above = iter(sorted(j for j in kept if j >= keep))
            heads.append([j if j in kept else next(above) for j in range(keep)])
        out.append(heads)
    return out
