"""The operators of a streaming rollout's paged key/value cache: their calls and their plain forms.

A world model rolled out chunk by chunk keeps the keys and values of the frames
so far in pages. Per layer and chunk its program normalises and rotates the new
queries and keys and stores keys and values (``append``), attends from the
chunk over the cache (``attention``), adds up how much weight each cached key
received (``mass``) and, when the cache is full, drops the keys of least weight
(``evict``). Several sequences share one call: their chunk rows are packed, and
each has a table of pages and a number of cached keys, its chunk included.

Query i of a chunk of q rows over n cached keys sees key j if j < n and, with
``frame`` > 0, j < n - q + (i // frame + 1) * frame: everything cached before
the chunk and the chunk's own frames up to its own.

The plain forms are elementary torch operations in float32 (angles in float64),
rounded once at the end; ``exact`` computes the definitions in float64.
"""
from __future__ import annotations

import math
from functools import lru_cache
from types import SimpleNamespace

import torch

own = False
DEV = "cuda:0"
EPS = 1e-6
ROPE = {64: (16, 24, 24), 128: (16, 56, 56)}   # rotary dimensions of the frame, row and column coordinates

# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------


def _case(kind, dtype, heads, kv_heads, hd, page, q, kv, **more):
    """q, kv: chunk rows and cached keys (chunk included) of each sequence."""
    text = lambda v: " ".join(str(x) for x in v)  # noqa: E731
    return {"kind": kind, "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "hd": hd, "page": page, "q": text(q),
            "kv": text(kv), **more}


def listed():
    return [
        # sixteen streams, one new token each (an action or control token): launch latency
        {"name": "append_token", **_case("append", "bf16", 16, 16, 64, 16, [1] * 16, [37 + 211 * i for i in range(16)],
                                         weights=False)},
        # two frames of 34 x 60 tokens of a large model, with learned norm weights: bandwidth
        {"name": "append_chunk", **_case("append", "bf16", 16, 16, 128, 64, [4080], [8160], weights=True)},
        # float32 runs at odd lengths, rows without rotation among them
        {"name": "append_f32", **_case("append", "f32", 4, 4, 64, 32, [301, 1, 64], [301, 900, 77], weights=False)},
        # eight streams of very different age, one token each, four query heads per key head
        {"name": "attention_token", **_case("attention", "bf16", 32, 8, 128, 64, [1] * 8,
                                            [32768, 30001, 17, 4096, 9999, 24576, 1, 12345], frame=1, lse=False)},
        # one frame of 16 x 24 tokens over a clip of eight: an interactive rollout's layer
        {"name": "attention_frame", **_case("attention", "bf16", 16, 16, 64, 64, [384], [3072 + 384], frame=0, lse=True)},
        # two frames of 34 x 60 tokens over 33 frames, the new frames causal among themselves
        {"name": "attention_long", **_case("attention", "bf16", 16, 16, 128, 64, [4080], [67320], frame=2040, lse=False)},
        # ragged chunks, small pages, token-causal; a single token, an empty chunk and rows that see nothing
        {"name": "attention_ragged", **_case("attention", "bf16", 12, 4, 64, 16, [77, 1, 0, 513, 256, 40],
                                             [1000, 1, 40, 4133, 256, 25], frame=1, lse=True)},
        # float32 runs
        {"name": "attention_f32", **_case("attention", "f32", 4, 4, 64, 32, [256, 100], [1500, 777], frame=64, lse=True)},
        # weights of one frame's attention at the mid size
        {"name": "mass_frame", **_case("mass", "bf16", 16, 16, 64, 64, [384], [3072 + 384], frame=0, decay=0.9)},
        # weights of one frame of 34 x 60 tokens over 17 frames
        {"name": "mass_long", **_case("mass", "bf16", 16, 16, 128, 64, [2040], [34680], frame=2040, decay=1.0)},
        # four streams trimmed by about a quarter
        {"name": "evict_streams", **_case("evict", "bf16", 16, 16, 64, 64, [384] * 4, [3001, 3456, 2000, 3072], keep=2304,
                                          sink=384, recent=384)},
        # 33 frames trimmed to 30
        {"name": "evict_long", **_case("evict", "bf16", 16, 16, 128, 64, [4080], [67320], keep=61200, sink=2040,
                                       recent=4080)},
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "append", "attention", "attention", "attention", "mass", "mass", "evict", "evict"])
    hd = rng.choice([64, 128])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    kv_heads = rng.choice([1, 2, 4, 8, 12, 16])
    heads = kv_heads * rng.choice([1, 1, 2, 3, 4])
    heads = heads if heads <= 32 else kv_heads
    page = rng.choice([16, 32, 64, 128, 256])
    batch = rng.choice([1, 1, 2, 3, 5, 8])
    big = dtype == "bf16"
    if rng.random() < 0.3:
        q = [1] * batch
    else:
        q = [_logint(rng, 8, (3000 if big else 600) / batch) for _ in range(batch)]
    kv = [n + _logint(rng, 40, (40000 if big else 5000) / batch) for n in q]
    if batch > 2 and rng.random() < 0.5:
        q[rng.randrange(batch)] = 0
    frame = rng.choice([0, 1, 7, 64, 384])
    if kind == "append":
        return _case(kind, dtype, heads, kv_heads, hd, page, q, kv, weights=rng.random() < 0.5)
    if kind == "attention":
        return _case(kind, dtype, heads, kv_heads, hd, page, q, kv, frame=frame, lse=rng.random() < 0.5)
    if kind == "mass":
        return _case(kind, dtype, heads, kv_heads, hd, page, q, kv, frame=frame, decay=rng.choice([0.0, 0.5, 0.9, 1.0]))
    keep = max(4, int(max(kv) * rng.uniform(0.3, 1.0)))
    return _case(kind, dtype, heads, kv_heads, hd, page, q, kv, keep=keep, sink=int(keep * rng.uniform(0, 0.4)),
                 recent=int(keep * rng.uniform(0, 0.5)))


# ---------------------------------------------------------------------------
# seeded inputs
# ---------------------------------------------------------------------------


def _lens(case):
    return [int(x) for x in case["q"].split()], [int(x) for x in case["kv"].split()]


def _gen(seed, what):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + what * 7919 + 29) % (1 << 62))
    return g


def _randn(g, shape, dtype=torch.float32):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(dtype)


def prepare(case, seed):
    """The cache as earlier chunks left it, the page tables, and the chunk's rows."""
    q, kv = _lens(case)
    td = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    heads, hk, hd, page = case["heads"], case["kv_heads"], case["hd"], case["page"]
    s = SimpleNamespace(case=case, kind=case["kind"], rows=sum(q), max_q=max(q), max_kv=max(kv))
    need = [-(-n // page) for n in kv]
    pages = sum(need) + 3
    g = _gen(seed, 1)
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    s.table = torch.full((len(kv), max(1, max(need))), -1, dtype=torch.int32, device=DEV)   # -1: no page yet
    at = 0
    for b, n in enumerate(need):
        s.table[b, :n] = order[at:at + n]
        at += n
    s.kv_len = torch.tensor(kv, dtype=torch.int32, device=DEV)
    s.q_start = torch.tensor([sum(q[:b]) for b in range(len(q) + 1)], dtype=torch.int32, device=DEV)
    shape = (pages, hk, page, hd)
    if s.kind != "mass":
        s.v = _randn(_gen(seed, 2), shape, td)
    s.k = _randn(_gen(seed, 3), shape, td)
    if s.kind == "append":
        g = _gen(seed, 4)
        s.qkv = _randn(g, (s.rows, (heads + 2 * hk) * hd), td)
        # frames of 60 columns far into a long rollout; every eleventh row is a text token (t < 0: not rotated)
        i = torch.arange(s.rows, device=DEV)
        first = int(torch.randint(0, 100000, (1,), generator=g, device=DEV))
        s.pos = torch.stack([first + i // 2040, i // 60 % 34, i % 60], 1)
        s.pos[i % 11 == 10] = -1
        s.pos = s.pos.to(torch.int32).contiguous()
        s.qw = 1 + 0.1 * _randn(g, (hd,)) if case["weights"] else None
        s.kw = 1 + 0.1 * _randn(g, (hd,)) if case["weights"] else None
        s.q = torch.empty((s.rows, heads * hd), dtype=td, device=DEV)
    if s.kind in ("attention", "mass"):
        # normalised heads times 1.5, so that some keys stand out
        s.q = (1.5 * _randn(_gen(seed, 5), (s.rows, heads * hd))).to(td)
        s.o = torch.empty_like(s.q)
    if s.kind == "attention":
        s.lse = torch.empty((s.rows, heads), device=DEV) if case["lse"] else None
    if s.kind in ("mass", "evict"):
        # attention weight is spread over orders of magnitude
        s.mass = torch.exp(1.5 * _randn(_gen(seed, 6), shape[:3]))
        s.mass_out = torch.zeros_like(s.mass)
    if s.kind == "mass":
        s.lse = _softmax(s)[2]
    if s.kind == "evict":
        s.len_out = torch.empty_like(s.kv_len)
        s.index = torch.empty((len(kv), hk, case["keep"]), dtype=torch.int32, device=DEV)
    return s


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------


def _of_rows(s):
    """Sequence of each packed row, its place in the chunk, and its slot in the sequence."""
    r = torch.arange(s.rows, device=DEV)
    b = torch.searchsorted(s.q_start[1:], r.to(torch.int32), right=True)
    i = r - s.q_start[b]
    return b, i, s.kv_len[b] - (s.q_start[b + 1] - s.q_start[b]) + i


def _gather(s, pool):
    """Pages [pages, Hk, page, ...] in sequence order [B, Hk, slots, ...] (anything past a sequence's end)."""
    t = s.table.clamp(min=0).long()
    x = pool[t].transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], -1, *x.shape[4:])


def _flat(s, hk, page):
    """Index of (sequence, kv head, slot) in the pool's [pages * Hk * page] rows: [B, Hk, slots]."""
    slots = torch.arange(s.table.shape[1] * page, device=DEV)
    pg = s.table.clamp(min=0).long()[:, slots // page]
    return (pg[:, None, :] * hk + torch.arange(hk, device=DEV)[None, :, None]) * page + slots % page


def _scores(s):
    """Scores of the padded chunks [B, Hk, rows x group, slots] and where a key is not seen."""
    case, hk, hd = s.case, s.case["kv_heads"], s.case["hd"]
    group = case["heads"] // hk
    i, n = torch.arange(s.max_q, device=DEV), s.q_start[1:] - s.q_start[:-1]
    at = (s.q_start[:-1, None] + i).clamp(max=max(s.rows - 1, 0)).long()
    q = s.q[at].float().reshape(len(at), s.max_q, hk, group, hd).transpose(1, 2).reshape(len(at), hk, -1, hd)
    sc = torch.matmul(q, _gather(s, s.k).float().transpose(2, 3).contiguous())
    sc *= 1 / math.sqrt(hd)
    lim = s.kv_len[:, None].expand(-1, s.max_q)
    if case["frame"]:
        lim = torch.minimum(lim, (s.kv_len - n)[:, None] + (i // case["frame"] + 1) * case["frame"])
    lim = torch.where(i < n[:, None], lim, 0).repeat_interleave(group, 1)
    return sc, torch.arange(sc.shape[3], device=DEV) >= lim[:, None, :, None]


def _softmax(s):
    """Unnormalised weights, their sums, and the rows' log-sum-exp [rows, H]."""
    sc, unseen = _scores(s)
    sc.masked_fill_(unseen, -math.inf)
    m = sc.amax(3, keepdim=True)
    m = torch.where(m == -math.inf, 0, m)
    p = (sc - m).exp_()
    total = p.sum(3, keepdim=True)
    return p, total, _packed(s, m + total.log())[..., 0]


def _packed(s, x):
    """[B, Hk, rows x group, n] of padded chunks -> [rows, heads, n]."""
    b, i, _ = _of_rows(s)
    case = s.case
    x = x.reshape(x.shape[0], case["kv_heads"], s.max_q, -1, x.shape[3]).transpose(1, 2)
    return x[b, i].reshape(s.rows, case["heads"], -1)


def _append(s):
    case = s.case
    heads, hk, hd = case["heads"], case["kv_heads"], case["hd"]
    x = s.qkv.float().reshape(s.rows, heads + 2 * hk, hd)
    qk = x[:, :heads + hk]
    qk = qk * torch.rsqrt((qk * qk).mean(2, keepdim=True) + EPS)
    if s.qw is not None:
        qk = qk * torch.cat([s.qw.expand(heads, hd), s.kw.expand(hk, hd)])
    ang = _angles(s, torch.float64)
    co, si = torch.cos(ang).float()[:, None], torch.sin(ang).float()[:, None]
    a, c = qk[..., 0::2], qk[..., 1::2]
    qk = torch.stack([a * co - c * si, a * si + c * co], -1).reshape(s.rows, heads + hk, hd)
    s.q.copy_(qk[:, :heads].reshape(s.rows, -1))
    b, _, slot = _of_rows(s)
    page = s.table[b, slot // case["page"]].long()
    s.k[page, :, slot % case["page"]] = qk[:, heads:].to(s.k.dtype)
    s.v[page, :, slot % case["page"]] = x[:, heads + hk:].to(s.v.dtype)
    return {"q": s.q, "k": s.k, "v": s.v}


def _angles(s, dtype):
    """Rotation angle of each pair of each row (0 where t < 0)."""
    dims = ROPE[s.case["hd"]]
    freq = torch.cat([10000.0 ** (-2 * torch.arange(d // 2, dtype=dtype, device=DEV) / d) for d in dims])
    axis = torch.repeat_interleave(torch.arange(3, device=DEV), torch.tensor([d // 2 for d in dims], device=DEV),
                                   output_size=sum(dims) // 2)
    return torch.where(s.pos[:, :1] < 0, 0, s.pos.to(dtype)[:, axis] * freq)


def _attention(s):
    p, total, lse = _softmax(s)
    v = _gather(s, s.v).float()
    v = torch.where(torch.arange(v.shape[2], device=DEV)[:, None] < s.kv_len[:, None, None, None], v, 0)
    o = torch.matmul(p, v) / torch.where(total == 0, 1, total)
    s.o.copy_(_packed(s, o).reshape(s.rows, -1))
    if s.lse is None:
        return {"o": s.o}
    s.lse.copy_(lse)
    return {"o": s.o, "lse": s.lse}


def _mass(s):
    case, hk = s.case, s.case["kv_heads"]
    n = s.q_start[1:] - s.q_start[:-1]
    at = (s.q_start[:-1, None] + torch.arange(s.max_q, device=DEV)).clamp(max=max(s.rows - 1, 0)).long()
    lse = s.lse[at].reshape(len(at), s.max_q, hk, -1).transpose(1, 2).reshape(len(at), hk, -1, 1)
    sc, unseen = _scores(s)
    sc -= lse
    add = sc.exp_().masked_fill_(unseen, 0).sum(2)
    j = torch.arange(add.shape[2], device=DEV)
    old = torch.where(j < (s.kv_len - n)[:, None, None], case["decay"] * _gather(s, s.mass), 0)
    to = torch.where(j < s.kv_len[:, None, None], _flat(s, hk, case["page"]), s.mass.numel())
    out = torch.cat([s.mass_out.reshape(-1), s.mass_out.new_zeros(1)])
    out[to.reshape(-1)] = (old + add).reshape(-1)
    s.mass_out.copy_(out[:-1].reshape(s.mass_out.shape))
    return {"mass": s.mass_out}


def _evict(s):
    case = s.case
    hk, hd, page, keep = case["kv_heads"], case["hd"], case["page"], case["keep"]
    n = s.kv_len[:, None, None].long()
    mass = _gather(s, s.mass)
    j = torch.arange(mass.shape[2], device=DEV).expand_as(mass)
    key = torch.where(torch.isnan(mass), -math.inf, mass)
    key = torch.where((j < case["sink"]) | (j >= n - case["recent"]), math.inf, key)
    key = torch.where(j < n, key, -math.inf)
    best = torch.sort(key, dim=2, descending=True, stable=True)[1][..., :keep]
    kept = torch.zeros_like(j, dtype=torch.bool).scatter(2, best, True) | (n <= keep)
    kept &= j < n
    hole, mover = ~kept & (j < keep) & (j < n), kept & (j >= keep)
    rank = torch.where(mover, mover.cumsum(2) - 1, keep)
    source = torch.zeros((*j.shape[:2], keep + 1), dtype=torch.long, device=DEV).scatter(2, rank, j)
    index = torch.where(hole, source.gather(2, (hole.cumsum(2) - 1).clamp(0, keep)), j)[..., :keep]
    live = j[..., :keep] < n
    pad = keep - index.shape[2]
    s.index.copy_(torch.nn.functional.pad(torch.where(live, index, -1), (0, pad), value=-1))
    s.len_out.copy_(s.kv_len.clamp(max=keep))
    flat = _flat(s, hk, page)
    src, rows = flat.gather(2, index.clamp(min=0)), s.mass.numel()
    to = torch.where(live, flat[..., :keep], rows).reshape(-1)
    new = [torch.cat([t.reshape(rows, -1), t.new_zeros(1, t.numel() // rows)]) for t in (s.k, s.v, s.mass_out)]
    for t, old in zip(new, (s.k, s.v, s.mass)):
        t[to] = old.reshape(rows, -1)[src.reshape(-1)]
    for t, x in zip((s.k, s.v, s.mass_out), new):
        t.copy_(x[:-1].reshape(t.shape))
    return {"k": s.k, "v": s.v, "mass": s.mass_out, "kv_len": s.len_out, "index": s.index}


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------


@lru_cache(maxsize=None)
def _context(dtype, heads, hd):
    """A context for the attention shape: no blocks, one latent patch."""
    import paper_2608_01845_amd as wdc
    cfg = SimpleNamespace(name="stream", dtype=dtype, hidden=heads * hd, heads=heads, head_dim=hd, mlp_ratio=4, n_seq=0,
                          n_dual=0, n_single=0, cond_dim=0, cam_dim=0, text_tokens=0, text_dim=0, latent=(16, 1, 2, 2),
                          patch=(1, 2, 2), rope=ROPE[hd], qk_norm=True, n_video=1)
    return wdc.Context(cfg, allocate_weights=False)


def _handles(s):
    """The context, cache and chunk descriptors that a program keeps beside its tensors."""
    if not hasattr(s, "ctx"):
        import paper_2608_01845_amd as wdc
        case = s.case
        s.ctx = _context(case["dtype"], case["heads"], case["hd"])
        s.cache = wdc.PagedCache(s.k, s.v if hasattr(s, "v") else s.k)
        s.chunks = wdc.Chunks(s.q_start, s.kv_len, s.table, rows=s.rows, max_q=s.max_q, max_kv=s.max_kv)
    return s.ctx


def _own(s):
    case, ctx = s.case, _handles(s)
    if s.kind == "append":
        ctx.cache_append(s.cache, s.chunks, s.qkv, s.q, pos=s.pos, q_weight=s.qw, k_weight=s.kw)
        return {"q": s.q, "k": s.k, "v": s.v}
    if s.kind == "attention":
        ctx.cache_attention(s.cache, s.chunks, s.q, s.o, frame=case["frame"], lse=s.lse)
        return {"o": s.o} if s.lse is None else {"o": s.o, "lse": s.lse}
    if s.kind == "mass":
        ctx.cache_mass(s.cache, s.chunks, s.q, s.lse, s.mass, frame=case["frame"], decay=case["decay"], out=s.mass_out)
        return {"mass": s.mass_out}
    ctx.cache_evict(s.cache, s.chunks, s.mass, keep=case["keep"], sink=case["sink"], recent=case["recent"],
                    kv_len_out=s.len_out, index=s.index, out=s.mass_out)
    return {"k": s.k, "v": s.v, "mass": s.mass_out, "kv_len": s.len_out, "index": s.index}


def run(s):
    if own:
        return _own(s)
    return {"append": _append, "attention": _attention, "mass": _mass, "evict": _evict}[s.kind](s)


# ---------------------------------------------------------------------------
# work and exact values
# ---------------------------------------------------------------------------


def _pairs(case):
    """Visible (query, key) pairs."""
    q, kv = _lens(case)
    total = 0
    for m, n in zip(q, kv):
        f = case["frame"] or max(m, 1)
        for c in range(-(-m // f)):
            total += min(f, m - c * f) * max(0, min(n, n - m + (c + 1) * f if case["frame"] else n))
    return total


def work(case):
    q, kv = _lens(case)
    e = 2 if case["dtype"] == "bf16" else 4
    heads, hk, hd = case["heads"], case["kv_heads"], case["hd"]
    rows, keys = sum(q), sum(n for m, n in zip(q, kv) if m)
    if case["kind"] == "append":
        return {"bytes": 2 * rows * (heads + 2 * hk) * hd * e + 12 * rows, "flops": 0}
    if case["kind"] == "attention":
        return {"bytes": 2 * rows * heads * hd * e + 2 * keys * hk * hd * e + (4 * rows * heads if case["lse"] else 0),
                "flops": 4 * hd * heads * _pairs(case)}
    if case["kind"] == "mass":
        return {"bytes": rows * heads * (hd * e + 4) + keys * hk * (hd * e + 8), "flops": 2 * hd * heads * _pairs(case)}
    total, keep, sink, recent = 0, case["keep"], case["sink"], case["recent"]
    for n in kv:
        total += 4 * hk * min(n, keep)                           # the index
        if n > keep:
            middle = n - sink - recent
            moved = min(n - keep, recent) + max(0, n - keep - recent) * (keep - sink - recent) / max(1, middle)
            total += hk * (4 * n + 8 * keep + 2 * moved * 2 * hd * e)   # masses read, kept ones written; rows moved
        else:
            total += hk * 8 * n
    return {"bytes": total, "flops": 0}


def exact(case, seed):
    s = prepare(case, seed)
    q, kv = _lens(case)
    heads, hk, hd, page = case["heads"], case["kv_heads"], case["hd"], case["page"]
    grp, first = heads // hk, [sum(q[:b]) for b in range(len(q))]
    where = [s.table[b, torch.arange(n, device=DEV) // page].long() for b, n in enumerate(kv)]
    slot = [torch.arange(n, device=DEV) % page for n in kv]
    if case["kind"] == "append":
        x = s.qkv.double().reshape(s.rows, heads + 2 * hk, hd)
        qk = x[:, :heads + hk]
        qk = qk / torch.sqrt(qk.square().mean(2, keepdim=True) + EPS)
        if s.qw is not None:
            qk = qk * torch.cat([s.qw.double().expand(heads, hd), s.kw.double().expand(hk, hd)])
        z = torch.view_as_complex(qk.reshape(s.rows, heads + hk, hd // 2, 2).contiguous())
        col = 0
        for a, d in enumerate(ROPE[hd]):
            for p in range(d // 2):
                turn = torch.where(s.pos[:, 0] < 0, 0, s.pos[:, a].double() * 10000.0 ** (-2 * p / d))
                z[..., col] *= torch.polar(torch.ones_like(turn), turn)[:, None]
                col += 1
        qk = torch.view_as_real(z).reshape(s.rows, heads + hk, hd)
        k, v = s.k.double(), s.v.double()
        for b, (m, n) in enumerate(zip(q, kv)):
            k[where[b][n - m:], :, slot[b][n - m:]] = qk[first[b]:first[b] + m, heads:]
            v[where[b][n - m:], :, slot[b][n - m:]] = x[first[b]:first[b] + m, heads + hk:].double()
        return {"q": qk[:, :heads].reshape(s.rows, -1), "k": k, "v": v}
    if case["kind"] == "evict":
        return None                              # values are moved, not computed
    o = torch.zeros((s.rows, heads, hd), dtype=torch.float64, device=DEV)
    lse = torch.full((s.rows, heads), -math.inf, dtype=torch.float64, device=DEV)
    mass = s.mass_out.double() if case["kind"] == "mass" else None
    for b, (m, n) in enumerate(zip(q, kv)):
        if mass is not None:
            old = s.mass[where[b], :, slot[b]].double() * case["decay"]
            old[max(0, n - m):] = 0
        rows = slice(first[b], first[b] + m)
        i = torch.arange(m, device=DEV)
        see = torch.full((m,), n, device=DEV)
        if case["frame"]:
            see = torch.clamp(n - m + (torch.div(i, case["frame"], rounding_mode="floor") + 1) * case["frame"], max=n)
        hidden = torch.arange(n, device=DEV) >= see[:, None]
        for h in range(heads if m and n else 0):
            k = s.k[where[b], h // grp, slot[b]].double()
            sc = (s.q[rows, h * hd:(h + 1) * hd].double() @ k.T) / math.sqrt(hd)
            sc.masked_fill_(hidden, -math.inf)
            if mass is not None:
                old[:, h // grp] += (sc - s.lse[rows, h, None].double()).exp_().masked_fill_(hidden, 0).sum(0)
                continue
            lse[rows, h] = torch.logsumexp(sc, 1)
            sc -= lse[rows, h, None]
            o[rows, h] = sc.exp_().masked_fill_(hidden, 0) @ s.v[where[b], h // grp, slot[b]].double()
        if mass is not None:
            mass[where[b], :, slot[b]] = old
    if mass is not None:
        return {"mass": mass}
    out = {"o": o.reshape(s.rows, -1)}
    return {**out, "lse": lse} if case["lse"] else out
