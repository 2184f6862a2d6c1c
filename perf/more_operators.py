"""A paged key/value cache in 8 bits and attention from sequences that share a past: calls and plain forms.

Long clips are kept in pages of e4m3 codes: per slot and kv head one power of two
for the key and one for the value, so that a code times its power is exact in the
model's type. A chunk's program normalises and rotates the new queries and keys
and stores keys and values as codes (``append``), reads stored rows back in the
model's type (``read``) and attends over the codes (``attention8``). Where several
rollouts branch off one past, their chunks attend over the shared pages once for
all of them (``shared`` over a cache in the model's type, ``shared8`` over codes).

Row i of a chunk of q rows over n cached keys has slot n - q + i. It sees slot j if
j < n and, with ``frame`` > 0, j < n - q + (i // frame + 1) * frame. With groups of
sequences, the first P slots (whole pages) are those of the group's first sequence.

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
E4M3 = torch.float8_e4m3fn
ROPE = {64: (16, 24, 24), 128: (16, 56, 56)}   # rotary dimensions of the frame, row and column coordinates

# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------


def _text(v):
    return " ".join(str(x) for x in v)


def _case(kind, dtype, heads, kv_heads, hd, page, q, kv, **more):
    """q, kv: chunk rows and cached keys (chunk included) of each sequence."""
    return {"kind": kind, "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "hd": hd, "page": page, "q": _text(q),
            "kv": _text(kv), **more}


def listed():
    return [
        # sixteen streams, one new token each (an action or control token): launch latency
        {"name": "append_token", **_case("append", "bf16", 16, 16, 64, 16, [1] * 16, [37 + 211 * i for i in range(16)],
                                         weights=False)},
        # two frames of 34 x 60 tokens of a large model, with learned norm weights: bandwidth
        {"name": "append_chunk", **_case("append", "bf16", 16, 16, 128, 64, [4080], [8160], weights=True)},
        # float32 runs at odd lengths, rows without rotation among them
        {"name": "append_f32", **_case("append", "f32", 4, 4, 64, 32, [301, 1, 64], [301, 900, 77], weights=False)},
        # half a clip's keys and values for a consumer that takes the model's type
        {"name": "read_clip", **_case("read", "bf16", 16, 16, 128, 64, [33660], [33660])},
        # ragged pieces over small pages, float32
        {"name": "read_ragged", **_case("read", "f32", 12, 4, 64, 16, [77, 1, 0, 513, 40], [1000, 1, 40, 4133, 40])},
        # eight streams of very different age, one token each, four query heads per key head
        {"name": "attention8_token", **_case("attention8", "bf16", 32, 8, 128, 64, [1] * 8,
                                             [32768, 30001, 17, 4096, 9999, 24576, 1, 12345], frame=1, lse=False)},
        # two frames of 34 x 60 tokens over 33 frames, the new frames causal among themselves
        {"name": "attention8_long", **_case("attention8", "bf16", 16, 16, 128, 64, [4080], [67320], frame=2040, lse=False)},
        # ragged chunks, small pages, token-causal; a single token, an empty chunk and rows that see nothing
        {"name": "attention8_ragged", **_case("attention8", "bf16", 12, 4, 64, 16, [77, 1, 0, 513, 256, 40],
                                              [1000, 1, 40, 4133, 256, 25], frame=1, lse=True)},
        # float32 runs
        {"name": "attention8_f32", **_case("attention8", "f32", 4, 4, 64, 32, [256, 100], [1500, 777], frame=64, lse=True)},
        # thirty-two candidate actions, one token each, off one clip of twelve frames of 34 x 60 tokens
        {"name": "shared_token", **_case("shared", "bf16", 32, 8, 128, 64, [1] * 32, [24448 + 1 + 29 * i for i in range(32)],
                                         frame=1, lse=False, groups="32", prefix="24448")},
        # four candidate actions, one frame of 16 x 24 tokens each, off nine frames
        {"name": "shared_frame", **_case("shared", "bf16", 16, 16, 64, 64, [384] * 4, [3840, 4224, 3840, 4608], frame=0,
                                         lse=True, groups="4", prefix="3456")},
        # two pasts of unlike length with five and three rollouts of a few tokens, codes over small pages
        {"name": "shared8_tokens", **_case("shared8", "bf16", 32, 8, 128, 16, [1, 4, 2, 1, 7, 3, 1, 5],
                                           [40001, 40800, 40004, 41007, 40321, 9999, 9700, 10240], frame=1, lse=False,
                                           groups="5 3", prefix="40000 9600")},
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "append", "read", "attention8", "attention8", "attention8", "shared", "shared", "shared8"])
    hd = rng.choice([64, 128])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    kv_heads = rng.choice([1, 2, 4, 8, 12, 16])
    heads = kv_heads * rng.choice([1, 1, 2, 3, 4])
    heads = heads if heads <= 32 else kv_heads
    page = rng.choice([16, 32, 64, 128, 256])
    big = dtype == "bf16"
    if kind in ("shared", "shared8"):
        sizes = [rng.choice([1, 2, 3, 5, 8, 13]) for _ in range(rng.choice([1, 1, 2, 3]))]
        batch = sum(sizes)
        rows = 1 if rng.random() < 0.5 else _logint(rng, 2, max(3, (1500 if big else 300) / batch))
        prefix = [_logint(rng, 300, (40000 if big else 5000) / len(sizes)) // page * page for _ in sizes]
        q = [rng.randint(1, rows) for _ in range(batch)]
        past = [p for p, n in zip(prefix, sizes) for _ in range(n)]
        kv = [p + n + rng.choice([0, _logint(rng, 1, 1500)]) for p, n in zip(past, q)]
        return _case(kind, dtype, heads, kv_heads, hd, page, q, kv, frame=rng.choice([0, 1, 7, 64]), lse=rng.random() < 0.5,
                     groups=_text(sizes), prefix=_text(prefix))
    batch = rng.choice([1, 1, 2, 3, 5, 8])
    if rng.random() < 0.3:
        q = [1] * batch
    else:
        q = [_logint(rng, 8, (3000 if big else 600) / batch) for _ in range(batch)]
    kv = [n + _logint(rng, 40, (40000 if big else 5000) / batch) for n in q]
    if batch > 2 and rng.random() < 0.5:
        q[rng.randrange(batch)] = 0
    if kind == "append":
        return _case(kind, dtype, heads, kv_heads, hd, page, q, kv, weights=rng.random() < 0.5)
    if kind == "read":
        return _case(kind, dtype, heads, kv_heads, hd, page, kv if rng.random() < 0.5 else q, kv)
    return _case(kind, dtype, heads, kv_heads, hd, page, q, kv, frame=rng.choice([0, 1, 7, 64, 384]), lse=rng.random() < 0.5)


# ---------------------------------------------------------------------------
# seeded inputs
# ---------------------------------------------------------------------------


def _ints(case, name):
    return [int(x) for x in case[name].split()]


def _gen(seed, what):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + what * 7919 + 31) % (1 << 62))
    return g


def _randn(g, shape, dtype=torch.float32):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(dtype)


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    """The cache as earlier chunks left it, the page tables, and the chunk's rows."""
    q, kv = _ints(case, "q"), _ints(case, "kv")
    td = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    heads, hk, hd, page = case["heads"], case["kv_heads"], case["hd"], case["page"]
    s = SimpleNamespace(case=case, kind=case["kind"], td=td, rows=sum(q), max_q=max(q), max_kv=max(kv))
    need = [-(-n // page) for n in kv]
    shared = [0] * len(kv)                           # pages of a group's past that a sequence takes from its first one
    if "groups" in case:
        sizes, s.prefix = _ints(case, "groups"), _ints(case, "prefix")
        s.first = [sum(sizes[:g]) for g in range(len(sizes) + 1)]
        for g, p in enumerate(s.prefix):
            for b in range(s.first[g] + 1, s.first[g + 1]):
                shared[b] = p // page
        s.max_own = max(kv[b] - p for g, p in enumerate(s.prefix) for b in range(s.first[g], s.first[g + 1]))
        s.group_start, s.prefix_len = _int32(s.first), _int32(s.prefix)
    pages = sum(n - m for n, m in zip(need, shared)) + 3
    g = _gen(seed, 1)
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    s.table = torch.full((len(kv), max(1, max(need))), -1, dtype=torch.int32, device=DEV)   # -1: no page yet
    at = 0
    for b, n in enumerate(need):
        if shared[b]:
            s.table[b, :shared[b]] = s.table[max(f for f in s.first if f <= b), :shared[b]]
        s.table[b, shared[b]:n] = order[at:at + n - shared[b]]
        at += n - shared[b]
    s.kv_len, s.q_start = _int32(kv), _int32([sum(q[:b]) for b in range(len(q) + 1)])
    shape = (pages, hk, page, hd)
    if s.kind == "shared":
        s.k, s.v = _randn(_gen(seed, 3), shape, td), _randn(_gen(seed, 2), shape, td)
    else:
        # keys are normalised; values differ in size from slot to slot
        k, ke = _quantised(_randn(_gen(seed, 3), shape))
        v, ve = _quantised(_randn(_gen(seed, 2), shape) * torch.exp(0.5 * _randn(_gen(seed, 7), shape[:3]))[..., None])
        s.k, s.v, s.scale = k, v, torch.stack([ke, ve], -1).contiguous()
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
    elif s.kind == "read":
        s.kr, s.vr = (torch.empty((s.rows, hk * hd), dtype=td, device=DEV) for _ in range(2))
    else:
        # normalised heads times 1.5, so that some keys stand out
        s.q = (1.5 * _randn(_gen(seed, 5), (s.rows, heads * hd))).to(td)
        s.o = torch.empty_like(s.q)
        s.lse = torch.empty((s.rows, heads), device=DEV) if case["lse"] else None
    return s


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------


def _quantised(x):
    """Codes and exponent bytes of heads x [..., hd] float32: the smallest power of two, from 2^-117 on, that keeps them
    within 448 (so that every value is a normal number)."""
    m, e = torch.frexp(torch.where(torch.isfinite(x), x.abs(), 0).amax(-1))
    e = torch.where(m == 0, -117, (e - 9 + (m > 0.875)).clamp(min=-117))
    return torch.ldexp(x, -e[..., None]).to(E4M3), (e + 127).to(torch.uint8)


def _values(codes, byte):
    """What codes [..., hd] with exponent bytes [...] stand for, float32."""
    return torch.ldexp(codes.float(), byte.to(torch.int32)[..., None] - 127)


def _of_rows(s):
    """Sequence of each packed row, its place in the chunk, and its slot in the sequence."""
    r = torch.arange(s.rows, device=DEV)
    b = torch.searchsorted(s.q_start[1:], r.to(torch.int32), right=True)
    i = r - s.q_start[b]
    return b, i, s.kv_len[b] - (s.q_start[b + 1] - s.q_start[b]) + i


def _table(s):
    """Each sequence's pages, those of a shared past from its group's first sequence."""
    t = s.table.clamp(min=0).long()
    if "groups" not in s.case:
        return t
    g = torch.searchsorted(s.group_start[1:], torch.arange(len(t), dtype=torch.int32, device=DEV), right=True)
    past = torch.arange(t.shape[1], device=DEV) < (s.prefix_len[g] // s.case["page"])[:, None]
    return torch.where(past, t[s.group_start[g].long()], t)


def _gather(s, pool, which=None):
    """Pages [pages, Hk, page, hd] in sequence order [B, Hk, slots, hd] float32 (anything past a sequence's end)."""
    t = _table(s)
    x = pool[t] if which is None or s.kind == "shared" else _values(pool[t], s.scale[..., which][t])
    x = x.float().transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], -1, x.shape[4])


def _append(s):
    case = s.case
    heads, hk, hd = case["heads"], case["kv_heads"], case["hd"]
    x = s.qkv.float().reshape(s.rows, heads + 2 * hk, hd)
    qk = x[:, :heads + hk]
    qk = qk * torch.rsqrt((qk * qk).mean(2, keepdim=True) + EPS)
    if s.qw is not None:
        qk = qk * torch.cat([s.qw.expand(heads, hd), s.kw.expand(hk, hd)])
    dims = ROPE[hd]
    freq = torch.cat([10000.0 ** (-2 * torch.arange(d // 2, dtype=torch.float64, device=DEV) / d) for d in dims])
    axis = torch.repeat_interleave(torch.arange(3, device=DEV), torch.tensor([d // 2 for d in dims], device=DEV),
                                   output_size=hd // 2)
    ang = torch.where(s.pos[:, :1] < 0, 0, s.pos.double()[:, axis] * freq)
    co, si = torch.cos(ang).float()[:, None], torch.sin(ang).float()[:, None]
    a, c = qk[..., 0::2], qk[..., 1::2]
    qk = torch.stack([a * co - c * si, a * si + c * co], -1).reshape(s.rows, heads + hk, hd)
    s.q.copy_(qk[:, :heads].reshape(s.rows, -1))
    b, _, slot = _of_rows(s)
    page = s.table[b, slot // case["page"]].long()
    for pool, which, rows in ((s.k, 0, qk[:, heads:]), (s.v, 1, x[:, heads + hk:])):
        code, byte = _quantised(rows)
        pool.view(torch.uint8)[page, :, slot % case["page"]] = code.view(torch.uint8)
        s.scale[page, :, slot % case["page"], which] = byte
    # a power of two's byte, as the number that it stands for
    return {"q": s.q, "k": s.k, "v": s.v, "scale": s.scale.view(torch.float8_e8m0fnu)}


def _read(s):
    b, _, slot = _of_rows(s)
    page, at = s.table[b, slot // s.case["page"]].long(), slot % s.case["page"]
    byte = s.scale[page, :, at]
    s.kr.copy_(_values(s.k[page, :, at], byte[..., 0]).reshape(s.rows, -1))
    s.vr.copy_(_values(s.v[page, :, at], byte[..., 1]).reshape(s.rows, -1))
    return {"k": s.kr, "v": s.vr}


def _attention(s):
    case, hk, hd = s.case, s.case["kv_heads"], s.case["hd"]
    group = case["heads"] // hk
    i, n = torch.arange(s.max_q, device=DEV), s.q_start[1:] - s.q_start[:-1]
    at = (s.q_start[:-1, None] + i).clamp(max=max(s.rows - 1, 0)).long()
    q = s.q[at].float().reshape(len(at), s.max_q, hk, group, hd).transpose(1, 2).reshape(len(at), hk, -1, hd)
    sc = torch.matmul(q, _gather(s, s.k, 0).transpose(2, 3).contiguous())
    sc *= 1 / math.sqrt(hd)
    lim = s.kv_len[:, None].expand(-1, s.max_q)
    if case["frame"]:
        lim = torch.minimum(lim, (s.kv_len - n)[:, None] + (i // case["frame"] + 1) * case["frame"])
    lim = torch.where(i < n[:, None], lim, 0).repeat_interleave(group, 1)
    sc.masked_fill_(torch.arange(sc.shape[3], device=DEV) >= lim[:, None, :, None], -math.inf)
    m = sc.amax(3, keepdim=True)
    m = torch.where(m == -math.inf, 0, m)
    sc -= m
    p = sc.exp_()
    total = p.sum(3, keepdim=True)
    v = _gather(s, s.v, 1)
    v.masked_fill_(torch.arange(v.shape[2], device=DEV)[:, None] >= s.kv_len[:, None, None, None], 0)
    o = torch.matmul(p, v) / torch.where(total == 0, 1, total)
    s.o.copy_(_packed(s, o).reshape(s.rows, -1))
    if s.lse is None:
        return {"o": s.o}
    s.lse.copy_(_packed(s, m + total.log())[..., 0])
    return {"o": s.o, "lse": s.lse}


def _packed(s, x):
    """[B, Hk, rows x group, n] of padded chunks -> [rows, heads, n]."""
    b, i, _ = _of_rows(s)
    case = s.case
    x = x.reshape(x.shape[0], case["kv_heads"], s.max_q, -1, x.shape[3]).transpose(1, 2)
    return x[b, i].reshape(s.rows, case["heads"], -1)


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
        s.cache = wdc.PagedCache(s.k, s.v) if s.kind == "shared" else wdc.PagedCache8(s.k, s.v, s.scale)
        s.chunks = wdc.Chunks(s.q_start, s.kv_len, s.table, rows=s.rows, max_q=s.max_q, max_kv=s.max_kv)
        if "groups" in case:
            s.past = wdc.Prefix(s.group_start, s.prefix_len, max_prefix=max(s.prefix), max_own=s.max_own)
    return s.ctx


def _own(s):
    case, ctx = s.case, _handles(s)
    if s.kind == "append":
        ctx.cache8_append(s.cache, s.chunks, s.qkv, s.q, pos=s.pos, q_weight=s.qw, k_weight=s.kw)
        return {"q": s.q, "k": s.k, "v": s.v, "scale": s.scale.view(torch.float8_e8m0fnu)}
    if s.kind == "read":
        ctx.cache8_read(s.cache, s.chunks, k=s.kr, v=s.vr)
        return {"k": s.kr, "v": s.vr}
    if s.kind == "attention8":
        ctx.cache8_attention(s.cache, s.chunks, s.q, s.o, frame=case["frame"], lse=s.lse)
    elif s.kind == "shared8":
        ctx.cache8_attention(s.cache, s.chunks, s.q, s.o, frame=case["frame"], lse=s.lse, prefix=s.past)
    else:
        ctx.cache_attention_shared(s.cache, s.chunks, s.past, s.q, s.o, frame=case["frame"], lse=s.lse)
    return {"o": s.o} if s.lse is None else {"o": s.o, "lse": s.lse}


def run(s):
    if own:
        return _own(s)
    return {"append": _append, "read": _read}.get(s.kind, _attention)(s)


# ---------------------------------------------------------------------------
# work and exact values
# ---------------------------------------------------------------------------


def work(case):
    q, kv = _ints(case, "q"), _ints(case, "kv")
    e = 2 if case["dtype"] == "bf16" else 4
    heads, hk, hd = case["heads"], case["kv_heads"], case["hd"]
    rows = sum(q)
    if case["kind"] == "append":
        return {"bytes": rows * ((2 * heads + 2 * hk) * hd * e + 2 * hk * (hd + 1) + 12), "flops": 0}
    if case["kind"] == "read":
        return {"bytes": 2 * rows * hk * (hd * e + hd + 1), "flops": 0}
    keys = sum(n for m, n in zip(q, kv) if m)
    if "groups" in case:                             # a past is read once for its group
        for size, p in zip(_ints(case, "groups"), _ints(case, "prefix")):
            keys -= (size - 1) * p
    pairs = 0
    for m, n in zip(q, kv):
        f = case["frame"] or max(m, 1)
        for c in range(-(-m // f)):
            pairs += min(f, m - c * f) * max(0, min(n, n - m + (c + 1) * f if case["frame"] else n))
    slot = hd * e if case["kind"] == "shared" else hd + 1
    return {"bytes": 2 * rows * heads * hd * e + 2 * keys * hk * slot + (4 * rows * heads if case["lse"] else 0),
            "flops": 4 * hd * heads * pairs}


def _power64(x):
    """The cache's power of two for heads x [..., hd] float64."""
    big = torch.where(torch.isfinite(x), x.abs(), 0).amax(-1, keepdim=True).clamp(min=448 * 2.0 ** -117)
    p = torch.exp2(torch.floor(torch.log2(big)) - 8)           # 448 is 1.75 * 2^8
    return torch.where(big > 448 * p, 2 * p, p)


def exact(case, seed):
    s = prepare(case, seed)
    q, kv = _ints(case, "q"), _ints(case, "kv")
    heads, hk, hd, page = case["heads"], case["kv_heads"], case["hd"], case["page"]
    grp, first = heads // hk, [sum(q[:b]) for b in range(len(q))]
    where = [s.table[b, torch.arange(n, device=DEV) // page].long() for b, n in enumerate(kv)]
    slot = [torch.arange(n, device=DEV) % page for n in kv]
    for g, p in enumerate(getattr(s, "prefix", [])):
        for b in range(s.first[g], s.first[g + 1]):
            where[b][:p] = where[s.first[g]][:p]
    power = None if case["kind"] == "shared" else torch.exp2(s.scale.double() - 127)
    if case["kind"] == "append":                     # codes before their rounding
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
            for which, pool, rows in ((0, k, qk[first[b]:first[b] + m, heads:]), (1, v, x[first[b]:first[b] + m, heads + hk:])):
                p = _power64(rows)
                pool[where[b][n - m:], :, slot[b][n - m:]] = rows / p
                power[where[b][n - m:], :, slot[b][n - m:], which] = p[..., 0]
        return {"q": qk[:, :heads].reshape(s.rows, -1), "k": k, "v": v, "scale": power}
    if case["kind"] == "read":
        k, v = (torch.zeros((s.rows, hk, hd), dtype=torch.float64, device=DEV) for _ in range(2))
        for b, (m, n) in enumerate(zip(q, kv)):
            w, j = where[b][n - m:], slot[b][n - m:]
            k[first[b]:first[b] + m] = s.k[w, :, j].double() * power[w, :, j, 0, None]
            v[first[b]:first[b] + m] = s.v[w, :, j].double() * power[w, :, j, 1, None]
        return {"k": k.reshape(s.rows, -1), "v": v.reshape(s.rows, -1)}
    o = torch.zeros((s.rows, heads, hd), dtype=torch.float64, device=DEV)
    lse = torch.full((s.rows, heads), -math.inf, dtype=torch.float64, device=DEV)
    for b, (m, n) in enumerate(zip(q, kv)):
        rows = slice(first[b], first[b] + m)
        i = torch.arange(m, device=DEV)
        see = torch.full((m,), n, device=DEV)
        if case["frame"]:
            see = torch.clamp(n - m + (torch.div(i, case["frame"], rounding_mode="floor") + 1) * case["frame"], max=n)
        hidden = torch.arange(n, device=DEV) >= see[:, None]
        for h in range(heads if m and n else 0):
            at = (where[b], h // grp, slot[b])
            k, v = s.k[at].double(), s.v[at].double()
            if power is not None:
                k, v = k * power[at][:, :1], v * power[at][:, 1:]
            sc = (s.q[rows, h * hd:(h + 1) * hd].double() @ k.T) / math.sqrt(hd)
            sc.masked_fill_(hidden, -math.inf)
            lse[rows, h] = torch.logsumexp(sc, 1)
            sc -= lse[rows, h, None]
            o[rows, h] = sc.exp_().masked_fill_(hidden, 0) @ v
    out = {"o": o.reshape(s.rows, -1)}
    return {**out, "lse": lse} if case["lse"] else out
