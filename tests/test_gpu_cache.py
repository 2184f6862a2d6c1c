"""The paged key/value cache operators against their definitions in float64:
append (norms, rotation, page writes), attention of chunks, accumulated weights,
eviction, and a rollout's run of them together."""
import math

import pytest
import torch

from tests import cache_util as cu
from tests.gpu_util import torch_cuda

pytestmark = pytest.mark.gpu

EPS32 = 2.0 ** -24          # half a float32 step
EPS = {"bf16": 2.0 ** -8, "f32": EPS32}   # half a step of the type


def ctx_of(s, **kw):
    torch_cuda()
    import paper_2608_01845_amd as wdc
    return wdc, wdc.Context(cu.config(s.dtype, s.heads, s.hd, **kw), allocate_weights=False)


def within(got, want, bound, what):
    got, want = got.double(), want.double()
    bad = ~((got - want).abs() <= bound)
    bad &= ~(torch.isnan(got) & torch.isnan(want)) & ~(got == want)
    assert not bad.any(), (what, int(bad.sum()), got[bad][:4].tolist(), want[bad][:4].tolist())


def few(x):
    """A list in a test's name: itself, or its length."""
    return x if len(x) <= 8 else f"{len(x)}seqs"


# more sequences than a wave has lanes: chunks of none to three rows, caches of none to 85 keys
MANY_Q = [(3 * i + i // 7) % 4 for i in range(150)]
MANY_KV = [q + 11 * i % 83 for i, q in enumerate(MANY_Q)]

# ---------------------------------------------------------------- append


def append64(s, qk_norm, qw, kw, pos, rope):
    x = s.qkv.double().reshape(s.rows, s.heads + 2 * s.kvh, s.hd).clone()
    qk = x[:, :s.heads + s.kvh]
    if qk_norm:
        qk /= torch.sqrt(qk.square().mean(2, keepdim=True) + 1e-6)
    if qw is not None:
        qk[:, :s.heads] *= qw.double()
    if kw is not None:
        qk[:, s.heads:] *= kw.double()
    size = torch.sqrt(qk[..., 0::2] ** 2 + qk[..., 1::2] ** 2).repeat_interleave(2, 2)
    if pos is not None and sum(rope):
        p = 0
        for ax, d in enumerate(rope):
            for j in range(d // 2):
                ang = torch.where(pos[:, 0] < 0, 0, pos[:, ax].double() * 10000.0 ** (-2 * j / d))[:, None]
                a, b = qk[..., 2 * p].clone(), qk[..., 2 * p + 1].clone()
                qk[..., 2 * p] = a * torch.cos(ang) - b * torch.sin(ang)
                qk[..., 2 * p + 1] = a * torch.sin(ang) + b * torch.cos(ang)
                p += 1
    return x, size


APPEND = [
    # dtype, heads, kvh, hd, page, q, kv, qk_norm, weights, pos, rope
    ("bf16", 4, 4, 64, 16, [1], [1], True, False, "near", None),
    ("bf16", 4, 2, 64, 16, [5, 0, 1, 33], [5, 7, 100, 40], True, True, "near", None),
    ("bf16", 6, 2, 128, 64, [70, 1300], [200, 1311], True, True, "far", None),
    ("bf16", 3, 1, 128, 256, [17], [300], False, False, "near", None),
    ("bf16", 4, 4, 128, 32, [9], [9], True, False, None, None),
    ("bf16", 4, 4, 64, 32, [9, 40], [30, 64], True, False, "near", (0, 0, 0)),
    ("bf16", 4, 4, 64, 32, [50, 3], [20, 3], True, False, "near", (32, 16, 16)),   # a chunk longer than its cache
    ("f32", 4, 2, 64, 16, [5, 0, 1, 33], [5, 7, 100, 40], True, True, "far", None),
    ("f32", 5, 5, 128, 128, [1500], [1501], True, False, "far", None),
    ("bf16", 4, 2, 64, 16, MANY_Q, MANY_KV, True, False, "near", None),
    ("f32", 4, 2, 64, 16, [7 * x for x in MANY_Q], [7 * x for x in MANY_KV], True, True, "near", None),
]


@pytest.mark.parametrize("case", APPEND, ids=lambda c: f"{c[0]}-{c[1]}x{c[2]}x{c[3]}-p{c[4]}-{few(c[5])}")
def test_append_matches_definition(case):
    dtype, heads, kvh, hd, page, q, kv, norm, weights, pos, rope = case
    s = cu.state(dtype, heads, kvh, hd, page, q, kv, seed=1, tail_rows=2)
    rope = cu.ROPE[hd] if rope is None else rope
    wdc, ctx = ctx_of(s, qk_norm=norm, rope=rope)
    g = torch.Generator().manual_seed(2)
    qw = kw = None
    if weights:
        qw, kw = ((1 + 0.2 * torch.randn(hd, generator=g)).cuda() for _ in range(2))
    p = None
    if pos is not None:
        base = 2 ** 30 if pos == "far" else 0
        p = torch.randint(0, 2000, (s.rows, 3), generator=g).to(torch.int32)
        p[:, 0] += base
        p[3::7, 0] = -1
        p = p.cuda()
    k0, v0 = s.k.clone(), s.v.clone()
    out = torch.full((s.rows, heads * hd), 7.0, dtype=s.td, device="cuda")
    ctx.cache_append(wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s), s.qkv, out, pos=p, q_weight=qw, k_weight=kw)
    want, size = append64(s, norm, qw, kw, p, rope)
    # one rounding to the type, and float32 arithmetic: a sum of hd squares, root, quotient (together under
    # (hd / 8 + 8) steps), cosine and sine (2^-22 with the angle's reduction), products and sum (3 steps)
    tol = EPS[dtype] * want[:, :heads + kvh].abs() + size * ((hd / 8 + 16) * EPS32 + 2.0 ** -22)
    n = sum(q)
    within(out[:n], want[:n, :heads].reshape(n, -1), tol[:n, :heads].reshape(n, -1), "q")
    assert (out[n:] == 7).all()                       # rows of no chunk
    first = 0
    for b, (m, c) in enumerate(zip(q, kv)):
        lo = max(0, m - c)                            # rows with a slot
        pg, sl = cu.where(s, b)
        at = (pg[c - m + lo:], slice(None), sl[c - m + lo:])
        rows = slice(first + lo, first + m)
        within(s.k[at], want[rows, heads:heads + kvh], tol[rows, heads:], "k")
        assert torch.equal(s.v[at], s.qkv[rows].reshape(-1, heads + 2 * kvh, hd)[:, heads + kvh:])
        k0[at], v0[at] = s.k[at], s.v[at]
        first += m
    assert torch.equal(k0.nan_to_num(9), s.k.nan_to_num(9)) and torch.equal(v0.nan_to_num(9), s.v.nan_to_num(9))


def test_append_in_place_strided_and_bad_pages():
    s = cu.state("bf16", 4, 2, 64, 16, [40], [60], seed=3)
    wdc, ctx = ctx_of(s)
    pos = torch.arange(120, device="cuda", dtype=torch.int32).reshape(40, 3).contiguous()
    ref_k, ref_v = s.k.clone(), s.v.clone()
    ref = torch.empty_like(s.x)
    ctx.cache_append(wdc.PagedCache(ref_k, ref_v), cu.chunks(wdc, s), s.qkv, ref, pos=pos)
    wide = torch.zeros((40, 1024), dtype=torch.bfloat16, device="cuda")
    wide[:, 64:64 + 512] = s.qkv
    ctx.cache_append(wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s), wide[:, 64:64 + 512], wide[:, 64:64 + 256], pos=pos)
    assert torch.equal(wide[:, 64:320], ref) and (wide[:, :64] == 0).all() and (wide[:, 576:] == 0).all()
    assert torch.equal(s.k.nan_to_num(9), ref_k.nan_to_num(9)) and torch.equal(s.v.nan_to_num(9), ref_v.nan_to_num(9))
    # entries that are not pages: their rows are dropped, nothing else is written
    s2 = cu.state("bf16", 4, 2, 64, 16, [40], [60], seed=3)
    s2.table[0, 2], s2.table[0, 3] = -5, s2.pages
    k0 = s2.k.clone()
    out = torch.empty_like(ref)
    ctx.cache_append(wdc.PagedCache(s2.k, s2.v), cu.chunks(wdc, s2), s2.qkv, out, pos=pos)
    assert torch.equal(out, ref)
    p1 = int(s2.table[0, 1])
    k0[p1] = ref_k[p1]
    assert torch.equal(s2.k.nan_to_num(9), k0.nan_to_num(9))


# ---------------------------------------------------------------- attention


def attention_bound(s, pv, o, qk, n):
    """What rounding may add to o: the weights' rounding to the type of the product with v (bf16) and the
    result's; scores off by ds (hd products and their sum in float32, q scaled in float32, the argument's
    scaling and the exponential) move weights and their sum by ds each; n terms are added in float32."""
    ds = (s.hd + 8) * EPS32 * qk + 2.0 ** -21
    rel = 2 * ds + 2 * (n + 8) * EPS32 + (EPS["bf16"] if s.dtype == "bf16" else 0)
    return rel[..., None] * pv + EPS[s.dtype] * o.abs() + 1e-30, ds + 2 * (n + 8) * EPS32


ATTENTION = [
    # dtype, heads, kvh, hd, page, q, kv, frame
    ("bf16", 2, 2, 64, 16, [1], [1], 0),
    ("bf16", 4, 4, 64, 64, [1, 1, 1], [70, 1, 1000], 1),
    ("bf16", 8, 2, 128, 64, [1, 1, 1, 1], [700, 64, 33, 4097], 1),
    ("bf16", 16, 1, 64, 128, [2, 1], [300, 5], 1),
    ("bf16", 4, 4, 128, 16, [100], [333], 0),
    ("bf16", 4, 4, 64, 32, [300], [300], 1),
    ("bf16", 6, 2, 64, 16, [77, 1, 0, 130, 40], [500, 1, 40, 1033, 25], 1),     # an empty chunk; rows that see nothing
    ("bf16", 6, 2, 128, 256, [65, 0, 200], [65, 9, 900], 7),
    ("bf16", 3, 3, 128, 32, [520], [1500], 128),
    ("bf16", 2, 1, 64, 64, [33, 10], [0, 4], 3),                                  # no keys at all
    ("f32", 4, 4, 64, 16, [1, 1], [1, 300], 1),
    ("f32", 4, 2, 64, 32, [100, 0, 33], [400, 5, 33], 1),
    ("f32", 3, 1, 128, 64, [70, 40], [333, 25], 16),
    ("f32", 2, 2, 128, 16, [20], [0], 0),
    ("bf16", 4, 2, 64, 16, MANY_Q, MANY_KV, 1),
    ("bf16", 4, 1, 128, 16, [20 * x for x in MANY_Q], [20 * x for x in MANY_KV], 7),
    ("f32", 4, 2, 64, 16, MANY_Q, MANY_KV, 2),
]
ids = lambda c: f"{c[0]}-{c[1]}x{c[2]}x{c[3]}-p{c[4]}-{few(c[5])}-{few(c[6])}-f{c[7]}"  # noqa: E731


@pytest.mark.parametrize("case", ATTENTION, ids=ids)
def test_attention_matches_definition(case):
    check_attention(case)


def check_attention(case):
    dtype, heads, kvh, hd, page, q, kv, frame = case
    s = cu.state(dtype, heads, kvh, hd, page, q, kv, seed=5, tail_rows=3)
    wdc, ctx = ctx_of(s)
    o, lse, pv, qk = cu.attention64(s, frame)
    bound, lse_bound = attention_bound(s, pv, o, qk, max(max(kv), 1))
    n = sum(q)
    for with_lse in (True, False):
        out = torch.full_like(s.x, 7.0)
        z = torch.full((s.rows, heads), 7.0, device="cuda") if with_lse else None
        ctx.cache_attention(wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s), s.x, out, frame=frame, lse=z)
        within(out[:n], o[:n].reshape(n, -1), bound[:n].reshape(n, -1), "o")
        assert (out[n:] == 7).all()
        if with_lse:
            within(z[:n], lse[:n], lse_bound[:n] + 4 * EPS32 * lse[:n].abs(), "lse")
            assert (z[n:] == 7).all()


# Rows enough for blocks of 256 (16 query heads per kv head): each head dim, pages shorter than a tile of 64
# keys and not, one range and several, a short sequence beside a long one
ATTENTION_WIDE = [
    ("bf16", 16, 1, 64, 16, [4090], [4200], 64),
    ("bf16", 16, 1, 64, 64, [2500, 0, 2000], [3000, 40, 2001], 7),
    ("bf16", 16, 1, 64, 128, [2500, 2000], [9000, 100], 100),     # ranges; rows before the first key
    ("bf16", 16, 1, 128, 32, [2600, 2500], [2700, 2650], 0),
    ("bf16", 16, 1, 128, 256, [4000, 96], [4050, 700], 33),
    ("bf16", 12, 1, 128, 16, [5000], [5200], 1000),               # a group that does not divide the block's rows
    ("bf16", 16, 16, 64, 64, [1024], [8192], 256),                # ranges of blocks of 256
    ("bf16", 16, 16, 128, 32, [1024], [8192], 0),
    ("bf16", 16, 16, 64, 128, [384], [3457], 1),                  # blocks of 128, an odd number of tiles of 64
    ("bf16", 4, 4, 64, 16, [1000, 130], [1000, 4001], 1),
    ("bf16", 16, 16, 128, 64, [200, 64], [2000, 1999], 64),
]


@pytest.mark.parametrize("case", ATTENTION_WIDE, ids=ids)
def test_attention_of_many_rows_matches_definition(case):
    check_attention(case)


@pytest.mark.parametrize("dtype,hd,q,kv,frame", [("bf16", 64, [40], [200], 8), ("bf16", 128, [1, 90], [5, 91], 1),
                                                  ("bf16", 128, [600], [700], 64), ("f32", 64, [40], [100], 8),
                                                  ("f32", 128, [33], [40], 1)])
def test_attention_unseen_keys_have_no_influence(dtype, hd, q, kv, frame):
    """Infinities and NaN in keys that only later rows see change later rows only."""
    s = cu.state(dtype, 4, 2, hd, 32, q, kv, seed=6)
    for b in range(len(q)):
        pg, sl = cu.where(s, b)
        j = kv[b] - q[b] // 2 - 1                     # in the chunk: seen from its middle on
        s.v[pg[j], 0, sl[j], 3] = math.nan
        s.v[pg[j], 1, sl[j], 1] = math.inf
        s.k[pg[-1], 1, sl[-1], 5] = math.nan
    wdc, ctx = ctx_of(s)
    o, lse, pv, qk = cu.attention64(s, frame)
    bound, lse_bound = attention_bound(s, pv.nan_to_num(1e30, 1e30, 1e30), o.nan_to_num(0, 0, 0), qk, max(kv))
    out, z = torch.empty_like(s.x), torch.empty((s.rows, 4), device="cuda")
    ctx.cache_attention(wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s), s.x, out, frame=frame, lse=z)
    assert torch.isnan(o).any() and torch.isfinite(o).any()
    got, want = out.reshape(o.shape).double(), o
    fine = torch.isfinite(want)
    assert torch.equal(fine, torch.isfinite(got))
    within(got[fine], want[fine], bound[fine], "o")
    fine = torch.isfinite(lse)
    within(z[fine], lse[fine], (lse_bound + 4 * EPS32 * lse.abs())[fine], "lse")


@pytest.mark.parametrize("heads,kvh,hd,q", [(4, 4, 64, 1), (4, 2, 128, 7), (4, 4, 64, 40), (4, 4, 128, 40), (4, 2, 64, 200),
                                           (4, 2, 128, 200), (16, 1, 64, 4090), (16, 1, 128, 4090)])
def test_attention_over_one_key_is_its_value(heads, kvh, hd, q):
    """The first row of a chunk at the start of a cache sees one key: whatever its weight's rounding, the result is v. (The
    weight over its sum is 1 up to a few float32 steps, which do not reach half a bf16 step.)"""
    s = cu.state("bf16", heads, kvh, hd, 16, [q, 1], [q, 1], seed=28, scale=1.3)
    wdc, ctx = ctx_of(s)
    out = ctx.cache_attention(wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s), s.x, torch.empty_like(s.x), frame=1)
    for b, row in ((0, 0), (1, q)):
        pg, sl = cu.where(s, b)
        v = s.v[pg[0], :, sl[0]].repeat_interleave(heads // kvh, 0)
        assert torch.equal(out[row].reshape(heads, hd), v)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_large_scores_and_rising_maxima(dtype):
    """Scores of some hundreds, rising along the keys: the softmax reference has to move, late and far."""
    s = cu.state(dtype, 2, 2, 64, 64, [20], [900], seed=7)
    pg, sl = cu.where(s, 0)
    ramp = torch.linspace(0.1, 40, 900, device="cuda")[:, None, None].to(s.td)
    s.k[pg, :, sl] = s.k[pg, :, sl].abs() * ramp
    s.x = s.x.abs()
    s.x[10:] *= -1
    wdc, ctx = ctx_of(s)
    o, lse, pv, qk = cu.attention64(s, 0)
    bound, lse_bound = attention_bound(s, pv, o, qk, 900)
    out, z = torch.empty_like(s.x), torch.empty((s.rows, 2), device="cuda")
    ctx.cache_attention(wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s), s.x, out, lse=z)
    within(out.reshape(o.shape), o, bound, "o")
    within(z, lse, lse_bound + 4 * EPS32 * lse.abs(), "lse")


def test_attention_wrong_bounds_and_bad_pages_stay_in_the_buffers():
    """Lengths past the host's bounds are cut; entries that are no page read one; strided q and out; any scratch."""
    s = cu.state("bf16", 4, 2, 64, 16, [30, 20], [100, 60], seed=8, fill=0.5)
    wdc, ctx = ctx_of(s)
    cache = wdc.PagedCache(s.k, s.v)
    full = ctx.cache_attention(cache, cu.chunks(wdc, s), s.x, torch.empty_like(s.x), frame=1)
    wide = torch.zeros((50, 1024), dtype=torch.bfloat16, device="cuda")
    wide[:, 8:264] = s.x
    ctx.cache_attention(cache, cu.chunks(wdc, s), wide[:, 8:264], wide[:, 512:768], frame=1)
    assert torch.equal(wide[:, 512:768], full) and (wide[:, 768:] == 0).all() and (wide[:, 264:512] == 0).all()
    out = torch.full_like(s.x, 7.0)
    ctx.cache_attention(cache, cu.chunks(wdc, s, max_q=25), s.x, out, frame=1)
    assert (out[25:30] == 7).all() and torch.equal(out[:25], full[:25]) and torch.equal(out[30:], full[30:])
    s.kv_len[0] = 1 << 30
    s.kv_len[1] = -4
    s.q_start[2] = 1 << 30
    s.table[0, 1], s.table[0, 2] = -7, 1 << 30
    out = torch.full_like(s.x, 7.0)
    ctx.cache_attention(cache, cu.chunks(wdc, s), s.x, out, frame=1)
    assert torch.isfinite(out).all() and (out[30:] == 0).all()


# ---------------------------------------------------------------- accumulated weights


@pytest.mark.parametrize("case", [c for c in ATTENTION if max(c[6])] + [
    ("bf16", 12, 1, 64, 64, [700], [900], 0), ("f32", 8, 1, 64, 64, [300], [90], 0)], ids=ids)
@pytest.mark.parametrize("decay", [0.0, 0.75])
def test_mass_matches_definition(case, decay):
    dtype, heads, kvh, hd, page, q, kv, frame = case
    s = cu.state(dtype, heads, kvh, hd, page, q, kv, seed=9, tail_rows=1)
    wdc, ctx = ctx_of(s)
    _, lse, _, qk = cu.attention64(s, frame)
    lse = lse.float()
    want, add = cu.mass64(s, frame, lse, decay)
    out = torch.full_like(s.mass, 7.0)
    ctx.cache_mass(wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s), s.x, lse, s.mass, frame=frame, decay=decay, out=out)
    # exponents off by the scores' and the argument's rounding, sums of rows x group terms in float32
    big = lse[torch.isfinite(lse)].abs().max().item() if torch.isfinite(lse).any() else 0.0
    rel = (hd + 8) * EPS32 * qk.max().item() + 4 * EPS32 * (big + qk.max().item()) + 2.0 ** -21
    rel += (max(q) * heads / kvh + 8) * EPS32
    for b, n in enumerate(kv):
        pg, sl = cu.where(s, b)
        within(out[pg, :, sl], want[pg, :, sl], rel * add[pg, :, sl] + 4 * EPS32 * want[pg, :, sl].abs(), "mass")
        want[pg, :, sl] = 7.0
        out[pg, :, sl] = 7.0
    assert (out == 7).all()                           # slots of no key
    # in place
    m = s.mass.clone()
    ctx.cache_mass(wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s), s.x, lse, m, frame=frame, decay=decay)
    ref = torch.full_like(m, 7.0)
    ctx.cache_mass(wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s), s.x, lse, s.mass, frame=frame, decay=decay, out=ref)
    for b in range(len(kv)):
        pg, sl = cu.where(s, b)
        assert torch.equal(m[pg, :, sl], ref[pg, :, sl])


def test_mass_of_all_keys_is_the_number_of_rows():
    s = cu.state("bf16", 8, 2, 128, 64, [300], [2000], seed=10, scale=1.5)
    wdc, ctx = ctx_of(s)
    cache, ch = wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s)
    lse = torch.empty((s.rows, 8), device="cuda")
    ctx.cache_attention(cache, ch, s.x, torch.empty_like(s.x), frame=100, lse=lse)
    out = ctx.cache_mass(cache, ch, s.x, lse, s.mass, frame=100, decay=0.0, out=torch.zeros_like(s.mass))
    pg, sl = cu.where(s, 0)
    total = out[pg, :, sl].double().sum(0)
    assert torch.allclose(total, torch.full_like(total, 300 * 4), rtol=1e-4, atol=0)


# ---------------------------------------------------------------- eviction


EVICT = [
    # dtype, kvh, hd, page, kv, keep, sink, recent, masses
    ("bf16", 2, 64, 16, [100, 30, 31, 0, 64], 30, 4, 10, "random"),
    ("bf16", 1, 128, 64, [5000], 1, 0, 0, "random"),
    ("bf16", 2, 128, 32, [1500, 700], 600, 0, 0, "ties"),
    ("bf16", 2, 64, 64, [1500], 1000, 300, 700, "random"),          # nothing left to choose
    ("bf16", 1, 64, 256, [2100], 2000, 0, 1900, "equal"),
    ("bf16", 2, 64, 16, [300], 100, 10, 20, "odd"),
    ("f32", 3, 64, 16, [100, 200], 64, 0, 33, "ties"),
    ("f32", 1, 128, 128, [900], 899, 1, 1, "random"),
    ("bf16", 1, 64, 64, [70000], 40000, 1000, 2000, "random"),
    ("bf16", 2, 64, 16, [6000, 200, 4501, 0], 4500, 1000, 3500, "random"),
    ("bf16", 2, 64, 32, [9000, 4000, 5000], 4200, 100, 200, "odd"),
    ("f32", 1, 64, 64, [9000], 17, 5, 6, "ties"),
    ("bf16", 1, 128, 256, [9000, 8999], 8990, 0, 0, "equal"),
    ("bf16", 64, 64, 64, [4200] * 4, 4000, 10, 20, "ties"),
    ("bf16", 2, 64, 16, MANY_KV, 20, 3, 4, "random"),
    ("bf16", 2, 64, 16, [1024, 1000, 257, 255, 64, 65], 250, 3, 4, "odd"),       # blocks of 256 threads
    ("bf16", 2, 64, 16, [1024, 700], 600, 0, 0, "near"),
    ("bf16", 2, 64, 16, [1025, 700], 600, 0, 0, "ties"),
    ("bf16", 128, 64, 64, [2048, 2000, 1999, 3], 1500, 700, 800, "equal"),
    ("bf16", 128, 64, 64, [2048, 2000, 1999, 3], 1500, 7, 80, "ties"),
    ("bf16", 2, 64, 64, [30000, 9000, 21000], 20000, 100, 200, "near"),
    ("f32", 1, 64, 32, [40000], 12345, 0, 0, "near"),
    ("bf16", 1, 64, 32, [40000], 39000, 50, 60, "ties"),
]


@pytest.mark.parametrize("case", EVICT, ids=lambda c: f"{c[0]}-{c[1]}x{c[2]}-p{c[3]}-{few(c[4])}-keep{c[5]}-{c[6]}-{c[7]}-{c[8]}")
@pytest.mark.parametrize("in_place", [False, True])
def test_evict_matches_definition(case, in_place):
    dtype, kvh, hd, page, kv, keep, sink, recent, kind = case
    s = cu.state(dtype, kvh, kvh, hd, page, [0] * len(kv), kv, seed=11)
    if kind == "ties":
        s.mass = torch.round(s.mass)
    elif kind == "near":                               # distinct, within a factor of 1.2
        s.mass = torch.where(torch.isnan(s.mass), s.mass, 1 + 0.2 * torch.rand_like(s.mass))
    elif kind == "equal":
        s.mass = torch.where(torch.isnan(s.mass), s.mass, 0.5)
    elif kind == "odd":
        m = s.mass.reshape(-1)
        live = torch.nonzero(~torch.isnan(m))[:, 0]
        for i, x in enumerate((math.nan, math.inf, -math.inf, -0.0, 0.0, -3.0, 1e-42)):
            m[live[i::9]] = x
    wdc, ctx = ctx_of(s)
    want = cu.evict64(s, s.mass, keep, sink, recent)
    k0, v0, m0 = s.k.clone(), s.v.clone(), s.mass.clone()
    ch = cu.chunks(wdc, s, rows=0, max_q=0)
    index = torch.full((len(kv), kvh, keep), -9, dtype=torch.int32, device="cuda")
    out = s.mass if in_place else torch.full_like(s.mass, 7.0)
    new_len = s.kv_len if in_place else torch.empty_like(s.kv_len)
    ctx.cache_evict(wdc.PagedCache(s.k, s.v), ch, s.mass, keep, sink, recent, kv_len_out=None if in_place else new_len,
                    index=index, out=None if in_place else out)
    assert new_len.tolist() == [min(n, keep) for n in kv]
    touched = torch.zeros(s.mass.shape, dtype=torch.bool, device="cuda")
    for b, n in enumerate(kv):
        pg, sl = cu.where(s, b)
        live = min(n, keep)
        for h in range(kvh):
            assert index[b, h].tolist() == want[b][h] + [-1] * (keep - live)
            src = torch.tensor(want[b][h], dtype=torch.long, device="cuda")
            for now, before in ((s.k, k0), (s.v, v0), (out, m0)):
                assert torch.equal(now[pg[:live], h, sl[:live]].nan_to_num(9, 8, -8),
                                   before[pg[src], h, sl[src]].nan_to_num(9, 8, -8))
            touched[pg[:live], h, sl[:live]] = True
    for now, before in ((s.k, k0), (s.v, v0)) + (() if not in_place else ((out, m0),)):
        assert torch.equal(now[~touched].nan_to_num(9, 8, -8), before[~touched].nan_to_num(9, 8, -8))
    if not in_place:
        assert (out[~touched] == 7).all()


def test_evict_bad_pages_are_not_written():
    s = cu.state("bf16", 2, 2, 64, 16, [0], [200], seed=12, fill=0.25)
    wdc, ctx = ctx_of(s)
    s.table[0, 1], s.table[0, 9] = -1, s.pages + 3
    k0, m0 = s.k.clone(), s.mass.clone()
    ctx.cache_evict(wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s, rows=0, max_q=0), s.mass, 100, 0, 50)
    own = torch.zeros(s.pages, dtype=torch.bool)
    own[[int(p) for p in s.table[0].tolist() if 0 <= p < s.pages]] = True
    assert torch.equal(s.k[~own.cuda()], k0[~own.cuda()]) and torch.equal(s.mass[~own.cuda()], m0[~own.cuda()])
    assert s.kv_len.tolist() == [100]


# ---------------------------------------------------------------- edges of all four


def run_all(ctx, wdc, s, frame=5, keep=20, **kw):
    """append, attention, mass, eviction on state s; every result."""
    cache, ch = wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s, **kw)
    q, out = torch.full_like(s.x, 7.0), torch.full_like(s.x, 7.0)
    lse = torch.full((s.rows, s.heads), 7.0, device="cuda")
    pos = torch.arange(3 * s.rows, dtype=torch.int32, device="cuda").reshape(s.rows, 3)
    index = torch.empty((len(s.q), s.kvh, keep), dtype=torch.int32, device="cuda")
    ctx.cache_append(cache, ch, s.qkv, q, pos=pos)
    ctx.cache_attention(cache, ch, q, out, frame=frame, lse=lse)
    ctx.cache_mass(cache, ch, q, lse, s.mass, frame=frame, decay=0.5)
    mass = s.mass.clone()
    ctx.cache_evict(cache, ch, s.mass, keep, 3, 4, index=index)
    return q, out, lse, mass, index


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_rows_and_no_keys(dtype):
    """Calls without rows change masses by the decay only; rows over no keys at all get zeros, however many they are."""
    s = cu.state(dtype, 4, 2, 64, 16, [0, 0], [30, 0], seed=21)
    wdc, ctx = ctx_of(s)
    k0, m0 = s.k.clone(), s.mass.clone()
    run_all(ctx, wdc, s, keep=40)
    assert torch.equal(s.k.nan_to_num(9), k0.nan_to_num(9))
    pg, sl = cu.where(s, 0)
    assert torch.equal(s.mass[pg, :, sl], 0.5 * m0[pg, :, sl])
    for rows in (5, 20, 300, 2000):
        s = cu.state(dtype, 4, 1, 64, 16, [rows], [0], seed=22)
        q, out, lse, _, index = run_all(ctx_of(s)[1], wdc, s, keep=40)
        assert torch.isfinite(q).all() and (out == 0).all() and (lse == -math.inf).all() and (index == -1).all()


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("f32", 64)])
def test_pool_beyond_32_bit_offsets(dtype, hd):
    """Pages past 4 GiB of a pool: the results of the same pages in a small pool."""
    q, kv, page = [3, 200], [400, 300], 64
    small = cu.state(dtype, 4, 2, hd, page, q, kv, seed=23, fill=0.0)
    wdc, ctx = ctx_of(small)
    td = small.td
    pages = (1 << 33) // (2 * page * hd * td.itemsize)            # 8 GiB each of k and v
    far = torch.tensor([pages - 1 - 37 * i for i in range(small.pages)], device="cuda")
    big = cu.state(dtype, 4, 2, hd, page, q, kv, seed=23, fill=0.0)
    big.k, big.v = (torch.empty((pages, 2, page, hd), dtype=td, device="cuda") for _ in range(2))
    big.mass = torch.zeros((pages, 2, page), device="cuda")
    big.k[far], big.v[far], big.mass[far] = small.k, small.v, small.mass
    big.table = torch.where(small.table < 0, -1, far[small.table.clamp(min=0).long()]).to(torch.int32)
    for a, b in zip(run_all(ctx, wdc, small, keep=250), run_all(ctx, wdc, big, keep=250)):
        assert torch.equal(a, b[far] if a.shape != b.shape else b)
    for a, b in ((small.k, big.k), (small.v, big.v), (small.mass, big.mass)):
        assert torch.equal(a, b[far])


@pytest.mark.parametrize("dtype,heads,kvh,hd,q,kv", [("bf16", 4, 4, 64, 3, 900), ("bf16", 6, 2, 128, 40, 300),
                                                     ("bf16", 16, 1, 64, 300, 700), ("f32", 4, 2, 64, 50, 400)])
def test_attention_in_place_shared_pages_and_a_long_frame(dtype, heads, kvh, hd, q, kv):
    """out may be q; two sequences may share the pages of their past; a frame longer than any chunk is one frame."""
    s = cu.state(dtype, heads, kvh, hd, 16, [q, q], [kv, kv], seed=24, fill=0.0)
    shared = (kv - q) // 16
    s.table[1, :shared] = s.table[0, :shared]
    wdc, ctx = ctx_of(s)
    cache, ch = wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s)
    o, lse, pv, qk = cu.attention64(s, 0)
    bound, _ = attention_bound(s, pv, o, qk, kv)
    ref = ctx.cache_attention(cache, ch, s.x, torch.empty_like(s.x))
    within(ref.reshape(o.shape), o, bound, "o")
    assert torch.equal(ref, ctx.cache_attention(cache, ch, s.x, torch.empty_like(s.x), frame=0x7fffffff))
    x = s.x.clone()
    ctx.cache_attention(cache, ch, x, x)
    assert torch.equal(x, ref)


@pytest.mark.parametrize("dtype,heads,kvh,hd,q,kv", [("bf16", 4, 4, 128, [1, 1], [9000, 5000]), ("bf16", 4, 4, 64, [300], [9000]),
                                                     ("bf16", 4, 2, 128, [700, 90], [3000, 2000]),
                                                     ("bf16", 2, 2, 64, [40, 3], [4000, 9000]), ("f32", 4, 2, 64, [50], [4000])])
def test_less_scratch_and_no_byte_behind_it(dtype, heads, kvh, hd, q, kv):
    """Attention and masses with all, half, a seventh and none of the scratch; eviction with exactly its own."""
    import ctypes as C
    s = cu.state(dtype, heads, kvh, hd, 16, q, kv, seed=26)
    wdc, ctx = ctx_of(s)
    lib, cache, ch = ctx.lib, wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s)
    o, lse, pv, qk = cu.attention64(s, 7)
    bound, lse_bound = attention_bound(s, pv, o, qk, max(kv))
    z32 = lse.float()
    want, add = cu.mass64(s, 7, z32, 0.5)
    ld, ptr = heads * hd, lambda t: C.c_void_p(t.data_ptr())
    rel = (hd + 8) * EPS32 * qk.max().item() + 4 * EPS32 * (lse.abs().max().item() + qk.max().item()) + 2.0 ** -21
    rel += (max(q) * heads / kvh + 8) * EPS32
    need = lib.wdc_cache_attention_scratch(ctx.h, cache.ref, ch.ref)
    need_m = lib.wdc_cache_mass_scratch(ctx.h, cache.ref, ch.ref)
    assert need > 0

    def area(n):
        return torch.full((n + 4096,), 0x5a, dtype=torch.uint8, device="cuda")

    for part in (1, 2, 7, 0):
        n, m = (need // part // 16 * 16, need_m // part // 16 * 16) if part else (0, 0)
        mem, out, z = area(n), torch.full_like(s.x, 7.0), torch.empty((s.rows, heads), device="cuda")
        assert lib.wdc_cache_attention(ctx.h, cache.ref, ch.ref, ptr(s.x), ld, 7, ptr(out), ld, ptr(z), ptr(mem) if n else None,
                                       n) == 0
        within(out.reshape(o.shape), o, bound, "o")
        within(z, lse, lse_bound + 4 * EPS32 * lse.abs(), "lse")
        assert (mem[n:] == 0x5a).all()
        mem, got = area(m), torch.zeros_like(s.mass)
        assert lib.wdc_cache_mass(ctx.h, cache.ref, ch.ref, ptr(s.x), ld, 7, ptr(z32), 0.5, ptr(s.mass), ptr(got),
                                  ptr(mem) if m else None, m) == 0
        for b in range(len(kv)):
            pg, sl = cu.where(s, b)
            within(got[pg, :, sl], want[pg, :, sl], rel * add[pg, :, sl] + 4 * EPS32 * want[pg, :, sl].abs(), "mass")
        assert (mem[m:] == 0x5a).all()
    n = lib.wdc_cache_evict_scratch(ctx.h, cache.ref, ch.ref, 2000)
    mem, index = area(n), torch.empty((len(kv), kvh, 2000), dtype=torch.int32, device="cuda")
    want_idx = cu.evict64(s, s.mass, 2000, 5, 6)
    assert lib.wdc_cache_evict(ctx.h, cache.ref, ch.ref, ptr(s.mass), ptr(s.mass), 2000, 5, 6, ptr(s.kv_len), ptr(index), ptr(mem),
                               n) == 0
    assert index.tolist() == want_idx and (mem[n:] == 0x5a).all()


def test_bounds_that_32_bits_would_cut_are_refused():
    s = cu.state("bf16", 4, 2, 64, 16, [2], [20], seed=25)
    wdc, ctx = ctx_of(s)
    cache, ch, x = wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s), s.x
    lse = torch.zeros((2, 4), device="cuda")
    for frame in (1 << 32, -1):
        with pytest.raises(ValueError):
            ctx.cache_attention(cache, ch, x, x, frame=frame)
        with pytest.raises(ValueError):
            ctx.cache_mass(cache, ch, x, lse, s.mass, frame=frame)
    for a in (((1 << 32) + 9, 0, 0), (9, 1 << 32, 0), (9, 0, 1 << 32)):
        with pytest.raises(ValueError):
            ctx.cache_evict(cache, ch, s.mass, *a)


# ---------------------------------------------------------------- together


@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_rollout_of_chunks_append_attend_accumulate_evict(dtype, hd):
    """Two sequences, chunks of two frames each, a bounded cache; every step against float64 on the cache as it is."""
    heads, kvh, page, frame, n = 4, 2, 16, 20, 40
    s = cu.state(dtype, heads, kvh, hd, page, [n, n], [0, 0], seed=13, spare=40)
    s.table = torch.randperm(40, generator=torch.Generator().manual_seed(1))[:24].to(torch.int32).reshape(2, 12).cuda()
    s.mass.fill_(math.nan)
    wdc, ctx = ctx_of(s)
    g = torch.Generator().manual_seed(3)
    out, lse = torch.empty((2 * n, heads * hd), dtype=s.td, device="cuda"), torch.empty((2 * n, heads), device="cuda")
    index = torch.empty((2, kvh, 120), dtype=torch.int32, device="cuda")
    for step in range(6):
        qkv = torch.randn((2 * n, (heads + 2 * kvh) * hd), generator=g).to(s.td).cuda()
        i = torch.arange(2 * n) % n
        pos = torch.stack([2 * step + i // frame, i % frame // 5, i % 5], 1).to(torch.int32).cuda()
        before = s.mass.clone()
        prev = s.kv_len.tolist()
        s.kv_len += n
        cache = wdc.PagedCache(s.k, s.v)
        ch = wdc.Chunks(s.q_start, s.kv_len, s.table, rows=2 * n, max_q=2 * n, max_kv=s.table.shape[1] * page)
        q = torch.empty((2 * n, heads * hd), dtype=s.td, device="cuda")
        ctx.cache_append(cache, ch, qkv, q, pos=pos)
        ctx.cache_attention(cache, ch, q, out, frame=frame, lse=lse)
        ctx.cache_mass(cache, ch, q, lse, s.mass, frame=frame, decay=0.9)
        o, z = out, lse
        s.kv, s.x, s.q = s.kv_len.tolist(), q, [n, n]
        assert s.kv == [p + n for p in prev]
        s.rows = 2 * n
        want, want_lse, pv, qk = cu.attention64(s, frame)
        bound, lse_bound = attention_bound(s, pv, want, qk, max(s.kv))
        within(o.reshape(want.shape), want, bound, "o")
        within(z, want_lse, lse_bound + 4 * EPS32 * want_lse.abs(), "lse")
        after, s.mass = s.mass, before
        m64, add = cu.mass64(s, frame, z, 0.9)
        s.mass = after
        for b in range(2):
            pg, sl = cu.where(s, b)
            within(s.mass[pg, :, sl], m64[pg, :, sl], 1e-3 * add[pg, :, sl] + 1e-6 * m64[pg, :, sl].abs(), "mass")
        if max(s.kv) > 140:
            want_idx = cu.evict64(s, s.mass, 120, 8, n)
            ctx.cache_evict(wdc.PagedCache(s.k, s.v), wdc.Chunks(s.q_start, s.kv_len, s.table, rows=2 * n), s.mass, 120,
                            sink=8, recent=n, index=index)
            assert index.tolist() == want_idx and s.kv_len.tolist() == [120, 120]


def test_rollout_captured_and_replayed():
    """The four calls captured into one graph; replays on new inputs, with eager work between, equal the eager run."""
    heads, kvh, hd, page, n = 4, 2, 64, 16, 30
    side = torch.cuda.Stream()
    s = cu.state("bf16", heads, kvh, hd, page, [n], [200], seed=14, fill=0.0)
    import paper_2608_01845_amd as wdc
    torch_cuda()
    ctx = wdc.Context(cu.config("bf16", heads, hd), allocate_weights=False, stream=side)
    cache, ch = wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s)
    q, out = torch.empty_like(s.x), torch.empty_like(s.x)
    lse = torch.empty((n, heads), device="cuda")
    new_len = torch.empty_like(s.kv_len)
    index = torch.empty((1, kvh, 150), dtype=torch.int32, device="cuda")
    pos = torch.arange(3 * n, dtype=torch.int32, device="cuda").reshape(n, 3).contiguous()
    k0, v0, m0 = s.k.clone(), s.v.clone(), s.mass.clone()

    def calls():
        ctx.cache_append(cache, ch, s.qkv, q, pos=pos)
        ctx.cache_attention(cache, ch, q, out, frame=10, lse=lse)
        ctx.cache_mass(cache, ch, q, lse, s.mass, frame=10)
        ctx.cache_evict(cache, ch, s.mass, 150, 10, n, kv_len_out=new_len, index=index)

    def reset(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        s.qkv.copy_(torch.randn(s.qkv.shape, generator=g, device="cuda"))
        s.k.copy_(k0), s.v.copy_(v0), s.mass.copy_(m0)

    def results():
        return [t.clone() for t in (q, out, lse, s.k, s.v, s.mass, new_len, index)]

    eager = {}
    for seed in range(3):
        reset(seed)
        torch.cuda.synchronize()
        calls()
        torch.cuda.synchronize()
        eager[seed] = results()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        calls()
    for seed in (1, 2, 0, 1):
        reset(seed)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results(), eager[seed])), seed
        torch.randn(1 << 20, device="cuda").sum().item()          # eager work between replays


def test_another_stream_than_the_current_one():
    s = cu.state("bf16", 8, 2, 64, 64, [4, 4], [3000, 2500], seed=15)
    import paper_2608_01845_amd as wdc
    torch_cuda()
    side = torch.cuda.Stream()
    ref_ctx = wdc.Context(cu.config("bf16", 8, 64), allocate_weights=False)
    ctx = wdc.Context(cu.config("bf16", 8, 64), allocate_weights=False, stream=side)
    cache, ch = wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s)
    ref = ref_ctx.cache_attention(cache, ch, s.x, torch.empty_like(s.x))
    torch.cuda.synchronize()
    outs = [torch.empty_like(s.x) for _ in range(20)]
    for o in outs:
        ctx.cache_attention(cache, ch, s.x, o)
        torch.full((1 << 22,), 3.0, device="cuda")                # the current stream's allocations take what is free
    side.synchronize()
    assert all(torch.equal(o, ref) for o in outs)


def test_two_graphs_in_flight():
    """Two captured chains on the same cache, replayed on two streams at once, several times: each has its own scratch."""
    import paper_2608_01845_amd as wdc
    torch_cuda()
    s = cu.state("bf16", 8, 2, 128, 64, [4, 4], [7000, 6000], seed=27)
    ref_ctx = wdc.Context(cu.config("bf16", 8, 128), allocate_weights=False)
    cache, ch = wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s)
    xs = [s.x, s.x.flip(0).contiguous()]

    def calls(ctx, x, out, lse, mass):
        ctx.cache_attention(cache, ch, x, out, lse=lse)
        ctx.cache_mass(cache, ch, x, lse, s.mass, out=mass)

    def buffers():
        return [torch.zeros_like(s.x), torch.zeros((s.rows, 8), device="cuda"), torch.zeros_like(s.mass)]

    want, got, graphs, streams, ctxs = [], [], [], [], []
    for x in xs:
        want.append(buffers())
        calls(ref_ctx, x, *want[-1])
    torch.cuda.synchronize()
    for x in xs:
        side = torch.cuda.Stream()
        ctx = wdc.Context(cu.config("bf16", 8, 128), allocate_weights=False, stream=side)
        b = buffers()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            calls(ctx, x, *b)
        got.append(b), graphs.append(g), streams.append(side), ctxs.append(ctx)
    for _ in range(5):
        for b in got:
            for t in b:
                t.fill_(7)
        torch.cuda.synchronize()
        for _ in range(4):
            for g, st in zip(graphs, streams):
                with torch.cuda.stream(st):
                    g.replay()
        torch.cuda.synchronize()
        live = torch.zeros(s.mass.shape, dtype=torch.bool, device="cuda")
        for i in range(2):
            pg, sl = cu.where(s, i)
            live[pg, :, sl] = True
        for a, b in zip(want, got):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.equal(a[2][live], b[2][live])
