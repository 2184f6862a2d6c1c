"""The 8-bit paged cache against its definition in float64: append, read, attention, and a rollout's run of them."""
import math

import pytest
import torch

from tests import cache8_util as c8
from tests import cache_util as cu
from tests.gpu_util import torch_cuda
from tests.test_gpu_cache import (APPEND, ATTENTION, ATTENTION_WIDE, EPS, EPS32, append64, attention_bound, ctx_of, few, ids,
                                  within)

pytestmark = pytest.mark.gpu


def bits(s):
    return [t.view(torch.uint8).clone() for t in (s.k8, s.v8, s.scale)]


@pytest.mark.parametrize("case", APPEND, ids=lambda c: f"{c[0]}-{c[1]}x{c[2]}x{c[3]}-p{c[4]}-{few(c[5])}")
def test_append_matches_definition(case):
    dtype, heads, kvh, hd, page, q, kv, norm, weights, pos, rope = case
    s = c8.state8(dtype, heads, kvh, hd, page, q, kv, seed=1, tail_rows=2)
    rope = cu.ROPE[hd] if rope is None else rope
    wdc, ctx = ctx_of(s, qk_norm=norm, rope=rope)
    g = torch.Generator().manual_seed(2)
    s.qkv = (s.qkv.float() * torch.exp(2 * torch.randn((s.rows, 1), generator=g)).cuda()).to(s.td)
    qw = kw = None
    if weights:
        qw, kw = ((1 + 0.2 * torch.randn(hd, generator=g)).cuda() for _ in range(2))
    p = None
    if pos is not None:
        p = torch.randint(0, 2000, (s.rows, 3), generator=g).to(torch.int32)
        p[:, 0] += 2 ** 30 if pos == "far" else 0
        p[3::7, 0] = -1
        p = p.cuda()
    k0, v0, e0 = bits(s)
    out = torch.full((s.rows, heads * hd), 7.0, dtype=s.td, device="cuda")
    ctx.cache8_append(c8.cache8(wdc, s), cu.chunks(wdc, s), s.qkv, out, pos=p, q_weight=qw, k_weight=kw)
    want, size = append64(s, norm, qw, kw, p, rope)
    # float32 arithmetic as in the append of the cache in the model's type; then one rounding
    err = size * ((hd / 8 + 16) * EPS32 + 2.0 ** -22)
    n = sum(q)
    within(out[:n], want[:n, :heads].reshape(n, -1), (EPS[dtype] * want[:n, :heads].abs() + err[:n, :heads]).reshape(n, -1), "q")
    assert (out[n:] == 7).all()                       # rows of no chunk
    k1, v1, e1 = bits(s)
    first = 0
    for b, (m, c) in enumerate(zip(q, kv)):
        lo = max(0, m - c)                            # rows with a slot
        pg, sl = cu.where(s, b)
        at = (pg[c - m + lo:], slice(None), sl[c - m + lo:])
        rows = slice(first + lo, first + m)
        # values are moved into codes bit for bit as defined
        code, byte = c8.quantised64(s.qkv[rows].double().reshape(-1, heads + 2 * kvh, hd)[:, heads + kvh:])
        assert torch.equal(v1[at], code) and torch.equal(e1[at][..., 1], byte)
        # a key's codes are off by half a step (2^-4 of it, of code 1 to 8 half of code 1) of what float32 made of it; where
        # its largest element is within that error of a border, its power of two may be the neighbouring one
        x, e = want[rows, heads:heads + kvh], err[rows, heads:]
        power = torch.exp2(e1[at][..., :1].double() - 127)
        got = c8.values64(k1[at], e1[at][..., 0])
        within(got, x, torch.maximum((x.abs() + e) * 2.0 ** -4, power * 2.0 ** -10) + e, "k")
        big = x.abs().amax(2, keepdim=True)
        slack = e.amax(2, keepdim=True)
        assert ((big - slack <= 448 * power) & ((big + slack > 224 * power) | (e1[at][..., :1] == 10))).all()
        k0[at], v0[at], e0[at] = k1[at], v1[at], e1[at]
        first += m
    assert torch.equal(k0, k1) and torch.equal(v0, v1) and torch.equal(e0, e1)


@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
def test_append_of_extreme_values(dtype, hd):
    """Without norms and rotation keys are stored as values are: bit for bit, whatever their size."""
    s = c8.state8(dtype, 2, 2, hd, 16, [300], [300], seed=3)
    wdc, ctx = ctx_of(s, qk_norm=False, rope=(0, 0, 0))
    g = torch.Generator().manual_seed(4)
    x = torch.randn((300, 6 * hd), generator=g) * torch.exp2(torch.randint(-60, 60, (300, 1), generator=g).float())
    x[20:60] *= torch.exp2(torch.randint(-24, 1, (40, 6 * hd), generator=g).float())
    x[1] = 0
    x[2] = -0.0
    x[3, ::5], x[3, 1::5], x[3, 2::7] = math.inf, math.nan, -math.inf
    x[4] = math.nan
    x[5] = 2.0 ** -126                                # far below the smallest power
    x[6] = 448 * 2.0 ** -117
    x[7] = 2.0 ** 126
    x[8] = 1.75 * 2.0 ** torch.randint(-8, 8, (6 * hd,), generator=g).float()
    x[9] = torch.linspace(-448, 448, 6 * hd)
    x[10] = torch.tensor((c8.CODES * 8)[:6 * hd])     # every code
    mid = [(a + b) / 2 for a, b in zip(c8.CODES, c8.CODES[1:])]
    x[11] = torch.tensor((mid * 8)[:6 * hd])          # every tie
    x[10, ::hd] = x[11, ::hd] = 448
    x[12] = torch.linspace(-3.38e38, 3.38e38, 6 * hd)  # (the step is infinite: NaN and infinities)
    x[13] = 3.38e38                                   # the end of bf16's range
    x[14] = torch.linspace(-1, 1, 6 * hd) * 3.38e38
    s.qkv = x.to(s.td).cuda()
    ctx.cache8_append(c8.cache8(wdc, s), cu.chunks(wdc, s), s.qkv, torch.empty_like(s.x))
    pg, sl = cu.where(s, 0)
    rows = s.qkv.double().reshape(300, 6, hd)
    for pool, which, part in ((s.k8, 0, rows[:, 2:4]), (s.v8, 1, rows[:, 4:])):
        code, byte = c8.quantised64(part)
        got = pool.view(torch.uint8)[pg, :, sl]
        assert torch.equal(s.scale[pg, :, sl, which], byte)
        nan = (code & 127) == 127
        assert torch.equal(torch.isfinite(c8.values64(got, s.scale[pg, :, sl, which]).to(s.td)), torch.isfinite(part))
        assert torch.equal(nan, (got & 127) == 127) and torch.equal(got[~nan], code[~nan])


def test_append_in_place_strided_bad_pages_and_wrong_bounds():
    s = c8.state8("bf16", 4, 2, 64, 16, [40], [60], seed=3)
    wdc, ctx = ctx_of(s)
    pos = torch.arange(120, device="cuda", dtype=torch.int32).reshape(40, 3).contiguous()
    start, table = bits(s), s.table.clone()
    ref = ctx.cache8_append(c8.cache8(wdc, s), cu.chunks(wdc, s), s.qkv, torch.empty_like(s.x), pos=pos)
    done = bits(s)
    again = lambda: [t.view(torch.uint8).copy_(b) for t, b in zip((s.k8, s.v8, s.scale), start)]  # noqa: E731
    again()
    wide = torch.zeros((40, 1024), dtype=torch.bfloat16, device="cuda")
    wide[:, 64:64 + 512] = s.qkv
    ctx.cache8_append(c8.cache8(wdc, s), cu.chunks(wdc, s), wide[:, 64:64 + 512], wide[:, 64:64 + 256], pos=pos)
    assert torch.equal(wide[:, 64:320], ref) and (wide[:, :64] == 0).all() and (wide[:, 576:] == 0).all()
    assert all(torch.equal(a, b) for a, b in zip(bits(s), done))
    # entries that are not pages: their rows are dropped, nothing else is written
    again()
    s.table[0, 2], s.table[0, 3] = -5, s.pages
    out = ctx.cache8_append(c8.cache8(wdc, s), cu.chunks(wdc, s), s.qkv, torch.empty_like(ref), pos=pos)
    assert torch.equal(out, ref)
    p1 = int(table[0, 1])
    for a, b, c in zip(start, bits(s), done):
        a = a.clone()
        a[p1] = c[p1]
        assert torch.equal(a, b)
    # lengths past the host's bounds are cut
    again()
    s.table.copy_(table)
    s.kv_len[0], s.q_start[1] = 1 << 30, 1 << 30
    out = ctx.cache8_append(c8.cache8(wdc, s), cu.chunks(wdc, s), s.qkv, torch.empty_like(ref), pos=pos)
    assert torch.equal(out, ref) and all(torch.equal(a, b) for a, b in zip(bits(s), done))


READ = [c for c in ATTENTION if max(c[6])] + [("bf16", 16, 16, 128, 64, [2100], [2100], 0), ("f32", 12, 12, 64, 16, [1500, 700], [1600, 700], 0)]


@pytest.mark.parametrize("case", READ, ids=ids)
def test_read_gives_the_values(case):
    dtype, heads, kvh, hd, page, q, kv, _ = case
    s = c8.state8(dtype, heads, kvh, hd, page, q, kv, seed=6, tail_rows=2)
    wdc, ctx = ctx_of(s)
    cache, ch = c8.cache8(wdc, s), cu.chunks(wdc, s)
    k, v = (torch.full((s.rows, kvh * hd), 7.0, dtype=s.td, device="cuda") for _ in range(2))
    ctx.cache8_read(cache, ch, k=k, v=v)
    want_k, want_v, first = torch.full_like(k, 7.0), torch.full_like(v, 7.0), 0
    for b, (m, n) in enumerate(zip(q, kv)):
        pg, sl = cu.where(s, b)
        lo = max(0, m - n)
        for want, pool in ((want_k, s.k), (want_v, s.v)):
            want[first:first + lo] = 0                # rows of a chunk longer than its cache
            want[first + lo:first + m] = pool[pg[n - m + lo:], :, sl[n - m + lo:]].reshape(m - lo, kvh * hd)
        first += m
    assert torch.equal(k, want_k) and torch.equal(v, want_v)
    wide = torch.full((s.rows, (kvh + 2) * hd), 9.0, dtype=s.td, device="cuda")
    part = wide[:, hd:-hd]
    part.fill_(7.0)
    assert ctx.cache8_read(cache, ch, v=part)[0] is None
    assert torch.equal(part, want_v) and (wide[:, :hd] == 9).all() and (wide[:, -hd:] == 9).all()
    k.fill_(7.0)
    ctx.cache8_read(cache, ch, k=k)
    assert torch.equal(k, want_k)


def test_read_of_bad_pages_and_every_code():
    s = c8.state8("bf16", 2, 2, 64, 16, [40], [60], seed=7)
    s.k8.view(torch.uint8).copy_(torch.arange(s.k8.numel()).reshape(s.k8.shape) % 256)
    s.scale[..., 0] = (torch.arange(s.scale[..., 0].numel()) % 238 + 10).reshape(s.scale.shape[:3]).to(torch.uint8)
    c8.decode(s)
    pg, sl = cu.where(s, 0)
    want = s.k[pg, :, sl][20:].reshape(40, -1)
    s.table[0, 2], s.table[0, 3] = -5, s.pages       # slots 32 to 59
    want[12:] = 0
    for dtype in ("bf16", "f32"):
        s.dtype, s.td = dtype, torch.bfloat16 if dtype == "bf16" else torch.float32
        wdc, ctx = ctx_of(s)
        k = torch.full((40, 128), 7.0, dtype=s.td, device="cuda")
        ctx.cache8_read(c8.cache8(wdc, s), cu.chunks(wdc, s), k=k)
        got, ref = k.double(), want.double()
        assert torch.equal(got.nan_to_num(9.25, 1e300, -1e300), ref.nan_to_num(9.25, 1e300, -1e300))


# ---------------------------------------------------------------- attention


def check(s, frame, ctx, wdc, past=None):
    """cache8_attention with and without lse against the definition."""
    o, lse, pv, qk = c8.attention64(s, frame, past)
    bound, lse_bound = attention_bound(s, pv, o, qk, max(max(s.kv), 1))
    n = sum(s.q)
    kw = {} if past is None else dict(prefix=past.desc(wdc, s))
    for with_lse in (True, False):
        out = torch.full_like(s.x, 7.0)
        z = torch.full((s.rows, s.heads), 7.0, device="cuda") if with_lse else None
        ctx.cache8_attention(c8.cache8(wdc, s), cu.chunks(wdc, s), s.x, out, frame=frame, lse=z, **kw)
        within(out[:n], o[:n].reshape(n, -1), bound[:n].reshape(n, -1), "o")
        assert (out[n:] == 7).all()
        if with_lse:
            within(z[:n], lse[:n], lse_bound[:n] + 4 * EPS32 * lse[:n].abs(), "lse")
            assert (z[n:] == 7).all()


@pytest.mark.parametrize("case", ATTENTION + ATTENTION_WIDE, ids=ids)
def test_attention_matches_definition(case):
    dtype, heads, kvh, hd, page, q, kv, frame = case
    s = c8.state8(dtype, heads, kvh, hd, page, q, kv, seed=5, tail_rows=3, spread=0.5)
    wdc, ctx = ctx_of(s)
    check(s, frame, ctx, wdc)


FORMS = [("bf16", 4, 4, 64, 64, 3, 700), ("bf16", 4, 4, 128, 16, 20, 700), ("f32", 4, 2, 64, 32, 40, 700),
         ("f32", 2, 2, 128, 64, 40, 700), ("bf16", 4, 4, 128, 64, 1024, 2100), ("bf16", 4, 4, 128, 16, 1024, 2100),
         ("bf16", 4, 4, 64, 32, 20, 700)]
FORMS += [("bf16", heads, kvh, hd, page, q, q + 500) for heads, kvh, q in ((4, 4, 200), (16, 1, 4096)) for hd in (64, 128)
          for page in (16, 64)]
# (blocks of 128 rows with 40)
FORMS += [form for page in (16, 64) for form in (("bf16", 32, 8, 128, page, 10, 9100), ("bf16", 16, 4, 64, page, 10, 4100))]
forms = pytest.mark.parametrize("form", FORMS, ids=lambda f: "-".join(str(x) for x in f))


@forms
@pytest.mark.parametrize("frame", [1, 64])
def test_unseen_keys_have_no_influence(form, frame):
    """NaN in keys and values that only later rows see change later rows only."""
    dtype, heads, kvh, hd, page, q, kv = form
    s = c8.state8(dtype, heads, kvh, hd, page, [q], [kv], seed=6)
    pg, sl = cu.where(s, 0)
    j = kv - q // 2 - 1                               # in the chunk: seen from its middle on
    s.v8.view(torch.uint8)[pg[j], 0, sl[j], 3] = 127
    s.v8.view(torch.uint8)[pg[j], kvh - 1, sl[j], 1] = 255
    s.k8.view(torch.uint8)[pg[-1], kvh - 1, sl[-1], 5] = 127
    c8.decode(s)
    wdc, ctx = ctx_of(s)
    o, lse, pv, qk = c8.attention64(s, frame)
    bound, lse_bound = attention_bound(s, pv.nan_to_num(1e30, 1e30, 1e30), o.nan_to_num(0, 0, 0), qk, kv)
    out, z = torch.empty_like(s.x), torch.empty((s.rows, heads), device="cuda")
    ctx.cache8_attention(c8.cache8(wdc, s), cu.chunks(wdc, s), s.x, out, frame=frame, lse=z)
    assert torch.isnan(o).any() and torch.isfinite(o).any()
    got = out.reshape(o.shape).double()
    fine = torch.isfinite(o)
    assert torch.equal(fine, torch.isfinite(got))
    within(got[fine], o[fine], bound[fine], "o")
    fine = torch.isfinite(lse)
    within(z[fine], lse[fine], (lse_bound + 4 * EPS32 * lse.abs())[fine], "lse")


@forms
@pytest.mark.parametrize("ks,vs", [(40, 0), (-60, 60), (0, 110), (20, -100)], ids=str)
def test_powers_of_any_size(form, ks, vs):
    """Keys and values of very different powers of two beside each other: the result is of the largest weights' values. (q
    is made as small as the keys are large.)"""
    dtype, heads, kvh, hd, page, q, kv = form
    s = c8.state8(dtype, heads, kvh, hd, page, [q], [kv], seed=8)
    pg, sl = cu.where(s, 0)
    g = torch.Generator().manual_seed(9)
    one = (torch.randint(-3, 1, (kv, kvh, 1), generator=g).cuda() + torch.tensor([ks, vs], device="cuda")).to(torch.int32)
    one[::5, :, 1] -= 8
    s.scale[pg, :, sl] = (s.scale[pg, :, sl].int() + one).clamp(10, 247).to(torch.uint8)
    s.x = (s.x.float() * 2.0 ** -ks).to(s.td)
    c8.decode(s)
    wdc, ctx = ctx_of(s)
    check(s, 24, ctx, wdc)


@forms
@pytest.mark.parametrize("ramp", [3, 40], ids=str)
def test_rising_scores_move_the_reference(form, ramp):
    dtype, heads, kvh, hd, page, q, kv = form
    s = c8.state8(dtype, heads, kvh, hd, page, [q], [kv], seed=34)
    pg, sl = cu.where(s, 0)
    rise = torch.linspace(0.1, ramp * (64 / hd) ** 0.5, kv, device="cuda", dtype=torch.float64)[:, None, None]
    k, v = s.k.double(), s.v.double()
    k[pg, :, sl] = torch.randn((kv, kvh, hd), generator=torch.Generator().manual_seed(3)).cuda().double().abs() * rise
    c8.encode(s, k, v)
    s.x = s.x.abs()
    s.x[1::2] *= -1
    wdc, ctx = ctx_of(s)
    for frame in (0, 24):
        check(s, frame, ctx, wdc)


@forms
@pytest.mark.parametrize("odd", [math.nan, math.inf, 3e38], ids=str)
def test_an_odd_row_changes_no_other(form, odd):
    dtype, heads, kvh, hd, page, q, kv = form
    s = c8.state8(dtype, heads, kvh, hd, page, [q], [kv], seed=43)
    s.x[1] = odd
    wdc, ctx = ctx_of(s)
    z = torch.empty((s.rows, heads), device="cuda")
    out = ctx.cache8_attention(c8.cache8(wdc, s), cu.chunks(wdc, s), s.x, torch.empty_like(s.x), frame=24, lse=z)
    s.x[1] = 0
    o, lse, pv, qk = c8.attention64(s, 24)
    bound, lse_bound = attention_bound(s, pv, o, qk, kv)
    rest = torch.arange(s.rows, device="cuda") != 1
    within(out.reshape(o.shape)[rest], o[rest], bound[rest], "o")
    within(z[rest], lse[rest], (lse_bound + 4 * EPS32 * lse.abs())[rest], "lse")
    if math.isnan(odd):
        assert torch.isnan(out[1]).all()


@pytest.mark.parametrize("heads,kvh,hd,q", [(4, 4, 64, 1), (4, 2, 128, 7), (4, 4, 64, 40), (4, 4, 128, 40), (4, 2, 64, 200),
                                           (4, 2, 128, 200), (16, 1, 64, 4090), (16, 1, 128, 4090)])
def test_attention_over_one_key_is_its_value(heads, kvh, hd, q):
    s = c8.state8("bf16", heads, kvh, hd, 16, [q, 1], [q, 1], seed=28, scale=1.3)
    wdc, ctx = ctx_of(s)
    out = ctx.cache8_attention(c8.cache8(wdc, s), cu.chunks(wdc, s), s.x, torch.empty_like(s.x), frame=1)
    for b, row in ((0, 0), (1, q)):
        pg, sl = cu.where(s, b)
        assert torch.equal(out[row].reshape(heads, hd), s.v[pg[0], :, sl[0]].repeat_interleave(heads // kvh, 0))


@pytest.mark.parametrize("dtype,q,kv", [("bf16", [30, 20], [100, 60]), ("bf16", [300, 200], [400, 260]), ("f32", [30, 20], [100, 60])],
                         ids=str)
def test_wrong_bounds_bad_pages_strides_and_in_place(dtype, q, kv):
    s = c8.state8(dtype, 4, 2, 64, 16, q, kv, seed=8)
    s.k8.view(torch.uint8)[torch.isnan(s.k8.float())] = 40
    s.v8.view(torch.uint8)[torch.isnan(s.v8.float())] = 40
    s.scale[s.scale == 255] = 127
    wdc, ctx = ctx_of(s)
    cache = c8.cache8(wdc, s)
    full = ctx.cache8_attention(cache, cu.chunks(wdc, s), s.x, torch.empty_like(s.x), frame=1)
    wide = torch.zeros((s.rows, 1024), dtype=s.td, device="cuda")
    wide[:, 8:264] = s.x
    ctx.cache8_attention(cache, cu.chunks(wdc, s), wide[:, 8:264], wide[:, 512:768], frame=1)
    assert torch.equal(wide[:, 512:768], full) and (wide[:, 768:] == 0).all() and (wide[:, 264:512] == 0).all()
    ctx.cache8_attention(cache, cu.chunks(wdc, s), wide[:, 8:264], wide[:, 8:264], frame=1)
    assert torch.equal(wide[:, 8:264], full)
    out = torch.full_like(s.x, 7.0)
    ctx.cache8_attention(cache, cu.chunks(wdc, s, max_q=q[0] - 5), s.x, out, frame=1)
    assert (out[q[0] - 5:q[0]] == 7).all()
    s.kv_len[0], s.kv_len[1], s.q_start[2] = 1 << 30, -4, 1 << 30
    s.table[0, 1], s.table[0, 2] = -7, 1 << 30
    out = torch.full_like(s.x, 7.0)
    ctx.cache8_attention(cache, cu.chunks(wdc, s), s.x, out, frame=1)
    assert torch.isfinite(out).all() and (out[q[0]:] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_rows_and_no_keys(dtype):
    s = c8.state8(dtype, 4, 2, 64, 16, [3, 0], [0, 40], seed=13)
    wdc, ctx = ctx_of(s)
    before = bits(s)
    out, z = torch.full_like(s.x, 7.0), torch.full((3, 4), 7.0, device="cuda")
    ctx.cache8_attention(c8.cache8(wdc, s), cu.chunks(wdc, s), s.x, out, frame=1, lse=z)
    assert (out == 0).all() and (z == -math.inf).all()
    k = torch.full((3, 128), 7.0, dtype=s.td, device="cuda")
    ctx.cache8_read(c8.cache8(wdc, s), cu.chunks(wdc, s), k=k)
    assert (k == 0).all()
    for ch in (wdc.Chunks(s.q_start, s.kv_len, s.table, rows=0), cu.chunks(wdc, s, max_q=0), cu.chunks(wdc, s, max_kv=0)):
        x, y = s.x[:ch.rows], torch.full_like(s.x[:ch.rows], 7.0)
        ctx.cache8_append(c8.cache8(wdc, s), ch, s.qkv[:ch.rows], y)
        ctx.cache8_read(c8.cache8(wdc, s), ch, k=k[:ch.rows], v=k[:ch.rows])
        ctx.cache8_attention(c8.cache8(wdc, s), ch, x, torch.empty_like(x))
    assert all(torch.equal(a, b) for a, b in zip(before, bits(s)))


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("f32", 64)])
def test_pool_beyond_32_bit_offsets(dtype, hd):
    """Pages past 2^32 bytes of the pool."""
    page, kvh = 256, 4
    pages = (1 << 32) // (page * kvh * hd) + 40
    s = c8.state8(dtype, 4, kvh, hd, page, [20], [900], seed=14)
    small = s.k8, s.v8, s.scale
    s.k8, s.v8 = (torch.zeros((pages, kvh, page, hd), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    s.scale = torch.zeros((pages, kvh, page, 2), dtype=torch.uint8, device="cuda")
    for i in range(s.table.shape[1]):
        old, new = int(s.table[0, i]), pages - 1 - 3 * i
        for a, b in zip((s.k8, s.v8, s.scale), small):
            a.view(torch.uint8)[new] = b.view(torch.uint8)[old]
        s.table[0, i] = new
    k, v = {}, {}
    at = s.table[0].long()
    s_small = c8.state8(dtype, 4, kvh, hd, page, [20], [900], seed=14)
    wdc, ctx = ctx_of(s)
    out = ctx.cache8_attention(c8.cache8(wdc, s), cu.chunks(wdc, s), s.x, torch.empty_like(s.x), frame=1)
    ref = ctx.cache8_attention(c8.cache8(wdc, s_small), cu.chunks(wdc, s_small), s.x, torch.empty_like(s.x), frame=1)
    assert torch.equal(out, ref) and torch.isfinite(out).all()
    res = []
    for st in (s, s_small):
        q = ctx.cache8_append(c8.cache8(wdc, st), cu.chunks(wdc, st), s.qkv, torch.empty_like(s.x))
        res.append((q, *(x.clone() for x in ctx.cache8_read(c8.cache8(wdc, st), cu.chunks(wdc, st),
                                                            *(torch.empty((20, kvh * hd), dtype=s.td, device="cuda") for _ in range(2))))))
    for a, b in zip(*res):
        assert torch.equal(a, b)
    del k, v, at


def test_more_rows_than_one_launch_has():
    """Rows on both sides of 2^23 (and of 2^24 in the read) are stored and read back like others."""
    n, hd, page = (1 << 24) + 77, 64, 256
    torch_cuda()
    import paper_2608_01845_amd as wdc
    ctx = wdc.Context(cu.config("bf16", 1, hd, qk_norm=False, rope=(0, 0, 0)), allocate_weights=False)
    pages = -(-n // page)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.arange(pages, dtype=torch.int32, device="cuda").flip(0).reshape(1, -1).contiguous()
    k8, v8 = (torch.zeros((pages, 1, page, hd), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    scale = torch.zeros((pages, 1, page, 2), dtype=torch.uint8, device="cuda")
    cache, ch = wdc.PagedCache8(k8, v8, scale), wdc.Chunks(i32(0, n), i32(n), table, rows=n)
    qkv = torch.randn((n, 3 * hd), dtype=torch.bfloat16, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    q = ctx.cache8_append(cache, ch, qkv, torch.zeros((n, hd), dtype=torch.bfloat16, device="cuda"))
    v = ctx.cache8_read(cache, ch, v=torch.zeros((n, hd), dtype=torch.bfloat16, device="cuda"))[1]
    for at in (0, (1 << 23) - 50, (1 << 24) - 50, n - 100):
        rows = slice(at, at + 100)
        assert torch.equal(q[rows], qkv[rows, :hd])
        code, byte = c8.quantised64(qkv[rows, 2 * hd:].double())
        assert torch.equal(v[rows].double(), c8.values64(code, byte))


@pytest.mark.parametrize("dtype,heads,kvh,hd,q,kv", [("bf16", 4, 4, 128, [1, 1], [9000, 5000]), ("bf16", 4, 4, 64, [300], [9000]),
                                                     ("bf16", 16, 2, 128, [100, 64], [3000, 900]), ("f32", 4, 4, 64, [40], [3000])])
def test_less_scratch_and_no_byte_behind_it(dtype, heads, kvh, hd, q, kv):
    s = c8.state8(dtype, heads, kvh, hd, 64, q, kv, seed=17)
    wdc, ctx = ctx_of(s)
    lib, cache, ch = wdc.load(), c8.cache8(wdc, s), cu.chunks(wdc, s)
    o, lse, pv, qk = c8.attention64(s, 0)
    bound, _ = attention_bound(s, pv, o, qk, max(kv))
    need = lib.wdc_cache8_attention_scratch(ctx.h, cache.ref, ch.ref, None)
    assert need > 0
    for n in (need, need - 4, need // 2, need // 5, 0):
        mem = torch.full((need + 4096,), 171, dtype=torch.uint8, device="cuda")
        out = torch.empty_like(s.x)
        cols = heads * hd
        assert lib.wdc_cache8_attention(ctx.h, cache.ref, ch.ref, None, s.x.data_ptr(), cols, 0, out.data_ptr(), cols, None,
                                        mem.data_ptr(), n) == 0
        within(out.reshape(o.shape), o, bound, "o")
        assert (mem[n:] == 171).all()


# ---------------------------------------------------------------- as a rollout uses them


def rollout(ctx, wdc, s, qkv, pos, outs, sizes):
    """Chunks appended one after the other, each attending over what is there; returns what was computed."""
    at = 0
    for i, m in enumerate(sizes):
        at += m
        ch = wdc.Chunks(s.starts[i], s.lens[i], s.table, rows=m, max_q=m, max_kv=sum(sizes))
        q, o, z = outs[i]
        ctx.cache8_append(c8.cache8(wdc, s), ch, qkv[at - m:at], q, pos=pos[at - m:at])
        ctx.cache8_attention(c8.cache8(wdc, s), ch, q, o, frame=16, lse=z)
    return outs


def rollout_state(dtype, hd, sizes, heads=4, kvh=2):
    n = sum(sizes)
    s = c8.state8(dtype, heads, kvh, hd, 32, [n], [n], seed=20)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    s.starts = [i32(0, m) for m in sizes]
    s.lens = [i32(sum(sizes[:i + 1])) for i in range(len(sizes))]
    pos = torch.arange(3 * n, device="cuda", dtype=torch.int32).reshape(n, 3).contiguous()
    new = lambda: [(torch.empty((m, heads * hd), dtype=s.td, device="cuda"), torch.empty((m, heads * hd), dtype=s.td, device="cuda"),  # noqa: E731
                    torch.empty((m, heads), device="cuda")) for m in sizes]
    return s, pos, new


@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
def test_rollout_of_chunks_append_attend_read(dtype, hd):
    sizes = [40, 1, 200, 1, 33]
    s, pos, new = rollout_state(dtype, hd, sizes)
    wdc, ctx = ctx_of(s)
    outs = rollout(ctx, wdc, s, s.qkv, pos, new(), sizes)
    n = sum(sizes)
    k, v = ctx.cache8_read(c8.cache8(wdc, s), cu.chunks(wdc, s), *(torch.empty((n, 2 * hd), dtype=s.td, device="cuda") for _ in range(2)))
    c8.decode(s)
    pg, sl = cu.where(s, 0)
    assert torch.equal(k, s.k[pg, :, sl].reshape(n, -1)) and torch.equal(v, s.v[pg, :, sl].reshape(n, -1))
    # what the rows attended over are the stored values, near the rows' own ones by half a step of a code
    rows = s.qkv.double().reshape(n, 8, hd)[:, 6:]
    assert ((v.double().reshape(rows.shape) - rows).abs() <= 2.0 ** -4 * rows.abs() + 2.0 ** -10 * rows.abs().amax(2, keepdim=True) / 224).all()
    at = 0
    for m, (q, o, z) in zip(sizes, outs):
        at += m
        t = cu.SimpleNamespace(**vars(s))
        t.q, t.kv, t.rows, t.x = [m], [at], m, q
        want, lse, pv, qk = c8.attention64(t, 16)
        bound, lse_bound = attention_bound(t, pv, want, qk, at)
        within(o.reshape(want.shape), want, bound, "o")
        within(z, lse, lse_bound + 4 * EPS32 * lse.abs(), "lse")


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_rollout_captured_and_replayed(dtype, hd):
    """The calls captured into one graph; replays on new rows, with eager work between, equal the eager run."""
    sizes = [200, 1, 33, 300]
    s, pos, new = rollout_state(dtype, hd, sizes)
    side = torch.cuda.Stream()
    import paper_2608_01845_amd as wdc
    ctx = wdc.Context(cu.config(dtype, 4, hd), allocate_weights=False, stream=side)
    rows = [s.qkv * f for f in (1.0, 0.5, -2.0)]
    want = []
    side.wait_stream(torch.cuda.current_stream())
    for x in rows:
        want.append(rollout(ctx, wdc, s, x, pos, new(), sizes))
        side.synchronize()
    qkv, outs = s.qkv.clone(), new()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        rollout(ctx, wdc, s, qkv, pos, outs, sizes)
    for i in (1, 0, 2, 1):
        qkv.copy_(rows[i])
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            g.replay()
        side.synchronize()
        torch.full((1 << 20,), 3.0, device="cuda")
        for a, b in zip(outs, want[i]):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_calls_repeat_bit_for_bit():
    s = c8.state8("bf16", 8, 2, 128, 16, [70, 1, 33], [3000, 4000, 700], seed=23)
    wdc, ctx = ctx_of(s)
    first = None
    for _ in range(3):
        z = torch.empty((s.rows, 8), device="cuda")
        out = ctx.cache8_attention(c8.cache8(wdc, s), cu.chunks(wdc, s), s.x, torch.empty_like(s.x), frame=4, lse=z)
        first = first or (out, z)
        assert torch.equal(out, first[0]) and torch.equal(z, first[1])
