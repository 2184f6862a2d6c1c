"""Attention of groups of sequences that share a past, over the cache in the model's type and in 8 bits."""
import math

import pytest
import torch

from tests import cache8_util as c8
from tests import cache_util as cu
from tests.test_gpu_cache import EPS32, attention_bound, ctx_of, few, within
from tests.test_gpu_cache8 import check as check8

pytestmark = pytest.mark.gpu

SHARED = [
    # dtype, heads, kvh, hd, page, q, kv, frame, groups, prefix
    ("bf16", 4, 4, 64, 16, [1, 1, 1], [40, 33, 100], 1, [3], [32]),
    ("bf16", 8, 2, 128, 64, [1] * 16, [640 + 13 * i + 1 for i in range(16)], 1, [16], [640]),
    ("bf16", 32, 8, 128, 32, [1] * 9, [5000 + i for i in range(9)], 0, [4, 5], [4992, 3200]),
    ("bf16", 6, 2, 64, 16, [1, 4, 0, 2, 7, 1], [161, 164, 200, 85, 130, 1], 1, [3, 2, 1], [160, 80, 0]),
    ("bf16", 4, 2, 64, 64, [100, 30, 70], [800, 700, 1000], 7, [3], [640]),
    ("bf16", 4, 4, 128, 16, [333, 200], [1500, 1300], 64, [2], [1104]),
    ("bf16", 16, 1, 64, 128, [600, 700, 500], [1500, 1400, 2000], 100, [1, 2], [512, 640]),
    ("bf16", 16, 1, 128, 32, [1300, 1200], [2500, 2400], 0, [2], [1088]),
    ("f32", 4, 2, 64, 32, [1, 33, 2], [321, 400, 330], 1, [3], [320]),
    ("f32", 3, 1, 128, 16, [40, 20], [300, 333], 16, [2], [160]),
    ("bf16", 16, 1, 128, 64, [400, 300], [1500, 1300], 50, [2], [1024]),
    ("bf16", 16, 16, 128, 64, [40, 30], [9000, 8800], 1, [2], [8704]),
    ("bf16", 16, 1, 64, 16, [3000, 1500], [3500, 2300], 64, [2], [800]),
    ("f32", 4, 4, 128, 16, [1, 2, 1], [5000, 5003, 5100], 1, [3], [4992]),
    ("bf16", 4, 1, 128, 16, [i % 3 for i in range(300)], [40 + i % 3 + i % 17 for i in range(300)], 1, [3] * 100, [32] * 100),
    ("bf16", 4, 4, 64, 64, [1] * 200, [900 + i % 70 for i in range(200)], 0, [200], [896]),
    # prefixes inside a page, longer than the first sequence, than another one, and than a chunk leaves
    ("bf16", 4, 4, 64, 64, [1, 3, 2], [300, 290, 400], 1, [3], [250]),
    ("bf16", 4, 2, 128, 16, [1, 3, 2], [300, 100, 400], 1, [3], [100000]),
    ("bf16", 4, 4, 64, 16, [40, 30], [64, 60], 1, [2], [48]),
    ("f32", 4, 4, 64, 16, [4, 30], [64, 20], 1, [2], [48]),
    ("bf16", 4, 4, 64, 16, [5, 6], [0, 30], 1, [2], [16]),                       # a first sequence without keys
    ("bf16", 2, 1, 64, 16, [2, 3, 1, 1], [40, 50, 60, 20], 1, [0, 2, 0, 2, 0], [16, 32, 16, 16, 64]),   # empty groups
    ("bf16", 4, 2, 64, 16, [1 + i % 3 for i in range(150)], [96 + 3 + 7 * i % 50 for i in range(150)], 1, [70, 1, 79], [96, 16, 80]),
    ("bf16", 4, 2, 128, 16, [1] * 150, [130 + 5 * i for i in range(150)], 1, [1] * 75 + [75], [16 * (i % 7) for i in range(75)] + [112]),
]
# blocks of 128 rows with 40, many tiles each
SHARED += [("bf16", 32, 8, hd, page, [4, 6], [n + 30, n + 100], 1, [2], [n]) for hd, n in ((128, 20032), (64, 40000)) for page in (16, 64)]
ids = lambda c: f"{c[0]}-{c[1]}x{c[2]}x{c[3]}-p{c[4]}-{few(c[5])}-{few(c[6])}-f{c[7]}-{few(c[8])}-{few(c[9])}"  # noqa: E731


def check(s, frame, past, ctx, wdc):
    o, lse, pv, qk = c8.attention64(s, frame, past)
    bound, lse_bound = attention_bound(s, pv, o, qk, max(max(s.kv), 1))
    n = sum(s.q)
    for with_lse in (True, False):
        out = torch.full_like(s.x, 7.0)
        z = torch.full((s.rows, s.heads), 7.0, device="cuda") if with_lse else None
        ctx.cache_attention_shared(wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s), past.desc(wdc, s), s.x, out, frame=frame, lse=z)
        within(out[:n], o[:n].reshape(n, -1), bound[:n].reshape(n, -1), "o")
        assert (out[n:] == 7).all()
        if with_lse:
            within(z[:n], lse[:n], lse_bound[:n] + 4 * EPS32 * lse[:n].abs(), "lse")
            assert (z[n:] == 7).all()


@pytest.mark.parametrize("own_pages", [True, False])
@pytest.mark.parametrize("case", SHARED, ids=ids)
def test_attention_over_a_shared_past(case, own_pages):
    """own_pages: the sequences' tables have other pages in the shared part (never looked at); otherwise no pages."""
    dtype, heads, kvh, hd, page, q, kv, frame, groups, prefix = case
    s = cu.state(dtype, heads, kvh, hd, page, q, kv, seed=50, tail_rows=3)
    wdc, ctx = ctx_of(s)
    past = c8.Past(s, groups, prefix)
    if not own_pages:
        for b, (p, lead) in enumerate(zip(past.keys, past.lead)):
            if b != lead:
                s.table[b, :p // page] = -1
    check(s, frame, past, ctx, wdc)


@pytest.mark.parametrize("case", SHARED, ids=ids)
def test_attention_over_a_shared_past_in_8_bits(case):
    dtype, heads, kvh, hd, page, q, kv, frame, groups, prefix = case
    s = c8.state8(dtype, heads, kvh, hd, page, q, kv, seed=51, tail_rows=3, spread=0.5)
    wdc, ctx = ctx_of(s)
    check8(s, frame, ctx, wdc, c8.Past(s, groups, prefix))


@pytest.mark.parametrize("dtype,hd,q", [("bf16", 64, 1), ("bf16", 128, 50), ("f32", 64, 9)])
def test_loose_bounds_and_some_sequences_in_no_group(dtype, hd, q):
    s = cu.state(dtype, 4, 2, hd, 16, [q] * 5, [400, 410, 420, 430, 440], seed=52)
    wdc, ctx = ctx_of(s)
    past = c8.Past(s, [2, 3], [320, 160])
    check(s, 1, past, ctx, wdc)
    cache, ch = wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s)
    o, lse, pv, qk = c8.attention64(s, 1, past)
    bound, _ = attention_bound(s, pv, o, qk, 440)
    out = ctx.cache_attention_shared(cache, ch, wdc.Prefix(past.group_start, past.prefix_len), s.x, torch.empty_like(s.x), frame=1)
    within(out.reshape(o.shape), o, bound, "o")
    # sequences before the first group and behind the last are on their own
    past = c8.Past(s, [5], [0])
    o, lse, pv, qk = c8.attention64(s, 1, past)
    some = c8.Past(s, [2, 1, 2], [0, 320, 0])
    o2, _, _, _ = c8.attention64(s, 1, some)
    past.group_start, past.prefix_len = some.group_start[1:3].contiguous(), some.prefix_len[1:2].contiguous()
    out = ctx.cache_attention_shared(cache, ch, wdc.Prefix(past.group_start, past.prefix_len), s.x, torch.empty_like(s.x), frame=1)
    within(out.reshape(o2.shape), o2, bound, "o")


def test_wrong_device_values_stay_in_the_buffers():
    """Groups, prefixes and bounds that make no sense give some finite numbers."""
    s = cu.state("bf16", 4, 2, 64, 16, [3, 40, 1], [300, 200, 100], seed=53, fill=0.5)
    wdc, ctx = ctx_of(s)
    cache, ch = wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    for start, length in (((0, 2, 3), (1 << 30, 64)), ((-5, 1 << 30, 7), (64, -9)), ((3, 1, 0), (64, 64)), ((2, 2, 2), (16, 16)),
                          ((1, 3, 1), (64, 1 << 30))):
        for kw in ({}, dict(max_prefix=50), dict(max_own=20), dict(max_prefix=0, max_own=0)):
            # lse of 0 where a part of no pass is read: the scratch is zeros
            mem = torch.zeros(1 << 26, dtype=torch.uint8, device="cuda")
            pre = wdc.Prefix(i32(*start), i32(*length), **kw)
            out = torch.full_like(s.x, 7.0)
            need = wdc.load().wdc_cache_attention_shared_scratch(ctx.h, cache.ref, ch.ref, pre.ref)
            assert 0 < need <= mem.numel() - 4096
            assert wdc.load().wdc_cache_attention_shared(ctx.h, cache.ref, ch.ref, pre.ref, s.x.data_ptr(), 256, 1, out.data_ptr(),
                                                         256, None, mem.data_ptr(), need) == 0
            assert torch.isfinite(out).all() and (mem[need:] == 0).all()


def test_keys_past_the_own_bound_are_not_there():
    s = cu.state("bf16", 4, 2, 64, 16, [2, 3], [200, 180], seed=54)
    wdc, ctx = ctx_of(s)
    past = c8.Past(s, [2], [96])
    ref = cu.SimpleNamespace(**vars(s))
    ref.kv = [96 + 50, 96 + 50]
    o, _, pv, qk = c8.attention64(ref, 1, past)
    bound, _ = attention_bound(s, pv, o, qk, 200)
    out = ctx.cache_attention_shared(wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s), past.desc(wdc, s, max_own=50), s.x,
                                     torch.empty_like(s.x), frame=1)
    within(out.reshape(o.shape), o, bound, "o")


@pytest.mark.parametrize("dtype,hd,q,kv,prefix", [("bf16", 128, [1, 1, 1], [900, 800, 1000], 640), ("bf16", 64, [200, 150], [900, 800], 576),
                                                  ("f32", 64, [9, 4], [300, 250], 128)])
@pytest.mark.parametrize("codes", [False, True])
def test_captured_other_stream_and_repeated(dtype, hd, q, kv, prefix, codes):
    """On another stream, captured, with the prefix lengths changed between replays: the bits of the eager call."""
    s = c8.state8(dtype, 4, 2, hd, 16, q, kv, seed=55)
    past = c8.Past(s, [len(q)], [prefix])
    side = torch.cuda.Stream()
    import paper_2608_01845_amd as wdc
    ctx = wdc.Context(cu.config(dtype, 4, hd), allocate_weights=False, stream=side)
    pre, ch = past.desc(wdc, s, max_own=max(kv)), cu.chunks(wdc, s)
    cache = c8.cache8(wdc, s) if codes else wdc.PagedCache(s.k, s.v)

    def call(out, z):
        if codes:
            ctx.cache8_attention(cache, ch, s.x, out, frame=1, lse=z, prefix=pre)
        else:
            ctx.cache_attention_shared(cache, ch, pre, s.x, out, frame=1, lse=z)
    new = lambda: (torch.empty_like(s.x), torch.empty((s.rows, 4), device="cuda"))  # noqa: E731
    lens, want = (prefix, 0, prefix - 64), []
    for n in lens:
        past.prefix_len.fill_(n)
        res = new()
        torch.cuda.synchronize()
        call(*res)
        torch.full((1 << 22,), 3.0, device="cuda")
        side.synchronize()
        want.append(res)
    o, _, pv, qk = c8.attention64(s, 1, past if prefix else None)
    got = new()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        call(*got)
    for i in (0, 2, 1, 0):
        past.prefix_len.fill_(lens[i])
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            g.replay()
        side.synchronize()
        torch.full((1 << 20,), 3.0, device="cuda")
        assert torch.equal(got[0], want[i][0]) and torch.equal(got[1], want[i][1])


def test_two_graphs_in_flight():
    """Two captured calls over the same past, replayed on two streams at once, several times: each has its own scratch."""
    s = cu.state("bf16", 8, 2, 128, 64, [1] * 6, [3000 + 10 * i for i in range(6)], seed=56)
    past = c8.Past(s, [6], [2944])
    import paper_2608_01845_amd as wdc
    want, got, graphs, streams, keep = [], [], [], [], []
    for i in range(2):
        side = torch.cuda.Stream()
        ctx = wdc.Context(cu.config("bf16", 8, 128), allocate_weights=False, stream=side)
        x, ch = s.x * (1 + i), cu.chunks(wdc, s)
        cache, pre = wdc.PagedCache(s.k, s.v), past.desc(wdc, s)
        a, b = torch.empty_like(x), torch.empty_like(x)
        torch.cuda.synchronize()
        ctx.cache_attention_shared(cache, ch, pre, x, a, frame=1)
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            ctx.cache_attention_shared(cache, ch, pre, x, b, frame=1)
        want.append(a), got.append(b), graphs.append(g), streams.append(side), keep.append((ctx, x, ch, cache, pre))
    for _ in range(4):
        for b in got:
            b.fill_(7.0)
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a, b)


@pytest.mark.parametrize("hd, page, q", [(64, 32, [40, 30]), (128, 32, [400, 300]), (128, 64, [400, 300])])
def test_unseen_own_keys_have_no_influence(hd, page, q):
    s = cu.state("bf16", 4, 2, hd, page, q, [160 + n for n in q], seed=57)
    for b in range(2):
        pg, sl = cu.where(s, b)
        j = s.kv[b] - s.q[b] // 2
        s.v[pg[j], 0, sl[j], 3] = math.nan
        s.k[pg[-1], 1, sl[-1], 5] = math.nan
    past = c8.Past(s, [2], [128])
    wdc, ctx = ctx_of(s)
    o, _, pv, qk = c8.attention64(s, 8, past)
    bound, _ = attention_bound(s, pv.nan_to_num(1e30), o.nan_to_num(0), qk, max(s.kv))
    out = ctx.cache_attention_shared(wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s), past.desc(wdc, s), s.x, torch.empty_like(s.x), frame=8)
    got, fine = out.reshape(o.shape).double(), torch.isfinite(o)
    assert not fine.all() and fine.any() and torch.equal(fine, torch.isfinite(got))
    within(got[fine], o[fine], bound[fine], "o")


def test_shared_is_the_unshared_attention():
    """Tables that name the same pages: the same result as wdc_cache_attention up to the order of its float32 sums."""
    s = cu.state("bf16", 8, 2, 128, 64, [1] * 8, [1000 + 20 * i for i in range(8)], seed=58)
    past = c8.Past(s, [8], [960])
    s.table[1:, :15] = s.table[0, :15]
    wdc, ctx = ctx_of(s)
    cache, ch = wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s)
    a = ctx.cache_attention(cache, ch, s.x, torch.empty_like(s.x), frame=1)
    b = ctx.cache_attention_shared(cache, ch, past.desc(wdc, s), s.x, torch.empty_like(s.x), frame=1)
    o, _, pv, qk = c8.attention64(s, 1, past)
    bound, _ = attention_bound(s, pv, o, qk, 1200)
    within(a.reshape(o.shape), o, bound, "o")
    within(b.reshape(o.shape), o, bound, "o")


@pytest.mark.parametrize("codes", [False, True])
def test_no_rows(codes):
    s = c8.state8("bf16", 4, 2, 64, 16, [0, 0], [40, 30], seed=59)
    wdc, ctx = ctx_of(s)
    past = c8.Past(s, [2], [32])
    for ch in (cu.chunks(wdc, s), cu.chunks(wdc, s, max_kv=0)):
        if codes:
            ctx.cache8_attention(c8.cache8(wdc, s), ch, s.x, torch.empty_like(s.x), prefix=past.desc(wdc, s))
        else:
            ctx.cache_attention_shared(wdc.PagedCache(s.k, s.v), ch, past.desc(wdc, s), s.x, torch.empty_like(s.x))
    s = c8.state8("bf16", 4, 2, 64, 16, [2, 1], [40, 30], seed=59)
    past = c8.Past(s, [2], [32])
    out = torch.full_like(s.x, 7.0)
    ctx.cache8_attention(c8.cache8(wdc, s), cu.chunks(wdc, s, max_kv=0), s.x, out, prefix=past.desc(wdc, s))
    assert (out == 0).all()
