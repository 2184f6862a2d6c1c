"""Attention over a shared past: bounds beyond what unshared calls allow, the unshared result, sequences in no group,
prefixes that change between replays."""
import pytest
import torch

from tests import cache8_util as c8
from tests import cache_util as cu
from tests.test_gpu_cache import EPS, EPS32, attention_bound, ctx_of, few, within

pytestmark = pytest.mark.gpu


def both(ctx, wdc, s, ch, pre, frame):
    """The shared attention over the state's cache in the model's type and over its codes: o, lse of each."""
    for codes in (False, True):
        out, z = torch.full_like(s.x, 7.0), torch.full((s.rows, s.heads), 7.0, device="cuda")
        if codes:
            ctx.cache8_attention(c8.cache8(wdc, s), ch, s.x, out, frame=frame, lse=z, prefix=pre)
        else:
            ctx.cache_attention_shared(wdc.PagedCache(s.k, s.v), ch, pre, s.x, out, frame=frame, lse=z)
        yield out.reshape(s.rows, s.heads, s.hd), z


@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_bounds_that_only_sharing_allows(dtype, hd):
    """128 sequences of 32 kv heads and bounds of 70,016 keys, 69,888 of them shared: more than 2^28 if each sequence had its own."""
    s = c8.state8(dtype, 32, 32, hd, 16, [1] * 128, [40 + i % 30 for i in range(128)], seed=70, spread=0.5)
    s.table = torch.cat([s.table, torch.full((128, 70016 // 16 - s.table.shape[1]), -1, dtype=torch.int32, device="cuda")], 1).contiguous()
    wdc, ctx = ctx_of(s)
    ch, past = cu.chunks(wdc, s, max_kv=70016), c8.Past(s, [128], [32])
    with pytest.raises(wdc.WdcError):
        ctx.cache_attention(wdc.PagedCache(s.k, s.v), ch, s.x, torch.empty_like(s.x))
    o, lse, pv, qk = c8.attention64(s, 1, past)
    bound, lse_bound = attention_bound(s, pv, o, qk, max(s.kv))
    for out, z in both(ctx, wdc, s, ch, past.desc(wdc, s, max_prefix=69888, max_own=40), 1):
        within(out, o, bound, "o")
        within(z, lse, lse_bound + 4 * EPS32 * lse.abs(), "lse")


SAME = [
    # dtype, heads, kvh, hd, page, q, kv, frame, groups, prefix
    ("f32", 4, 2, 64, 32, [1, 33, 2], [321, 400, 330], 1, [3], [320]),
    ("f32", 3, 1, 128, 16, [1, 1, 1, 1], [3000 + 40 * i for i in range(4)], 1, [2, 2], [2992, 1600]),
    ("bf16", 8, 2, 128, 64, [1] * 8, [1000 + 20 * i for i in range(8)], 1, [8], [960]),      # few rows apart, many together
    ("bf16", 32, 8, 64, 16, [1] * 24, [5000 + 20 * i for i in range(24)], 1, [24], [4992]),
    ("bf16", 4, 4, 128, 16, [333, 200], [1500, 1300], 64, [2], [960]),                        # many apart too
    ("bf16", 16, 1, 64, 128, [600, 700], [1500, 1400], 100, [2], [640]),
]
ids = lambda c: f"{c[0]}-{c[1]}x{c[2]}x{c[3]}-p{c[4]}-{few(c[5])}"  # noqa: E731


@pytest.mark.parametrize("scale", [1.0, 3.0])
@pytest.mark.parametrize("case", SAME, ids=ids)
def test_tables_that_name_the_same_pages(case, scale):
    """Shared and unshared calls compared with each other. float32: two orders of the same sums, each off by float32's arithmetic.
    bf16: both round weights to bf16; divided by the sum of the weights that is off by 2^-8 sum p|v|, by the sum of the rounded ones
    by 2^-8 sum p|v - o| <= 2^-8 (sum p|v| + |o|); each result is rounded once. scale: of q and k; at 3 a few keys have most of the weight."""
    dtype, heads, kvh, hd, page, q, kv, frame, groups, prefix = case
    s = c8.state8(dtype, heads, kvh, hd, page, q, kv, seed=71, spread=0.3, scale=scale)
    wdc, ctx = ctx_of(s)
    past, ch = c8.Past(s, groups, prefix), cu.chunks(wdc, s)
    for b, lead in enumerate(past.lead):
        s.table[b, :past.keys[b] // page] = s.table[lead, :past.keys[b] // page]
    o, lse, pv, qk = c8.attention64(s, frame, past)
    arithmetic, lse_bound = attention_bound(s, pv, o, qk, max(kv))
    arithmetic = arithmetic - (EPS[dtype] * o.abs() + (EPS["bf16"] * pv if dtype == "bf16" else 0))
    bound = 2 * arithmetic + 2 * EPS[dtype] * o.abs() + (EPS["bf16"] * (2 * pv + o.abs()) if dtype == "bf16" else 0)
    for codes, (out, z) in enumerate(both(ctx, wdc, s, ch, past.desc(wdc, s), frame)):
        ref, y = torch.empty_like(s.x), torch.empty_like(z)
        if codes:
            ctx.cache8_attention(c8.cache8(wdc, s), ch, s.x, ref, frame=frame, lse=y)
        else:
            ctx.cache_attention(wdc.PagedCache(s.k, s.v), ch, s.x, ref, frame=frame, lse=y)
        within(out, ref.reshape(out.shape).double(), bound, "o")
        within(z, y.double(), 2 * (lse_bound + 4 * EPS32 * lse.abs()), "lse")


@pytest.mark.parametrize("dtype,hd,q", [("bf16", 64, 1), ("bf16", 128, 50), ("f32", 64, 9)])
@pytest.mark.parametrize("tight", [False, True])
def test_sequences_in_no_group(dtype, hd, q, tight):
    """Before the first group and behind the last one: each on its own keys, to the bound of these keys."""
    s = c8.state8(dtype, 4, 2, hd, 16, [q] * 5, [400, 410, 420, 430, 440], seed=72)
    wdc, ctx = ctx_of(s)
    some = c8.Past(s, [2, 1, 2], [0, 320, 0])
    pre = wdc.Prefix(some.group_start[1:3].contiguous(), some.prefix_len[1:2].contiguous(),
                     **(dict(max_prefix=320, max_own=440) if tight else {}))
    for frame in (0, 1):
        o, lse, pv, qk = c8.attention64(s, frame, some)
        bound, lse_bound = attention_bound(s, pv, o, qk, 440)
        for out, z in both(ctx, wdc, s, cu.chunks(wdc, s), pre, frame):
            within(out, o, bound, "o")
            within(z, lse, lse_bound + 4 * EPS32 * lse.abs(), "lse")


@pytest.mark.parametrize("dtype,hd,q,kv,prefix", [("bf16", 128, [1, 1, 1], [900, 800, 1000], 640), ("bf16", 64, [200, 150], [900, 800], 576),
                                                  ("f32", 64, [9, 4], [300, 250], 128)])
@pytest.mark.parametrize("codes", [False, True])
def test_replays_follow_the_prefix(dtype, hd, q, kv, prefix, codes):
    """One captured call, replayed with other prefix lengths, against the definition with each of them."""
    s = c8.state8(dtype, 4, 2, hd, 16, q, kv, seed=73)
    past = c8.Past(s, [len(q)], [prefix])
    import paper_2608_01845_amd as wdc
    side = torch.cuda.Stream()
    ctx = wdc.Context(cu.config(dtype, 4, hd), allocate_weights=False, stream=side)
    pre, ch = past.desc(wdc, s, max_own=max(kv)), cu.chunks(wdc, s)
    cache = c8.cache8(wdc, s) if codes else wdc.PagedCache(s.k, s.v)
    out, z = torch.empty_like(s.x), torch.empty((s.rows, 4), device="cuda")
    lens, want = (prefix, 0, prefix - 64), []
    for n in lens:
        o, lse, pv, qk = c8.attention64(s, 1, c8.Past(s, [len(q)], [n]))
        want.append((o, lse, *attention_bound(s, pv, o, qk, max(kv))))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        if codes:
            ctx.cache8_attention(cache, ch, s.x, out, frame=1, lse=z, prefix=pre)
        else:
            ctx.cache_attention_shared(cache, ch, pre, s.x, out, frame=1, lse=z)
    for i in (0, 2, 1, 0):
        past.prefix_len.fill_(lens[i])
        out.fill_(7.0)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            g.replay()
        side.synchronize()
        o, lse, bound, lse_bound = want[i]
        within(out.reshape(o.shape), o, bound, "o")
        within(z, lse, lse_bound + 4 * EPS32 * lse.abs(), "lse")
