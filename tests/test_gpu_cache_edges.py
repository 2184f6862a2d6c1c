"""The paged cache operators at the edges of what their documentation allows."""
import math

import pytest
import torch

from tests import cache_util as cu
from tests.test_gpu_cache import EPS32, attention_bound, ctx_of, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("far", [0, 1 << 20])
def test_append_turns_by_the_float64_angle(hd, far):
    """Pairs (1, 0) come out as cosine and sine of their angles: within one float32 step of sincospif (a half step of a
    value up to 1 is 2^-25) and one rounding; an angle rounded to float32 would add up to 2^-25 pi."""
    s = cu.state("f32", 2, 2, hd, 64, [3000], [3000], seed=41)
    wdc, ctx = ctx_of(s, qk_norm=False)
    s.qkv[:, 0::2], s.qkv[:, 1::2] = 1, 0
    g = torch.Generator().manual_seed(42)
    pos = (torch.randint(0, 5000, (3000, 3), generator=g) + far).to(torch.int32).cuda()
    out = ctx.cache_append(wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s), s.qkv, torch.empty_like(s.x), pos=pos)
    freq = torch.cat([10000.0 ** (-2 * torch.arange(d // 2, dtype=torch.float64) / d) for d in cu.ROPE[hd]]).cuda()
    axis = torch.cat([torch.full((d // 2,), a) for a, d in enumerate(cu.ROPE[hd])]).cuda()
    ang = pos.double()[:, axis] * freq                # (float64 rounds it by up to 2^-31)
    got = out.reshape(3000, 2, hd // 2, 2).double()
    bound = 2 * 2.0 ** -25 + 2.0 ** -25 + 2.0 ** -30
    for i, want in enumerate((torch.cos(ang), torch.sin(ang))):
        err = (got[..., i] - want[:, None]).abs()
        assert err.max().item() <= bound, (i, err.max().item() / EPS32)


@pytest.mark.parametrize("dtype,heads,kvh,hd,page,q,kv", [
    ("bf16", 4, 4, 64, 64, 3, 700), ("bf16", 4, 4, 128, 16, 20, 700), ("f32", 4, 2, 64, 32, 40, 700),
    ("bf16", 4, 4, 64, 16, 200, 700), ("bf16", 4, 4, 128, 64, 200, 700), ("bf16", 16, 1, 64, 64, 4096, 4596),
    ("bf16", 16, 1, 128, 16, 4096, 4596)])
@pytest.mark.parametrize("frame", [0, 24])
@pytest.mark.parametrize("odd", [math.nan, math.inf, 3e38], ids=str)
def test_attention_of_an_odd_row_changes_no_other(dtype, heads, kvh, hd, page, q, kv, frame, odd):
    """A row of NaN, infinities or values whose scores are infinite; the rows beside it are as always."""
    s = cu.state(dtype, heads, kvh, hd, page, [q], [kv], seed=43)
    s.x[1] = odd
    wdc, ctx = ctx_of(s)
    z = torch.empty((s.rows, heads), device="cuda")
    out = ctx.cache_attention(wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s), s.x, torch.empty_like(s.x), frame=frame, lse=z)
    s.x[1] = 0
    o, lse, pv, qk = cu.attention64(s, frame)
    bound, lse_bound = attention_bound(s, pv, o, qk, kv)
    rest = torch.arange(s.rows, device="cuda") != 1
    within(out.reshape(o.shape)[rest], o[rest], bound[rest], "o")
    within(z[rest], lse[rest], (lse_bound + 4 * EPS32 * lse.abs())[rest], "lse")
    if math.isnan(odd):
        assert torch.isnan(out[1]).all()


@pytest.mark.parametrize("dtype,heads,kvh,hd", [("bf16", 6, 2, 64), ("bf16", 64, 1, 128), ("f32", 6, 2, 64)])
def test_mass_and_attention_of_strided_rows(dtype, heads, kvh, hd):
    """Rows of a wider tensor give the bits of packed ones, for groups that divide a stage of 128 rows and not."""
    s = cu.state(dtype, heads, kvh, hd, 32, [90, 1], [700, 40], seed=44)
    wdc, ctx = ctx_of(s)
    cache, ch = wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s)
    wide = torch.full((s.rows, (heads + 3) * hd), 9.0, dtype=s.td, device="cuda")
    part = wide[:, hd:hd + heads * hd]
    part.copy_(s.x)
    res = []
    for x in (s.x, part):
        lse = torch.empty((s.rows, heads), device="cuda")
        out = ctx.cache_attention(cache, ch, x, torch.empty_like(s.x), frame=4, lse=lse)
        res.append((out, lse, ctx.cache_mass(cache, ch, x, lse, s.mass, frame=4, decay=0.0, out=torch.zeros_like(s.mass))))
    for a, b in zip(*res):
        assert torch.equal(a, b)
    total = res[0][2].double().sum()                  # every row's weights sum to 1
    assert abs(total.item() / (s.rows * heads) - 1) < 1e-4
