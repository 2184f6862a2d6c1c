"""Attention over a shared past: bounds beyond what unshared calls allow."""
import pytest
import torch

from tests import cache8_util as c8
from tests import cache_util as cu
from tests.test_gpu_cache import EPS32, attention_bound, ctx_of, within

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
