"""The paged cache operators at the edges of what their documentation allows."""
import pytest
import torch

from tests import cache_util as cu
from tests.test_gpu_cache import EPS32, ctx_of

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
