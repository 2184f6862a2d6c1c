"""The 8-bit cache's attention at the ends of the powers of two, over every form of its kernels."""
import pytest
import torch

from tests import cache8_util as c8
from tests import cache_util as cu
from tests.test_gpu_cache import EPS32, attention_bound, ctx_of, within
from tests.test_gpu_cache8 import forms

pytestmark = pytest.mark.gpu


def pasts(s):
    """No past, and one that ends on a page's border in front of the chunk."""
    return [None, c8.Past(s, [1], [(s.kv[0] - s.q[0]) // s.page * s.page])]


@forms
@pytest.mark.parametrize("byte", [247, 250, 255])
@pytest.mark.parametrize("frame", [1, 16])
def test_unseen_keys_of_overflowing_powers_have_no_influence(form, byte, frame):
    """Finite codes whose power makes them infinite in the model's type, in keys and values that only later rows see: the other
    rows are as if they were not there. (What the later rows get is not defined.)"""
    dtype, heads, kvh, hd, page, q, kv = form
    s = c8.state8(dtype, heads, kvh, hd, page, [q], [kv], seed=60)
    pg, sl = cu.where(s, 0)
    j = kv - q // 2 - 1                               # in the chunk: seen from its middle on
    s.v8.view(torch.uint8)[pg[j], 0, sl[j], ::3] = 126
    s.v8.view(torch.uint8)[pg[j], 0, sl[j], 1::3] = 254
    s.scale[pg[j], 0, sl[j], 1] = byte
    s.scale[pg[-1], kvh - 1, sl[-1], 0] = byte
    c8.decode(s)
    s.v[pg[j], 0, sl[j]] = float("nan")               # the definition's mark of rows that see one
    s.k[pg[-1], kvh - 1, sl[-1]] = float("nan")
    o, lse, pv, qk = c8.attention64(s, frame)
    bound, lse_bound = attention_bound(s, pv.nan_to_num(1e30, 1e30, 1e30), o.nan_to_num(0, 0, 0), qk, kv)
    fine, fine_lse = torch.isfinite(o), torch.isfinite(lse)
    assert fine.any() and not fine.all()
    wdc, ctx = ctx_of(s)
    for past in pasts(s):                             # (the chunk's own sequence: the same result)
        out, z = torch.empty_like(s.x), torch.empty((s.rows, heads), device="cuda")
        kw = {} if past is None else dict(prefix=past.desc(wdc, s))
        ctx.cache8_attention(c8.cache8(wdc, s), cu.chunks(wdc, s), s.x, out, frame=frame, lse=z, **kw)
        got = out.reshape(o.shape).double()
        assert torch.isfinite(got[fine]).all()
        within(got[fine], o[fine], bound[fine], "o")
        within(z[fine_lse], lse[fine_lse], (lse_bound + 4 * EPS32 * lse.abs())[fine_lse], "lse")


@forms
def test_smallest_powers_lose_no_digits(form):
    """Values at the smallest power, 2^-117, under weights of 2^-16 of the largest: the definition's bound, with nothing added.
    Every 32nd key has a score of 15.9 (hd 64) or 16.3 bits above the others' 0, and values of 0, so that a result is the sum of small
    weights times values of 256 to 448 times 2^-117: the products, from 2^-125 on, and their sums are normal float32 numbers."""
    dtype, heads, kvh, hd, page, q, kv = form
    s = c8.state8(dtype, heads, kvh, hd, page, [q], [kv], seed=61)
    pg, sl = cu.where(s, 0)
    tall = torch.arange(kv, device="cuda") % 32 == 0
    k = s.k.double()
    k[pg, :, sl] = torch.where(tall, 1.375 if hd == 64 else 1.0, 0.0).double()[:, None, None].expand(kv, kvh, hd)
    c8.encode(s, k, s.v.double())
    codes = torch.randint(120, 127, (kv, kvh, hd), generator=torch.Generator().manual_seed(62)).cuda()
    s.v8.view(torch.uint8)[pg, :, sl] = torch.where(tall[:, None, None], 0, codes).to(torch.uint8)
    s.scale[pg, :, sl, 1] = 10
    c8.decode(s)
    s.x.fill_(1.0)
    o, lse, pv, qk = c8.attention64(s, 0)
    bound = attention_bound(s, pv, o, qk, kv)[0] - 1e-30
    wdc, ctx = ctx_of(s)
    for past in pasts(s):
        kw = {} if past is None else dict(prefix=past.desc(wdc, s))
        out = ctx.cache8_attention(c8.cache8(wdc, s), cu.chunks(wdc, s), s.x, torch.empty_like(s.x), **kw)
        # (scaled, so that the comparison's own arithmetic is far from the end of float32)
        within(out.reshape(o.shape).double() * 2.0 ** 117, o * 2.0 ** 117, bound * 2.0 ** 117, "o")
