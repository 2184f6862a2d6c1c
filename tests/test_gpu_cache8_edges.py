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
