"""Cache attention over scores of every size: far from zero on either side, -inf, rising along the keys."""
import math

import pytest
import torch

from tests import cache_util as cu
from tests.test_gpu_cache import EPS, EPS32, attention_bound, ctx_of, within

pytestmark = pytest.mark.gpu

# dtype, heads, kvh, hd, page, q, kv. On 256 compute units: blocks of 16 and 32 rows, of 128 and of 256, each with
# pages shorter than a tile of 64 keys and not; ranges of keys; float32
FORMS = [("bf16", 4, 4, 64, 64, 3, 700), ("bf16", 4, 4, 128, 16, 20, 700), ("f32", 4, 2, 64, 32, 40, 700),
         ("f32", 2, 2, 128, 64, 40, 700), ("bf16", 4, 4, 128, 64, 1024, 2100)]
FORMS += [("bf16", heads, kvh, hd, page, q, q + 500) for heads, kvh, q in ((4, 4, 200), (16, 1, 4096)) for hd in (64, 128)
          for page in (16, 64)]
forms = pytest.mark.parametrize("form", FORMS, ids=lambda f: "-".join(str(x) for x in f))


def attend(s, frame):
    wdc, ctx = ctx_of(s)
    out, z = torch.empty_like(s.x), torch.empty((s.rows, s.heads), device="cuda")
    ctx.cache_attention(wdc.PagedCache(s.k, s.v), cu.chunks(wdc, s), s.x, out, frame=frame, lse=z)
    return out.reshape(s.rows, s.heads, s.hd), z


@forms
@pytest.mark.parametrize("frame", [0, 24])
@pytest.mark.parametrize("q0,k0", [(-(2.0 ** 46), 2.0 ** 60), (2.0 ** 46, 2.0 ** 60), (-(2.0 ** 16), 2.0 ** 17),
                                   (2.0 ** 16, 2.0 ** 17), (-(2.0 ** 70), 2.0 ** 56), (205 * 2.0 ** 39, 167 * 2.0 ** 53),
                                   (-205 * 2.0 ** 11, 167 * 2.0 ** 12)], ids=str)
def test_equal_scores_of_any_size_give_the_mean(form, frame, q0, k0):
    """q and k have one entry each, of 8 bits, so all scores of a row are the same number without rounding (to which the
    softmax scale adds bits unless both are powers of two)."""
    dtype, heads, kvh, hd, page, q, kv = form
    s = cu.state(dtype, heads, kvh, hd, page, [q], [kv], seed=31)
    pg, sl = cu.where(s, 0)
    s.x.zero_()
    s.x[:, ::hd] = q0
    s.k[pg, :, sl] = 0
    s.k[pg, :, sl, 0] = k0
    out, z = attend(s, frame)
    lim = cu.limits(s, 0, frame)
    v = s.v[pg, :, sl].double()                       # [kv, kvh, hd]
    mean, size = (x.cumsum(0)[lim - 1].repeat_interleave(heads // kvh, 1) / lim[:, None, None] for x in (v, v.abs()))
    # weights are 1: a sum of n terms and their count in float32, one rounding to the type
    within(out, mean, EPS[dtype] * mean.abs() + 2 * (kv + 8) * EPS32 * size, "o")
    # the constants log2 e, ln 2 and sqrt(hd), their quotient and two products, one float32 rounding each; + ln n
    want = q0 * k0 / math.sqrt(hd) + torch.log(lim.double())[:, None].expand(q, heads)
    within(z, want, 8 * EPS32 * want.abs() + 1e-30, "lse")


@forms
@pytest.mark.parametrize("frame", [0, 24])
@pytest.mark.parametrize("late", [False, True])
@pytest.mark.parametrize("q0,k0", [(-(2.0 ** 46), 2.0 ** 60), (2.0 ** 46, 2.0 ** 59), (2.0 ** 16, 2.0 ** 17),
                                   (205 * 2.0 ** 39, 167 * 2.0 ** 52), (-205 * 2.0 ** 11, 167 * 2.0 ** 12)], ids=str)
def test_one_score_far_above_the_others_gives_its_value(form, frame, late, q0, k0):
    dtype, heads, kvh, hd, page, q, kv = form
    s = cu.state(dtype, heads, kvh, hd, page, [q], [kv], seed=32)
    pg, sl = cu.where(s, 0)
    top = 451 if late else 5                          # below the chunk, so every row sees it
    s.x.zero_()
    s.x[:, ::hd] = q0
    s.k[pg, :, sl] = 0
    s.k[pg, :, sl, 0] = k0
    s.k[pg[top], :, sl[top], 0] = 2 * k0 if q0 > 0 else k0 / 2
    out, _ = attend(s, frame)
    want = s.v[pg[top], :, sl[top]].repeat_interleave(heads // kvh, 0)
    assert torch.equal(out, want[None].expand_as(out))


@forms
def test_scores_of_minus_infinity_have_weight_zero(form):
    """More keys at the start than any tile holds score -inf, then ordinary ones follow."""
    dtype, heads, kvh, hd, page, q, kv = form
    s = cu.state(dtype, heads, kvh, hd, page, [q], [kv], seed=33)
    pg, sl = cu.where(s, 0)
    s.x[:, ::hd] = -s.x[:, ::hd].abs() - 0.5
    s.k[pg[:300], :, sl[:300], 0] = math.inf
    out, z = attend(s, 24)
    o, lse, pv, qk = cu.attention64(s, 24)
    bound, lse_bound = attention_bound(s, pv, o, qk, kv)
    within(out, o, bound, "o")
    within(z, lse, lse_bound + 4 * EPS32 * lse.abs(), "lse")


@forms
@pytest.mark.parametrize("frame", [0, 24])
@pytest.mark.parametrize("ramp,size", [(3, 1.0), (40, 1.0), (12, 2.0 ** 80), (40, 2.0 ** 80)], ids=str)
def test_rising_scores_move_the_reference(form, frame, ramp, size):
    """Scores rise along the keys to some 15 to 200 (in half of the rows they fall): the softmax reference moves once or
    in every tile. Values of 2^80 times weights far above 1 would pass float32's range."""
    dtype, heads, kvh, hd, page, q, kv = form
    s = cu.state(dtype, heads, kvh, hd, page, [q], [kv], seed=34)
    pg, sl = cu.where(s, 0)
    rise = torch.linspace(0.1, ramp * (64 / hd) ** 0.5, kv, device="cuda")[:, None, None]
    s.k[pg, :, sl] = (s.k[pg, :, sl].float().abs() * rise).to(s.td)
    s.v *= size
    s.x = s.x.abs()
    s.x[1::2] *= -1
    o, lse, pv, qk = cu.attention64(s, frame)
    bound, lse_bound = attention_bound(s, pv, o, qk, kv)
    out, z = attend(s, frame)
    within(out, o, bound, "o")
    within(z, lse, lse_bound + 4 * EPS32 * lse.abs(), "lse")
