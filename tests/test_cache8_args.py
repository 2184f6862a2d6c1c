"""Refusals of the 8-bit cache's operators and of attention over a shared past (every call is refused before a launch),
and the tests' own definition of the codes."""
import ctypes as C
import math

import pytest
import torch

from tests import cache8_util as c8
from tests.test_cache_args import ALIGN, ARG, BAD, ROWS, SHAPE, WORKSPACE, descs, handle, wdc  # noqa: F401

P = C.c_void_p(1 << 20)
ODD, TWO = C.c_void_p((1 << 20) + 8), C.c_void_p((1 << 20) + 2)


def descs8(**kw):
    from paper_2608_01845_amd._binding import Cache8Desc, PrefixDesc
    c, q = descs(**{k: v for k, v in kw.items() if k not in ("d_scale", "d_group_start", "d_prefix_len", "groups", "max_prefix", "max_own")})
    v = dict(d_scale=16384, d_group_start=64, d_prefix_len=64, groups=1, max_prefix=128, max_own=100)
    v.update(kw)
    return (Cache8Desc(c.d_k, c.d_v, v["d_scale"], c.pages, c.page, c.kv_heads, 0), c, q,
            PrefixDesc(*[v[n] for n in ("d_group_start", "d_prefix_len", "groups", "max_prefix", "max_own")], 0))


def calls(lib, h, c8d, c, q, p):
    big = 1 << 40
    return [lib.wdc_cache8_append(h, c8d, q, P, 768, None, None, None, P, 256), lib.wdc_cache8_read(h, c8d, q, P, 256, P, 256),
            lib.wdc_cache8_attention(h, c8d, q, None, P, 256, 0, P, 256, None, None, 0),
            lib.wdc_cache8_attention(h, c8d, q, p, P, 256, 0, P, 256, None, P, big),
            lib.wdc_cache_attention_shared(h, c, q, p, P, 256, 0, P, 256, None, P, big)]


@pytest.mark.parametrize("bad,status", BAD + ROWS, ids=str)
def test_descriptors_are_refused(wdc, bad, status):  # noqa: F811
    lib, h = wdc.load(), handle(wdc)
    try:
        d = [C.byref(x) for x in descs8(**bad)]
        assert calls(lib, h, *d) == [status] * 5
        assert lib.wdc_cache8_attention_scratch(h, d[0], d[2], None) == lib.wdc_cache8_attention_scratch(h, d[0], d[2], d[3]) == 0
        assert lib.wdc_cache_attention_shared_scratch(h, d[1], d[2], d[3]) == 0
        assert lib.wdc_last_error(h)
    finally:
        lib.wdc_destroy(h)


@pytest.mark.parametrize("bad,status", [
    (dict(d_group_start=None), ARG), (dict(d_prefix_len=None), ARG), (dict(groups=0), ARG), (dict(groups=-1), ARG),
    (dict(max_prefix=-1), ARG), (dict(max_own=-1), ARG), (dict(d_group_start=66), ALIGN), (dict(d_prefix_len=65), ALIGN),
    (dict(groups=20000), SHAPE), (dict(groups=16000, max_kv=1 << 24, table_ld=1 << 20, max_prefix=1 << 13), SHAPE)], ids=str)
def test_prefixes_are_refused(wdc, bad, status):  # noqa: F811
    lib, h = wdc.load(), handle(wdc)
    try:
        d = [C.byref(x) for x in descs8(**bad)]
        assert calls(lib, h, *d)[3:] == [status] * 2
        assert lib.wdc_cache8_attention_scratch(h, d[0], d[2], d[3]) == lib.wdc_cache_attention_shared_scratch(h, d[1], d[2], d[3]) == 0
    finally:
        lib.wdc_destroy(h)


def test_tensors_are_refused(wdc):  # noqa: F811
    lib, h = wdc.load(), handle(wdc)
    try:
        for bad, status in ((dict(d_scale=None), ARG), (dict(d_scale=4104), ALIGN)):
            d = [C.byref(x) for x in descs8(**bad)]
            assert calls(lib, h, *d)[:4] == [status] * 4
        c, m, q, p = (C.byref(x) for x in descs8())
        app = lambda a=P, ld=768, pos=None, qw=None, kw=None, o=P, ldq=256: lib.wdc_cache8_append(  # noqa: E731
            h, c, q, a, ld, pos, qw, kw, o, ldq)
        assert app(a=None) == app(o=None) == app(ld=760) == app(ldq=248) == ARG
        assert app(a=ODD) == app(o=ODD) == app(ld=772) == app(ldq=260) == app(qw=ODD) == app(kw=ODD) == app(pos=TWO) == ALIGN
        assert app(ld=(1 << 22) + 8) == app(ldq=(1 << 22) + 8) == SHAPE
        read = lambda k=P, lk=256, v=P, lv=256: lib.wdc_cache8_read(h, c, q, k, lk, v, lv)  # noqa: E731
        assert read(k=None, v=None) == read(lk=248) == read(lv=8) == read(k=None, lv=0) == ARG
        assert read(k=ODD) == read(v=ODD) == read(lk=260) == read(lv=260) == ALIGN
        assert read(lk=(1 << 22) + 8) == read(v=None, lk=(1 << 22) + 8) == SHAPE
        for pre in (None, p):
            att = lambda x=P, ld=256, f=0, o=P, lo=256, z=None, sc=P: lib.wdc_cache8_attention(  # noqa: E731
                h, c, q, pre, x, ld, f, o, lo, z, sc, 1 << 40)
            assert att(x=None) == att(o=None) == att(ld=248) == att(lo=248) == att(f=-1) == ARG
            assert att(x=ODD) == att(o=ODD) == att(ld=260) == att(lo=260) == att(z=TWO) == att(sc=ODD) == ALIGN
        sh = lambda pre=p, x=P, ld=256, f=0, o=P, lo=256, z=None, sc=P, n=1 << 40: lib.wdc_cache_attention_shared(  # noqa: E731
            h, m, q, pre, x, ld, f, o, lo, z, sc, n)
        assert sh(pre=None) == sh(x=None) == sh(o=None) == sh(ld=248) == sh(lo=248) == sh(f=-1) == ARG
        assert sh(x=ODD) == sh(o=ODD) == sh(ld=260) == sh(lo=260) == sh(z=TWO) == sh(sc=ODD) == ALIGN
        need = lib.wdc_cache_attention_shared_scratch(h, m, q, p)
        assert need >= 2 * 10 * 4 * 66 * 4             # two parts of 10 rows, 4 heads
        assert sh(sc=None) == sh(n=need - 1) == WORKSPACE
        need = lib.wdc_cache8_attention_scratch(h, c, q, p)
        assert need >= 2 * 10 * 4 * 66 * 4
        assert lib.wdc_cache8_attention(h, c, q, p, P, 256, 0, P, 256, None, P, need - 1) == WORKSPACE
        assert lib.wdc_cache8_attention(h, c, q, p, P, 256, 0, P, 256, None, None, need) == WORKSPACE
        for hh, cc, mm, qq in ((None, c, m, q), (h, None, None, q), (h, c, m, None)):
            assert calls(lib, hh, cc, mm, qq, p) == [ARG] * 5
    finally:
        lib.wdc_destroy(h)


def test_python_descriptors_check_tensors(wdc):  # noqa: F811
    k = torch.zeros((4, 2, 16, 64)).to(torch.float8_e4m3fn)
    e = torch.zeros((4, 2, 16, 2), dtype=torch.uint8)
    wdc.PagedCache8(k, k.clone(), e)
    for bad in (k[..., :32], k.float(), k.view(torch.uint8), k.transpose(1, 2), k[0]):
        with pytest.raises(ValueError):
            wdc.PagedCache8(k, bad, e)
        with pytest.raises(ValueError):
            wdc.PagedCache8(bad, k, e)
    for bad in (e[..., :1], e.int(), e[:3], e.transpose(0, 1), e.view(torch.float8_e8m0fnu)):
        with pytest.raises(ValueError):
            wdc.PagedCache8(k, k, bad)
    t = k.view(torch.uint8).transpose(2, 3).view(torch.float8_e4m3fn)
    with pytest.raises(ValueError):
        wdc.PagedCache8(t, t, torch.zeros((4, 2, 64, 2), dtype=torch.uint8))
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    wdc.Prefix(i(3), i(2))
    for a in ((i(2), i(2)), (i(3).long(), i(2)), (i(3), i(2).float()), (i(6)[::2], i(2)), (i(3, 1), i(2))):
        with pytest.raises(ValueError):
            wdc.Prefix(*a)
    for kw in (dict(max_prefix=-1), dict(max_own=1 << 31)):
        with pytest.raises(ValueError):
            wdc.Prefix(i(3), i(2), **kw)


def test_codes_of_the_definition():
    """The table and the rounding of the tests' own definition against torch's type."""
    every = torch.arange(256, dtype=torch.uint8)
    one = c8.values64(every, torch.full((), 127, dtype=torch.uint8))
    want = every.view(torch.float8_e4m3fn).double()
    assert torch.equal(one.nan_to_num(1e9), want.nan_to_num(1e9))
    g = torch.Generator().manual_seed(1)
    x = torch.randn((4000, 64), generator=g).double()
    x[:, 5] = 0
    x[7] = 0
    x[8:2000] *= torch.exp2(torch.randint(-20, 3, (1992, 64), generator=g).double())
    x[9, 3], x[9, 4], x[9, 5] = math.nan, math.inf, -math.inf
    x[10] *= 2.0 ** -130
    x[11] = 0
    x[11, 0] = 448 * 2.0 ** 3
    x[12] = x[11]
    x[12, 1] = 448 * 2.0 ** 3 * (1 + 2.0 ** -40)
    code, byte = c8.quantised64(x)
    assert byte[7] == 10 and byte[10] == 10 and byte[11] == 130 and byte[12] == 131
    y = torch.ldexp(x, 127 - byte.int()[:, None])
    assert torch.equal(code.view(torch.float8_e4m3fn).float()[13:], y[13:].to(torch.float8_e4m3fn).float())
    assert torch.isnan(c8.values64(code, byte)[9, 3:6]).all()
    size = x[13:].abs().amax(1) / torch.exp2(byte[13:].double() - 127)
    assert (size <= 448).all() and (size > 224).all()
