"""Refusals of the paged cache operators (no GPU work: every call is refused before a launch)."""
import ctypes as C

import pytest
import torch

from tests import cache_util as cu

ARG, SHAPE, ALIGN, WORKSPACE, UNSUPPORTED = 1, 2, 4, 5, 9


@pytest.fixture(scope="module")
def wdc():
    import paper_2608_01845_amd as pkg
    pkg.load()
    return pkg


def handle(wdc, dtype="bf16", heads=4, hd=64, **kw):
    h = C.c_void_p()
    d = wdc.desc_from_config(cu.config(dtype, heads, 64, **kw))
    d.head_dim = hd
    d.hidden = heads * hd
    assert wdc.load().wdc_create(C.byref(d), None, None, C.byref(h)) == 0
    return h


def descs(**kw):
    from paper_2608_01845_amd._binding import CacheDesc, ChunksDesc
    v = dict(d_k=4096, d_v=8192, pages=8, page=64, kv_heads=4, d_q_start=64, d_kv_len=64, d_table=64, batch=2, table_ld=4,
             rows=10, max_q=10, max_kv=200)
    v.update(kw)
    return (CacheDesc(*[v[n] for n in ("d_k", "d_v", "pages", "page", "kv_heads")], 0),
            ChunksDesc(*[v[n] for n in ("d_q_start", "d_kv_len", "d_table", "batch", "table_ld", "rows", "max_q", "max_kv")], 0))


BAD = [
    (dict(d_k=None), ARG), (dict(d_kv_len=None), ARG), (dict(d_table=None), ARG), (dict(pages=0), ARG), (dict(batch=0), ARG),
    (dict(table_ld=0), ARG), (dict(max_kv=-1), ARG), (dict(page=48), UNSUPPORTED), (dict(page=8), UNSUPPORTED),
    (dict(page=512), UNSUPPORTED), (dict(kv_heads=3), SHAPE), (dict(kv_heads=0), SHAPE), (dict(d_k=4104), ALIGN),
    (dict(d_table=66), ALIGN), (dict(d_kv_len=65), ALIGN), (dict(batch=20000), SHAPE),
    (dict(max_kv=0x7fffffff, table_ld=0x7fffffff), SHAPE), (dict(batch=1, max_kv=(1 << 26) + 1, table_ld=1 << 22), SHAPE),
]
ROWS = [(dict(d_q_start=None), ARG), (dict(rows=-1), ARG), (dict(max_q=-1), ARG), (dict(d_q_start=62), ALIGN),
        (dict(rows=1 << 25, max_q=1), SHAPE), (dict(batch=1000, rows=1 << 20, max_q=1 << 20, max_kv=10), SHAPE)]


@pytest.mark.parametrize("bad,status", BAD + ROWS, ids=lambda x: str(x))
def test_descriptors_are_refused(wdc, bad, status):
    lib, h = wdc.load(), handle(wdc)
    try:
        c, q = descs(**bad)
        c, q = C.byref(c), C.byref(q)
        p = C.c_void_p(1 << 20)
        calls = [lib.wdc_cache_append(h, c, q, p, 768, None, None, None, p, 256),
                 lib.wdc_cache_attention(h, c, q, p, 256, 0, p, 256, None, None, 0),
                 lib.wdc_cache_mass(h, c, q, p, 256, 0, p, 1.0, p, p, None, 0)]
        scratch = [lib.wdc_cache_attention_scratch(h, c, q), lib.wdc_cache_mass_scratch(h, c, q)]
        if (bad, status) in BAD:
            calls.append(lib.wdc_cache_evict(h, c, q, p, p, 4, 0, 0, p, None, p, 1 << 30))
            scratch.append(lib.wdc_cache_evict_scratch(h, c, q, 4))
        assert calls == [status] * len(calls)
        assert scratch == [0] * len(scratch)
        assert lib.wdc_last_error(h)
    finally:
        lib.wdc_destroy(h)


def test_null_descriptors_and_context(wdc):
    lib, h = wdc.load(), handle(wdc)
    c, q = descs()
    p = C.c_void_p(1 << 20)
    try:
        for hh, cc, qq in ((None, C.byref(c), C.byref(q)), (h, None, C.byref(q)), (h, C.byref(c), None)):
            assert lib.wdc_cache_append(hh, cc, qq, p, 768, None, None, None, p, 256) == ARG
            assert lib.wdc_cache_attention(hh, cc, qq, p, 256, 0, p, 256, None, None, 0) == ARG
            assert lib.wdc_cache_mass(hh, cc, qq, p, 256, 0, p, 1.0, p, p, None, 0) == ARG
            assert lib.wdc_cache_evict(hh, cc, qq, p, p, 4, 0, 0, p, None, p, 1 << 30) == ARG
            assert lib.wdc_cache_attention_scratch(hh, cc, qq) == lib.wdc_cache_mass_scratch(hh, cc, qq) == 0
            assert lib.wdc_cache_evict_scratch(hh, cc, qq, 4) == 0
    finally:
        lib.wdc_destroy(h)


def test_tensors_are_refused(wdc):
    lib, h = wdc.load(), handle(wdc)
    c, q = descs()
    c, q = C.byref(c), C.byref(q)
    p, odd = C.c_void_p(1 << 20), C.c_void_p((1 << 20) + 8)
    two = C.c_void_p((1 << 20) + 2)
    try:
        app = lambda a=p, ld=768, pos=None, qw=None, kw=None, o=p, ldq=256: lib.wdc_cache_append(  # noqa: E731
            h, c, q, a, ld, pos, qw, kw, o, ldq)
        assert app(a=None) == ARG and app(o=None) == ARG and app(ld=760) == ARG and app(ldq=248) == ARG
        assert app(a=odd) == app(o=odd) == app(ld=772) == app(ldq=260) == app(qw=odd) == app(kw=odd) == app(pos=two) == ALIGN
        assert app(ld=(1 << 22) + 8) == app(ldq=(1 << 22) + 8) == SHAPE
        att = lambda x=p, ld=256, f=0, o=p, ldo=256, z=None, sc=None: lib.wdc_cache_attention(  # noqa: E731
            h, c, q, x, ld, f, o, ldo, z, sc, 64)
        assert att(x=None) == att(o=None) == att(ld=248) == att(ldo=248) == att(f=-1) == ARG
        assert att(x=odd) == att(o=odd) == att(ld=260) == att(ldo=260) == att(z=two) == att(sc=odd) == ALIGN
        mass = lambda x=p, ld=256, f=0, z=p, d=1.0, m=p, o=p, sc=None: lib.wdc_cache_mass(  # noqa: E731
            h, c, q, x, ld, f, z, d, m, o, sc, 64)
        assert mass(x=None) == mass(z=None) == mass(m=None) == mass(o=None) == mass(f=-1) == ARG
        assert mass(d=float("nan")) == mass(d=float("inf")) == mass(ld=8) == ARG
        assert mass(x=odd) == mass(ld=260) == mass(z=two) == mass(m=two) == mass(o=two) == mass(sc=odd) == ALIGN
        ev = lambda m=p, o=p, k=4, s=0, r=0, n=p, i=None, sc=p, b=1 << 30: lib.wdc_cache_evict(  # noqa: E731
            h, c, q, m, o, k, s, r, n, i, sc, b)
        assert ev(m=None) == ev(o=None) == ev(n=None) == ev(k=0) == ev(s=-1) == ev(r=-1) == ev(s=3, r=2) == ARG
        assert ev(s=0x7fffffff, r=0x7fffffff) == ARG
        assert ev(k=0x7fffffff, i=p) == ev(k=(1 << 25) + 1, i=p) == SHAPE
        assert ev(sc=None) == ev(b=8) == WORKSPACE
        assert ev(m=two) == ev(o=two) == ev(n=two) == ev(i=two) == ev(sc=odd) == ALIGN
        need = lib.wdc_cache_evict_scratch(h, c, q, 50)
        assert need >= 2 * 4 * 2 * 50 * 4              # 50 moves of 8 bytes per sequence and kv head
        assert lib.wdc_cache_evict(h, c, q, p, p, 50, 0, 0, p, None, p, need - 1) == WORKSPACE
    finally:
        lib.wdc_destroy(h)


def test_head_sizes_and_rotary_dims_are_refused(wdc):
    lib = wdc.load()
    c, q = descs()
    p = C.c_void_p(1 << 20)
    h = handle(wdc, hd=96)
    assert lib.wdc_cache_attention(h, C.byref(c), C.byref(q), p, 384, 0, p, 384, None, None, 0) == UNSUPPORTED
    lib.wdc_destroy(h)
    for rope in ((16, 24, 22), (15, 25, 24), (-16, 56, 24)):
        h = handle(wdc, rope=rope)
        assert lib.wdc_cache_append(h, C.byref(c), C.byref(q), p, 768, p, None, None, p, 256) == SHAPE
        lib.wdc_destroy(h)


def test_python_descriptors_check_tensors(wdc):
    k = torch.zeros((4, 2, 16, 64))
    wdc.PagedCache(k, k.clone())
    for bad in (k[..., :32], k.double(), k.transpose(1, 2), k[0]):
        with pytest.raises(ValueError):
            wdc.PagedCache(k, bad)
        with pytest.raises(ValueError):
            wdc.PagedCache(bad, k)
    with pytest.raises(ValueError):
        wdc.PagedCache(k.transpose(2, 3), k.transpose(2, 3))
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    wdc.Chunks(i(3), i(2), i(2, 5), rows=4)
    for a in ((i(2), i(2), i(2, 5)), (i(3), i(2), i(3, 5)), (i(3).long(), i(2), i(2, 5)), (i(3), i(2), i(5)),
              (i(6)[::2], i(2), i(2, 5)), (i(3), i(2), i(5, 2).T)):
        with pytest.raises(ValueError):
            wdc.Chunks(*a, rows=4)


@pytest.mark.parametrize("bad", [dict(rows=1 << 32), dict(rows=-1), dict(max_q=1 << 31), dict(max_kv=1 << 32), dict(max_kv=-1)],
                         ids=str)
def test_bounds_that_32_bits_would_cut_are_refused(wdc, bad):
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError):
        wdc.Chunks(i(3), i(2), i(2, 5), **{**dict(rows=4), **bad})
