"""Largest calls over a shared past: shared keys count once, not once per sequence (no GPU work)."""
import ctypes as C

import pytest

from tests.test_cache8_args import P, descs8
from tests.test_cache_args import ARG, SHAPE, WORKSPACE, handle, wdc  # noqa: F401

# 128 rollouts of 32 kv heads off 67,200 shared keys: 2.8e8 keys if each rollout had its own, 2.2e6 + 5e5 so
BIG = dict(pages=2000, kv_heads=32, batch=128, table_ld=1053, rows=128, max_q=1, max_kv=67320, groups=1, max_prefix=67200,
           max_own=120)


def answers(wdc, **kw):  # noqa: F811
    """Scratch and statuses (of calls with a byte too little) of both attentions."""
    lib, h = wdc.load(), handle(wdc, heads=32)
    try:
        c8d, c, q, p = (C.byref(x) for x in descs8(**kw))
        n = [lib.wdc_cache8_attention_scratch(h, c8d, q, p), lib.wdc_cache_attention_shared_scratch(h, c, q, p)]
        st = [lib.wdc_cache8_attention(h, c8d, q, p, P, 2048, 0, P, 2048, None, P, max(n[0], 1) - 1),
              lib.wdc_cache_attention_shared(h, c, q, p, P, 2048, 0, P, 2048, None, P, max(n[1], 1) - 1)]
        return n, st
    finally:
        lib.wdc_destroy(h)


def test_shared_keys_count_once(wdc):  # noqa: F811
    n, st = answers(wdc, **BIG)
    assert st == [WORKSPACE] * 2
    assert min(n) >= 2 * 128 * 32 * 66 * 4            # two parts of every row and head
    lib, h = wdc.load(), handle(wdc, heads=32)
    try:                                              # without a prefix they count for every sequence
        c8d, c, q, _ = (C.byref(x) for x in descs8(**BIG))
        assert lib.wdc_cache8_attention(h, c8d, q, None, P, 2048, 0, P, 2048, None, None, 0) == SHAPE
        assert lib.wdc_cache_attention(h, c, q, P, 2048, 0, P, 2048, None, None, 0) == SHAPE
        assert lib.wdc_cache_attention_scratch(h, c, q) == lib.wdc_cache8_attention_scratch(h, c8d, q, None) == 0
    finally:
        lib.wdc_destroy(h)


@pytest.mark.parametrize("bad,status", [
    (dict(max_own=0x7fffffff), SHAPE),                            # no bound on the own keys: all of them
    (dict(max_own=(1 << 16) + 1), SHAPE),                         # 128 * 32 * own
    (dict(groups=127, max_prefix=67200, max_own=0), SHAPE),       # groups * 32 * prefix
    (dict(batch=1, rows=1, max_kv=(1 << 23) + 1, table_ld=1 << 18, max_own=0), SHAPE),   # one sequence's
    (dict(max_own=-1), ARG)], ids=str)
def test_other_keys_still_count(wdc, bad, status):  # noqa: F811
    assert answers(wdc, **{**BIG, **bad}) == ([0, 0], [status] * 2)


@pytest.mark.parametrize("most", [dict(max_own=1 << 16), dict(groups=124), dict(batch=1, rows=1, max_kv=1 << 23, table_ld=1 << 18)], ids=str)
def test_the_limits_themselves_are_allowed(wdc, most):  # noqa: F811
    n, st = answers(wdc, **{**BIG, **most})
    assert st == [WORKSPACE] * 2 and min(n) > 0
