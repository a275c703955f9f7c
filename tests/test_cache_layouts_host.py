"""Which layouts of queries and results the attention over the paged 8-bit cache refuses, without a GPU: every call here is refused, for its
layout or, where that is a good one, for a workspace that is too small (device pointers are made up)."""
import ctypes
import itertools

import pytest

from test_cache_host import attn, cache, lib  # noqa: F401

BAD, NO_SPACE = -1, -3


def call(lib, n, H, s, o, **kw):
    return attn(lib, cache(**kw), n=n, H=H, s=s, o=o, size=256)


def shares(n, H, sn, sh, d):
    """by the definition: two rows of d elements that meet"""
    at = sorted(t * sn + h * sh for t, h in itertools.product(range(n), range(H)))
    return any(b - a < d for a, b in zip(at, at[1:]))


def test_results_that_share_elements(lib):  # noqa: F811
    assert call(lib, 3, 4, (256, 64), (64, 64)) == BAD          # token 0's head 1 is token 1's head 0
    assert b"overlap" in lib.sparge_last_error()
    for n, H in ((3, 4), (4, 2), (2, 6), (9, 2)):
        for sn, sh in itertools.product(range(64, 700, 40), range(64, 700, 40)):
            want = BAD if shares(n, H, sn, sh, 64) else NO_SPACE
            assert call(lib, n, H, (256, 64), (sn, sh)) == want, (n, H, sn, sh)
    assert call(lib, 1 << 30, 128, (256, 64), (1 << 62, 1 << 62)) == BAD
    assert call(lib, 1 << 30, 128, (256, 64), (1 << 62, 64)) == NO_SPACE


@pytest.mark.parametrize("n,H,s,o,want", [(1, 4, (256, 64), (0, 64), NO_SPACE), (3, 1, (64, 64), (64, 0), NO_SPACE), (1, 1, (64, 64), (0, 0), NO_SPACE)])
def test_lone_rows_share_nothing(lib, n, H, s, o, want):  # noqa: F811
    assert call(lib, n, H, s, o, H_kv=1) == want


@pytest.mark.parametrize("n,H,s,o", [(1, 4, (333, 64), (7, 64)), (1, 4, (-8, 64), (-1, 64)), (3, 1, (64, 5), (64, 9)), (1, 1, (3, 3), (5, -5))])
def test_strides_that_say_nothing(lib, n, H, s, o):  # noqa: F811
    """of a dimension of size 1: any number"""
    assert call(lib, n, H, s, o, H_kv=1) == NO_SPACE


@pytest.mark.parametrize("n,H,s,o", [(2, 4, (333, 64), (256, 64)), (3, 2, (128, 60), (128, 64)), (3, 1, (60, 64), (64, 64)), (1, 2, (64, -8), (64, 64)),
                                     (3, 1, (64, 64), (8, 64)), (1, 2, (64, 64), (64, 56))])
def test_strides_that_count(lib, n, H, s, o):  # noqa: F811
    assert call(lib, n, H, s, o, H_kv=1) == BAD


def test_results_in_the_queries_place(lib):  # noqa: F811
    """several workgroups read a token's queries, and one writes its results"""
    rc = attn(lib, Q=8192, O=8192)
    assert rc == BAD and b"overlap" in lib.sparge_last_error(), rc
