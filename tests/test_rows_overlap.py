"""Rows that are written must not lie on one another: every pair of strides against a plain search, on the host.  No call
here reaches a kernel launch."""
import ctypes as ct
import itertools

import pytest

import paper_2609_35065_amd as kv

A = 1 << 20   # a 16-byte aligned address; nothing reads it


def _status(num, heads, ts, hs):
    """Status of a rotary append with these rows as its result: stopped behind the check of the rows, by positions at an
    odd address (KV_EALIGN)."""
    layout = kv.make_layout(1, 1, 64, 2, 16, 16, 20, 1, 20 * 2048, 2048)
    b = kv.KvBatch(1, 4, num, num, 10, A, A, A)
    q = kv.KvRows(A, heads * 64, 64, heads, kv.KV_BF16)
    out = kv.KvRows(A, ts, hs, heads, kv.KV_BF16)
    p = ct.addressof
    return kv.lib().kv_rope_append(p(layout), A, p(b), p(q), p(out), None, None, A, 64, 0, 1.0, A + 2, kv.KV_BF16, None, None,
                                   None)


def _overlap(num, heads, ts, hs):
    at = sorted(t * ts + h * hs for t in range(num) for h in range(heads))
    return any(b - a < 64 for a, b in zip(at, at[1:]))


@pytest.mark.parametrize("num,heads", [(1, 1), (1, 5), (2, 1), (2, 2), (3, 2), (2, 3), (5, 4), (7, 5)])
def test_overlap(num, heads):
    for ts, hs in itertools.product(range(0, 520, 8), repeat=2):
        assert _status(num, heads, ts, hs) == (kv.KV_EINVAL if _overlap(num, heads, ts, hs) else kv.KV_EALIGN), (ts, hs)


def test_large_strides():
    big = 1 << 62
    for num, heads, ts, hs in ((3, 3, big, 64), (3, 3, 192, big), (3, 3, big, big + 64), (1 << 14, 1 << 14, 64, 64 << 14),
                               (1 << 14, 1 << 14, 64 << 14, 64)):
        assert _status(num, heads, ts, hs) == kv.KV_EALIGN, (ts, hs)
    for num, heads, ts, hs in ((3, 3, big, big), (1 << 14, 1 << 14, 64, (64 << 14) - 8), (3, 65536, (1 << 30) + 56, 1 << 15)):
        assert _status(num, heads, ts, hs) == kv.KV_EINVAL, (ts, hs)
