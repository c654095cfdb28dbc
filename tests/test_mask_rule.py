"""Which keys a row of a document sees, with g++ (no GPU): against the statement in whole numbers of any size, and at the ends of 32 bits."""
import ctypes as C

import numpy as np
import pytest

from oracle import layers as L
from test_dispatch_rules import _compile

SOURCE = r"""
#include "mask_rule.hpp"
extern "C" void seen(int r, int start, int end, int causal, int has_prefix, int prefix, int window, int* out) {
    mp::seen_in_document(r, start, end, causal, has_prefix != 0, prefix, window, out[0], out[1]);
}
"""


@pytest.fixture(scope="module")
def seen(tmp_path_factory):
    lib, out = _compile(str(tmp_path_factory.mktemp("mask")), "mask", SOURCE), (C.c_int * 2)()

    def ask(*a):
        lib.seen(*a, out)
        return tuple(out)
    return ask


def stated(r, start, end, causal, has_prefix, prefix, window):
    lo, hi = start, r + 1 if causal else end
    if has_prefix:
        hi = max(hi, min(end, start + prefix))
    if window:
        lo, hi = max(lo, r - window + 1), min(hi, r + window)
    return lo, hi


def test_small_documents(seen):
    for start, end in ((0, 1), (0, 7), (5, 12), (3, 4)):
        for causal in (0, 1):
            for r in range(start, end):
                for window in range(0, 10):
                    assert seen(r, start, end, causal, 0, 0, window) == stated(r, start, end, causal, 0, 0, window)
                for prefix in range(-3, 10):
                    assert seen(r, start, end, causal, 1, prefix, 0) == stated(r, start, end, causal, 1, prefix, 0)


def test_the_oracle_says_the_same(seen):
    start, prefix = [2, 9, 9, 20], [3, 1, 30]
    for kw in (dict(), dict(causal=True), dict(causal=True, prefix=prefix), dict(window=3), dict(causal=True, window=4)):
        lo, hi = L.attention_ranges(22, start, **kw)
        for b in (0, 2):
            for r in range(start[b], start[b + 1]):
                got = seen(r, start[b], start[b + 1], int(kw.get("causal", False)), int("prefix" in kw), prefix[b], kw.get("window", 0))
                assert got == (lo[r], hi[r])


MOST = 0x7FFFFF00
BIG = 2 ** 31 - 1


@pytest.mark.parametrize("start,end", [(0, MOST), (MOST - 10, MOST), (1200000000, MOST), (5, 1200000000)])
def test_rows_near_two_to_the_31(seen, start, end):
    """Windows and prefixes whose sum with a row passes 2^31."""
    r = np.random.default_rng(start % 1000)
    for at in sorted({start, start + 1, end - 1, (start + end) // 2, *(int(x) for x in r.integers(start, end, 20))}):
        for n in (1, 2, 63, 1100000000, MOST - 1, MOST, BIG - 1, BIG, *(int(x) for x in r.integers(1, BIG, 20))):
            for causal in (0, 1):
                assert seen(at, start, end, causal, 0, 0, n) == stated(at, start, end, causal, 0, 0, n)
            for prefix in (n, -n, 0, -BIG - 1):
                assert seen(at, start, end, 1, 1, prefix, 0) == stated(at, start, end, 1, 1, prefix, 0)
