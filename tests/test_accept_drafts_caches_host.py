"""Caches of accept_drafts that overlap, wherever in the list they are, are refused; looking for them takes no longer a cache with many of them.  No kernel is launched."""
import ctypes
import random
import time

import pytest

from test_decoder_abi_host import ERR_ALIGN, ERR_UNSUPPORTED, P, g  # noqa: F401

SIZE = 16 * 2 * 9216


def _status(g, addresses, stray=0):
    table = (ctypes.c_void_p * len(addresses))(*addresses)
    return g.lib().gpusq_accept_drafts(P, P, P, P, P, P, ctypes.addressof(table), len(addresses), P + stray, P, P, P, 70, 2, 40, 9, 16, 2, 128, None)


@pytest.mark.parametrize("layers", [2, 3, 24, 1024])
def test_any_two_that_overlap(g, layers):
    r = random.Random(layers)
    for trial in range(20):
        apart = [P + (1 + i) * SIZE for i in r.sample(range(4 * layers), layers)]
        assert _status(g, apart, stray=2) == ERR_ALIGN  # (nothing overlaps: what is refused is the path's address)
        i, j = r.sample(range(layers), 2)
        apart[i] = apart[j] + r.choice([0, 16, SIZE - 16, 16 - SIZE])
        assert _status(g, apart, stray=2) == ERR_UNSUPPORTED


def test_time_for_many(g):
    """1024 caches against 128: far from the 64 times that all pairs would take (the least of some runs, a factor of 2 above 8 log 1024 / log 128)"""
    def least(layers):
        table = (ctypes.c_void_p * layers)(*[P + i * SIZE for i in random.Random(1).sample(range(layers), layers)])
        call, at, best = g.lib().gpusq_accept_drafts, ctypes.addressof(table), 1.0
        for _ in range(200):
            a = time.perf_counter()
            for _ in range(10):
                call(P, P, P, P, P, P, at, layers, P + 2, P, P, P, 70, 2, 40, 9, 16, 2, 128, None)
            best = min(best, time.perf_counter() - a)
        return best

    assert least(1024) < 24 * least(128)
