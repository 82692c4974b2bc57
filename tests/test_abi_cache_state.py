"""Host-side checks of what the calls on the cache take beside their numbers: its state, its descriptor, sizes that a launch cannot hold (no GPU needed)."""
import ctypes

import pytest

from tests.test_abi_cache import ALIGN, FAKE, _attend, _append, _cache, cq  # noqa: F401


def test_the_place_for_what_lacked(cq):  # noqa: F811
    for call in (lambda f: _append(cq, f), lambda f: _attend(cq, f),
                 lambda f: cq.lib.cafeq_cache_reserve(ctypes.byref(_cache(cq, **f)), FAKE, 1, FAKE, FAKE, FAKE, None)):
        assert call(dict(missing=FAKE + 2)) == ALIGN
    assert _append(cq, dict(missing=FAKE), n=0) == 0 and _attend(cq, dict(missing=FAKE), n=0) == 0
