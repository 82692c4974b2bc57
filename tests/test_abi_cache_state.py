"""Host-side checks of what the calls on the cache take beside their numbers: its state, its descriptor, sizes that a launch cannot hold (no GPU needed)."""
import ctypes

import pytest

from tests.test_abi_cache import ALIGN, FAKE, UNSUPPORTED, _attend, _append, _cache, cq  # noqa: F401


def test_the_place_for_what_lacked(cq):  # noqa: F811
    for call in (lambda f: _append(cq, f), lambda f: _attend(cq, f),
                 lambda f: cq.lib.cafeq_cache_reserve(ctypes.byref(_cache(cq, **f)), FAKE, 1, FAKE, FAKE, FAKE, None)):
        assert call(dict(missing=FAKE + 2)) == ALIGN
    assert _append(cq, dict(missing=FAKE), n=0) == 0 and _attend(cq, dict(missing=FAKE), n=0) == 0


def _host_cache(cq, **more):  # noqa: F811
    """A cache in host memory: its descriptor is made and kept the same way, and nothing is launched."""
    import torch
    return torch, cq.kv_cache(3, 20, more.get("heads", 16), more.get("d", 32), block=16, width=4, device=torch.device("cpu"))


def _strided(torch, cache):
    # a table whose rows lie apart takes the place of one whose rows do not: same memory, address and shape
    base = torch.zeros((3, 8), dtype=torch.int32)
    cache.table = base.view(-1)[:12].view(3, 4)
    return lambda: cache.table.set_(base[:, :4])


CHANGES = {
    "v turned": lambda torch, c: lambda: c.v.transpose_(2, 3),
    "k turned, of the same shape": lambda torch, c: lambda: c.k.transpose_(1, 2),
    "v viewed": lambda torch, c: lambda: c.v.set_(c.v.view(20, 16, 16, 32)),
    "k shorter": lambda torch, c: lambda: c.k.set_(c.k[:, :, :, :16]),
    "fewer pages of v": lambda torch, c: lambda: c.v.set_(c.v[:19]),
    "lengths shorter": lambda torch, c: lambda: c.lengths.set_(c.lengths[:2]),
    "refs shorter": lambda torch, c: lambda: c.refs.resize_(7),
    "scales of k shorter": lambda torch, c: lambda: c.kscale.set_(c.kscale[:3]),
    "scales of v turned": lambda torch, c: lambda: c.vscale.transpose_(0, 1),
    "missing empty": lambda torch, c: lambda: c.missing.set_(c.missing[:0]),
    "rows of the table apart": _strided,
    "table of another type": lambda torch, c: lambda: setattr(c, "table", c.table.long()),
}


@pytest.mark.parametrize("what", CHANGES)
def test_a_cache_whose_tensors_change_their_form_is_checked_again(cq, what):  # noqa: F811
    torch, cache = _host_cache(cq)
    change = CHANGES[what](torch, cache)
    kept = cq._cache(cache, -1)
    assert cq._cache(cache, -1) is kept
    cache.lengths.add_(3)
    cache.k.zero_()
    assert cq._cache(cache, -1) is kept      # contents are free to change
    change()
    with pytest.raises(cq.CafeqError):
        cq._cache(cache, -1)


@pytest.mark.parametrize("heads,heads_q,n,sequences,d", [(257, 257, 100, 65535, 128), (1, 128, (1 << 24) - 1, 2, 16), (1, 1024, (1 << 21) - 1, 9, 64), (4096, 4096, 128, 4096, 256)])
def test_more_threads_than_a_launch_holds(cq, heads, heads_q, n, sequences, d):  # noqa: F811
    cache = dict(heads=heads, sequences=sequences, d=d)
    far = dict(ldq=1 << 20, ldo=1 << 20, hsq=d, hso=d, heads_q=heads_q, n=n, longest=n, out=1 << 46, dtype=1)
    assert _attend(cq, cache, size=True, **far) == 0
    assert _attend(cq, cache, ws=FAKE, **far) == UNSUPPORTED


@pytest.mark.parametrize("heads,sequences", [(4096, 65535), (7, 65535), (4096, 60000)])
def test_room_that_no_sequence_fills_takes_no_workspace(cq, heads, sequences):  # noqa: F811
    """2^30 tokens of room a sequence: more parts than a launch should have are not cut, nor room for them asked."""
    cache = dict(heads=heads, sequences=sequences, d=16, width=1 << 26)
    size = _attend(cq, cache, size=True, heads_q=heads, n=10, longest=1, ldq=1 << 20, ldo=1 << 20, hsq=16, hso=16, out=1 << 46)
    assert size <= 16384 * 4 * 16 * (16 + 2) * 4
