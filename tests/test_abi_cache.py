"""Host-side checks of the calls on positions, cache and attention: what they refuse, before anything is launched (no GPU needed)."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2511_19705_amd", "libcafeq.so")
FAKE = 1 << 20        # a non-null, aligned address that is never dereferenced on these paths
FAR = 1 << 40
INVALID, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE = -1, -2, -3, -4, -7


@pytest.fixture(scope="module")
def cq():
    if not os.path.exists(LIB):
        import __graft_entry__ as ge
        ge.build()
    from paper_2511_19705_amd import cafeq
    return cafeq


def _rotate(cq, n=4, cfg=None, q=None, k=None, positions=FAKE, freq=FAKE, **more):
    c = dict(dtype=0, d=64, rot=64, interleaved=0, norm=1, eps=1e-6, gain_offset=1.0, amplitude=1.0)
    c.update(more)
    cfg = cq.Rotation(**c)

    def part(p, at):
        if p is None:
            return None
        f = dict(x=at, out=at + FAR, ldx=256, hsx=64, ldo=256, hso=64, heads=4, gain=None)
        f.update(p)
        return ctypes.byref(cq.Heads(**f))

    return cq.lib.cafeq_rotate_heads(ctypes.byref(cfg), part(q, FAKE), part(k, FAKE + (1 << 30)), n, positions, freq, None)


def test_rotation_refuses(cq):
    assert cq.lib.cafeq_rotate_heads(None, None, None, 1, FAKE, FAKE, None) == INVALID
    assert _rotate(cq) == INVALID                                   # neither part
    assert _rotate(cq, q={}, n=0) == 0
    assert _rotate(cq, q={}, k={}, n=0) == 0
    assert _rotate(cq, q={}, positions=None) == INVALID
    assert _rotate(cq, q={}, freq=None) == INVALID
    assert _rotate(cq, q={}, freq=None, rot=0, n=0) == 0
    assert _rotate(cq, q={}, dtype=2) == INVALID
    assert _rotate(cq, q={"out": None}) == INVALID
    assert _rotate(cq, q={}, n=-1) == SHAPE
    for d, rot in ((63, 62), (0, 0), (64, 66), (64, 3), (64, -2)):
        assert _rotate(cq, q={}, d=d, rot=rot) == SHAPE
    assert _rotate(cq, q={"heads": 0}) == SHAPE
    assert _rotate(cq, q={"ldo": 255}) == SHAPE                     # tokens of the result over each other
    assert _rotate(cq, q={"hso": 63}) == SHAPE
    assert _rotate(cq, q={"ldx": -1}) == SHAPE
    assert _rotate(cq, q={"ldo": 64, "hso": 4 * 64}, n=0) == 0      # heads behind each other
    assert _rotate(cq, q={}, d=514, rot=0) == UNSUPPORTED
    assert _rotate(cq, q={}, n=(1 << 21) + 1) == UNSUPPORTED
    assert _rotate(cq, q={"heads": 4097, "ldx": 1 << 20, "ldo": 1 << 20}) == UNSUPPORTED
    assert _rotate(cq, q={"x": FAKE + 2}) == ALIGN
    assert _rotate(cq, q={"gain": FAKE + 2}) == ALIGN
    assert _rotate(cq, q={}, positions=FAKE + 1) == ALIGN
    assert _rotate(cq, q={}, freq=FAKE + 4) == ALIGN
    assert _rotate(cq, q={"out": FAKE + 64}) == INVALID             # over the input, not in its place
    assert _rotate(cq, q={"out": FAKE, "ldo": 320}) == INVALID
    assert _rotate(cq, q={}, k={"out": FAKE}) == INVALID            # over the other part's input
    assert _rotate(cq, q={}, k={"out": FAKE + FAR + 128}) == INVALID   # and over its result


def _cache(cq, **more):
    f = dict(k=FAKE, v=FAKE, kscale=FAKE, vscale=FAKE, table=FAKE, lengths=FAKE, refs=FAKE, pages=10, sequences=3, width=4, heads=2, d=64, block=16)
    f.update(more)
    return cq.Cache(**f)


BAD_CACHES = ([({n: None}, INVALID) for n in ("k", "v", "kscale", "vscale", "table", "lengths")] +
              [({n: FAKE + 2}, ALIGN) for n in ("k", "v", "kscale", "vscale", "table", "lengths", "refs")] +
              [(dict(sequences=-1), SHAPE), (dict(width=0), SHAPE), (dict(heads=0), SHAPE), (dict(pages=0), SHAPE), (dict(d=0), SHAPE), (dict(d=40), SHAPE),
               (dict(d=272), UNSUPPORTED), (dict(block=8), UNSUPPORTED), (dict(block=48), UNSUPPORTED), (dict(block=256), UNSUPPORTED),
               (dict(sequences=65537), UNSUPPORTED), (dict(heads=4097), UNSUPPORTED), (dict(pages=1 << 31), UNSUPPORTED),
               (dict(pages=1 << 30, heads=2), UNSUPPORTED), (dict(width=1 << 27), UNSUPPORTED)])


def _append(cq, cache=None, k=FAKE, v=FAKE, dtype=0, n=2, ld=128, hs=64, starts=FAKE, longest=2, **more):
    c = _cache(cq, **(cache or {}))
    return cq.lib.cafeq_cache_append(ctypes.byref(c), k, v, dtype, n, more.get("ldk", ld), more.get("hsk", hs), more.get("ldv", ld), more.get("hsv", hs),
                                     starts, longest, None)


def _values(cq, cache=None, begin=FAKE, starts=FAKE, n=2, k=FAKE, v=FAKE, dtype=0):
    c = _cache(cq, **(cache or {}))
    return cq.lib.cafeq_cache_values(ctypes.byref(c), begin, starts, n, k, v, dtype, None)


def _attend(cq, cache=None, ws=None, size=False, **more):
    c = _cache(cq, **(cache or {}))
    f = dict(q=FAKE, out=FAR, lse=None, n=2, ldq=256, hsq=64, ldo=256, hso=64, longest=2, starts=FAKE, dtype=0, heads_q=4, causal=1, window=0, scale=0.125,
             softcap=0.0)
    f.update(more)
    a = cq.Attention(**f)
    if size:
        return cq.lib.cafeq_cache_attend_workspace_bytes(ctypes.byref(c), ctypes.byref(a))
    return cq.lib.cafeq_cache_attend(ctypes.byref(c), ctypes.byref(a), ws, None)


@pytest.mark.parametrize("bad,code", BAD_CACHES)
def test_every_call_refuses_the_cache(cq, bad, code):
    c = _cache(cq, **bad)
    calls = [lambda: _append(cq, bad), lambda: _values(cq, bad), lambda: _attend(cq, bad),
             lambda: cq.lib.cafeq_cache_reserve(ctypes.byref(c), FAKE, 1, FAKE, FAKE, FAKE, None),
             lambda: cq.lib.cafeq_cache_reorder(ctypes.byref(c), FAKE, FAKE, None), lambda: cq.lib.cafeq_cache_compact(ctypes.byref(c), FAKE, FAKE, None)]
    for call in calls:
        assert call() == code
    assert cq.lib.cafeq_cache_pages_workspace_bytes(ctypes.byref(c)) == 0
    assert _attend(cq, bad, size=True) == 0


def test_append_refuses(cq):
    for name in ("k", "v", "starts"):
        assert _append(cq, **{name: None}) == INVALID
    assert _append(cq, dtype=2) == INVALID
    assert _append(cq, n=-1) == SHAPE
    assert _append(cq, longest=-1) == SHAPE
    assert _append(cq, ldk=-8) == SHAPE
    assert _append(cq, n=(1 << 24) + 1) == UNSUPPORTED
    assert _append(cq, k=FAKE + 8) == ALIGN
    assert _append(cq, ldv=130) == ALIGN
    assert _append(cq, hsk=66, dtype=1) == ALIGN
    assert _append(cq, starts=FAKE + 2) == ALIGN
    assert _append(cq, n=0) == 0 and _append(cq, longest=0) == 0 and _append(cq, {"sequences": 0}) == 0


def test_values_refuse(cq):
    for name in ("begin", "starts"):
        assert _values(cq, **{name: None}) == INVALID
        assert _values(cq, **{name: FAKE + 2}) == ALIGN
    assert _values(cq, k=None, v=None) == INVALID
    assert _values(cq, dtype=2) == INVALID
    assert _values(cq, n=-1) == SHAPE
    assert _values(cq, n=(1 << 24) + 1) == UNSUPPORTED
    assert _values(cq, k=FAKE + 8) == ALIGN
    assert _values(cq, n=0) == 0 and _values(cq, {"sequences": 0}) == 0


def test_attention_refuses(cq):
    for name in ("q", "out", "starts"):
        assert _attend(cq, **{name: None}) == INVALID
    assert _attend(cq, dtype=2) == INVALID
    for bad in (dict(n=-1), dict(longest=-1), dict(heads_q=0), dict(heads_q=3), dict(window=-1), dict(softcap=-1.0), dict(softcap=float("nan")), dict(ldq=-4),
                dict(ldo=252), dict(hso=60)):
        assert _attend(cq, **bad) == SHAPE, bad
    assert _attend(cq, n=(1 << 24) + 1) == UNSUPPORTED
    assert _attend(cq, heads_q=4098, ldo=1 << 20) == UNSUPPORTED
    assert _attend(cq, heads_q=4096, n=1 << 20, ldo=1 << 20) == UNSUPPORTED
    for bad in (dict(q=FAKE + 8), dict(out=FAR + 8), dict(ldq=258), dict(hso=66), dict(starts=FAKE + 2), dict(lse=FAKE + 2), dict(ldq=260, dtype=1)):
        assert _attend(cq, **bad) == ALIGN, bad
    assert _attend(cq, out=FAKE) == INVALID and _attend(cq, out=FAKE + 512) == INVALID
    assert _attend(cq, ws=FAKE + 4) == ALIGN
    assert _attend(cq, n=0) == 0 and _attend(cq, longest=0) == 0 and _attend(cq, {"sequences": 0}) == 0
    assert cq.lib.cafeq_cache_attend(ctypes.byref(_cache(cq)), None, None, None) == INVALID


def test_page_calls_refuse(cq):
    c = ctypes.byref(_cache(cq))
    lib = cq.lib
    assert lib.cafeq_cache_reserve(c, None, 1, FAKE, FAKE, FAKE, None) == INVALID
    assert lib.cafeq_cache_reserve(c, FAKE, 1, FAKE, None, FAKE, None) == INVALID
    assert lib.cafeq_cache_reserve(c, FAKE, -1, FAKE, FAKE, FAKE, None) == SHAPE
    assert lib.cafeq_cache_reserve(c, FAKE, (1 << 24) + 1, FAKE, FAKE, FAKE, None) == UNSUPPORTED
    assert lib.cafeq_cache_reserve(c, FAKE + 2, 1, FAKE, FAKE, FAKE, None) == ALIGN
    assert lib.cafeq_cache_reserve(c, FAKE, 1, FAKE, FAKE, None, None) == WORKSPACE
    assert lib.cafeq_cache_reserve(c, FAKE, 1, FAKE, FAKE, FAKE + 8, None) == ALIGN
    assert lib.cafeq_cache_reorder(c, None, FAKE, None) == INVALID
    assert lib.cafeq_cache_reorder(c, FAKE + 1, FAKE, None) == ALIGN
    assert lib.cafeq_cache_reorder(c, FAKE, None, None) == WORKSPACE
    assert lib.cafeq_cache_reorder(ctypes.byref(_cache(cq, sequences=0)), FAKE, FAKE, None) == 0
    assert lib.cafeq_cache_compact(c, None, FAKE, None) == INVALID
    assert lib.cafeq_cache_compact(c, FAKE + 2, FAKE, None) == ALIGN
    assert lib.cafeq_cache_compact(c, FAKE, None, None) == WORKSPACE
    for call in (lambda x: lib.cafeq_cache_reserve(x, FAKE, 1, FAKE, FAKE, FAKE, None), lambda x: lib.cafeq_cache_reorder(x, FAKE, FAKE, None),
                 lambda x: lib.cafeq_cache_compact(x, FAKE, FAKE, None)):
        assert call(ctypes.byref(_cache(cq, refs=None))) == INVALID
    assert lib.cafeq_cache_pages_workspace_bytes(c) >= 4 * (3 * 10 + 3 * 4 + 4 * 3)


def test_slices_of_one_buffer_are_apart(cq):
    """What counts as shared memory: rows of one leading dimension by their columns, heads behind each other by theirs."""
    # q and the result in turn within each row of 512 floats
    assert _attend(cq, out=FAKE + 256 * 4, ldq=512, ldo=512, n=0) == 0
    ok = [dict(out=FAKE + 256 * 4, ldq=512, ldo=512), dict(q=FAKE + 256 * 4, out=FAKE, ldq=512, ldo=512)]
    for f in ok:
        assert _attend(cq, longest=0, **f) == 0
    for off in (252, 260, 300, 508):
        assert _attend(cq, longest=0, out=FAKE + off * 4, ldq=512, ldo=512) == INVALID
    # heads 1024 floats apart, tokens 64 apart in each: 2 tokens are 128 floats
    assert _attend(cq, longest=0, ldq=64, hsq=1024, out=FAKE + 128 * 4, ldo=64, hso=1024) == 0
    assert _attend(cq, longest=0, ldq=64, hsq=1024, out=FAKE + 64 * 4, ldo=64, hso=1024) == INVALID
