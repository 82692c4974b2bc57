"""Host-side checks of the serving entry points: what they refuse, before anything is launched (no GPU needed)."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2511_19705_amd", "libcafeq.so")
FAKE = 4096          # a non-null, aligned address that is never dereferenced on these paths
INVALID, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE = -1, -2, -3, -4, -7


@pytest.fixture(scope="module")
def cq():
    if not os.path.exists(LIB):
        import __graft_entry__ as ge
        ge.build()
    from paper_2511_19705_amd import cafeq
    return cafeq


def _norm(cq, n=2, d=64, group=32, codes=FAKE, scales=FAKE, values=None, vdtype=0, ldv=64, xf=None, ws=FAKE, **fields):
    a = cq.Activations(x=FAKE, ldx=d, ldr=d, lds=d, dtype=0, norm=1, eps=1e-6)
    for k, v in fields.items():
        setattr(a, k, v)
    return cq.lib.cafeq_norm_quantize(ctypes.byref(a), n, d, None if xf is None else ctypes.byref(xf), group, codes, scales, values, vdtype, ldv,
                                      ws, None)


def test_norm_refuses(cq):
    assert cq.lib.cafeq_norm_quantize(None, 1, 64, None, 32, FAKE, FAKE, None, 0, 64, None, None) == INVALID
    assert _norm(cq, x=None) == INVALID
    assert _norm(cq, dtype=2) == INVALID
    assert _norm(cq, codes=None) == INVALID              # scales without codes
    assert _norm(cq, codes=None, scales=None) == INVALID  # nothing to write
    assert _norm(cq, values=FAKE, vdtype=2) == INVALID
    assert _norm(cq, n=-1) == SHAPE
    assert _norm(cq, d=0) == SHAPE
    assert _norm(cq, ldx=63) == SHAPE
    assert _norm(cq, residual=FAKE, ldr=63) == SHAPE
    assert _norm(cq, sum=FAKE, lds=63) == SHAPE
    assert _norm(cq, values=FAKE, ldv=63) == SHAPE
    for group in (-1, 16, 48):
        assert _norm(cq, group=group) == SHAPE
    assert _norm(cq, d=65568, group=0, ldv=65568) == UNSUPPORTED
    assert _norm(cq, n=(1 << 21) + 1) == UNSUPPORTED
    assert _norm(cq, x=FAKE + 2) == ALIGN
    assert _norm(cq, gain=FAKE + 2) == ALIGN
    assert _norm(cq, scales=FAKE + 2) == ALIGN
    assert _norm(cq, n=0) == 0
    assert _norm(cq, sum=FAKE + 4) == INVALID            # neither x itself nor apart from it
    assert _norm(cq, sum=FAKE, lds=68) == INVALID
    assert _norm(cq, residual=FAKE + 65536, sum=FAKE + 65536 + 128) == INVALID
    assert _norm(cq, ldx=96, sum=FAKE + 96, lds=96) == INVALID   # columns that reach into x's


def test_norm_with_a_transform_refuses(cq):
    def xf(k=32, nb=2, rep=1, tinv=FAKE):
        return cq.Xform(None, tinv, k, nb, rep)

    assert _norm(cq, xf=xf(tinv=None)) == INVALID
    assert _norm(cq, xf=xf(k=16, nb=4)) == UNSUPPORTED
    assert _norm(cq, xf=xf(nb=3)) == SHAPE
    assert _norm(cq, xf=xf(rep=2)) == SHAPE
    assert _norm(cq, xf=xf(tinv=FAKE + 4)) == ALIGN
    assert _norm(cq, xf=xf(), x=FAKE + 4) == ALIGN
    assert _norm(cq, xf=xf(), ldx=65) == ALIGN
    assert _norm(cq, xf=xf(), codes=FAKE + 8) == ALIGN
    assert _norm(cq, xf=xf(), values=FAKE, ldv=65) == ALIGN
    assert _norm(cq, xf=xf(), n=100, ws=None) == WORKSPACE
    assert _norm(cq, xf=xf(), group=0, d=64, n=1, codes=FAKE, ws=FAKE + 8, ) in (ALIGN,)
    far = FAKE + (1 << 20)
    assert _norm(cq, xf=xf(), sum=FAKE) == INVALID                       # the sum over x, which is read again
    assert _norm(cq, xf=xf(), residual=far, sum=far + 256) == INVALID    # and over the residual
    assert _norm(cq, xf=xf(), n=0, sum=FAKE) == 0


def test_workspaces(cq):
    def need(n, d, k, group):
        x = cq.Xform(None, None, k, d // k, 1)
        return cq.lib.cafeq_norm_workspace_bytes(n, d, ctypes.byref(x), group)

    assert cq.lib.cafeq_norm_workspace_bytes(100, 64, None, 32) == 0     # nothing without a transform
    assert need(0, 64, 32, 32) == 0
    assert need(1, 4608, 128, 128) == 0                                  # a few rows' norms are formed on the way
    assert need(100, 4608, 128, 128) == 512
    assert need(100, 4608, 128, -1) == 512
    assert need(100, 4608, 128, 0) == 512 + 100 * 4608 * 4               # groups that no tile holds: z itself
    size = cq.lib.cafeq_infer_packed_workspace_bytes
    assert size(cq.I8, 1, 3584, 14336, 128) == 0
    assert size(cq.F32, 4096, 3584, 14336, 128) >= 4096 * 14336 * 6      # three bfloat16 planes of the activations
    assert size(cq.I8, 4096, 3584, 14300, 128) == 0                      # refused sizes
    assert size(3, 4096, 3584, 14336, 128) == 0


def test_packing_refuses(cq):
    lib = cq.lib
    assert lib.cafeq_packed_bytes(16, 64, 0) == 32 * 64 + 2 * 16 * 4     # rows rounded to 32, columns to 128
    for out, width, group in ((0, 64, 32), (16, 63, 0), (16, 16, 0), (16, 64, 48), (16, 64, 16), (16, 64, -32), (16, 65568, 0), (1 << 24, 65536, 0)):
        assert lib.cafeq_packed_bytes(out, width, group) == 0
    pack = lib.cafeq_pack_nibbles
    for args in ((None, FAKE, FAKE), (FAKE, None, FAKE), (FAKE, FAKE, None)):
        assert pack(args[0], args[1], 16, 64, 32, args[2], None) == INVALID
    assert pack(FAKE, FAKE, 16, 64, 48, FAKE, None) == SHAPE
    assert pack(FAKE, FAKE, 16, 65568, 0, FAKE, None) == UNSUPPORTED
    assert pack(FAKE, FAKE, 16, 64, 32, FAKE + 8, None) == ALIGN
    assert pack(FAKE, FAKE + 1, 16, 64, 32, FAKE, None) == ALIGN


def _infer(cq, X=FAKE, kind=0, n=2, ldx=64, xs=None, xgroup=0, packed=FAKE, out=16, width=64, group=32, Y=FAKE, ykind=0, ldy=16, ws=FAKE):
    return cq.lib.cafeq_infer_packed(X, kind, n, ldx, xs, xgroup, packed, out, width, group, Y, ykind, ldy, ws, None)


def test_product_refuses(cq):
    for k in ("X", "packed", "Y"):
        assert _infer(cq, **{k: None}) == INVALID
    assert _infer(cq, kind=3) == INVALID
    assert _infer(cq, ykind=2) == INVALID
    assert _infer(cq, kind=2) == INVALID                 # 8 bits without scales
    assert _infer(cq, xs=FAKE) == INVALID                # scales without 8 bits
    assert _infer(cq, n=-1) == SHAPE
    assert _infer(cq, ldx=60) == SHAPE
    assert _infer(cq, ldy=15) == SHAPE
    assert _infer(cq, group=48) == SHAPE
    for xgroup in (-32, 16, 48):
        assert _infer(cq, kind=2, xs=FAKE, xgroup=xgroup) == SHAPE
    assert _infer(cq, n=(1 << 19) + 1) == UNSUPPORTED
    assert _infer(cq, ldx=(1 << 24) + 16) == UNSUPPORTED
    assert _infer(cq, X=FAKE + 8) == ALIGN
    assert _infer(cq, ldx=65) == ALIGN
    assert _infer(cq, Y=FAKE + 2) == ALIGN
    assert _infer(cq, kind=2, xs=FAKE + 2) == ALIGN
    assert _infer(cq, packed=FAKE + 8) == ALIGN
    assert _infer(cq, kind=0, n=4096, out=3584, width=14336, group=128, ldx=14336, ldy=3584, ws=None) == WORKSPACE
    assert _infer(cq, kind=0, n=4096, out=3584, width=14336, group=128, ldx=14336, ldy=3584, ws=FAKE + 4) == ALIGN
    assert _infer(cq, n=0) == 0
