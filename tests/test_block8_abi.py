"""Refusals of the operators on 8-bit tensors and of layer normalisation (CPU): every call below must be rejected before a launch."""
import pytest

import paper_2110_15032_amd as sbp

NULL, K, SHAPE, DTYPE, AXIS, SIGNATURE, ALIAS, ALIGN, UNSUPPORTED = -1, -2, -3, -4, -5, -6, -7, -8, -9
STREAM = 0


def T(k, rows, cols, dtype=sbp.BF16, at=0, trans=0, ld=0):
    """descriptor over made-up addresses, never dereferenced; `at`: buffers of another number lie elsewhere"""
    return sbp.SbpTensor([0x100000000 * (at + 1) + i * 0x1000000 for i in range(k)], rows, cols, dtype, trans, ld)


def SC(k, at=0, ld=0):
    return sbp.SbpScales([0x100000000 * (at + 1) + i * 0x1000000 for i in range(k)], ld)


def status(fn, *a, **kw):
    with pytest.raises(sbp.SbpError) as e:
        fn(*a, **kw)
    return e.value.status


def quantize(x=None, sx=sbp.S(0), q=None, s=None, k=2, epi=sbp.EPI_NONE):
    return status(sbp.sbp_quantize, x or T(2, 64, 256), sx, q or T(2, 64, 256, sbp.F8E4M3, 1), s or SC(2, 2), k, STREAM, epi)


def test_quantize_refusals():
    assert quantize(k=0) == K and quantize(x=T(65, 8, 8), q=T(65, 8, 8, sbp.F8E4M3, 1), s=SC(65, 2), k=65) == K
    assert quantize(sx=sbp.P_SUM) == SIGNATURE and quantize(sx=2) == AXIS
    assert quantize(q=T(2, 64, 256, sbp.BF16, 1)) == DTYPE and quantize(x=T(2, 64, 256, sbp.F8E4M3)) == DTYPE
    assert quantize(x=T(2, 64, 256, sbp.I32)) == DTYPE
    assert quantize(q=T(2, 64, 255, sbp.F8E4M3, 1)) == SHAPE
    assert quantize(x=T(2, 64, 256, trans=1)) == UNSUPPORTED
    assert quantize(epi=7) == UNSUPPORTED
    assert quantize(x=T(2, 64, 256, ld=255)) == SHAPE
    assert quantize(s=SC(2, 2, ld=1)) == SHAPE                                   # two blocks a row
    assert quantize(q=T(2, 64, 256, sbp.F8E4M3, 1, trans=1, ld=31)) == SHAPE     # 32 local rows a stored row
    assert quantize(q=T(2, 64, 256, sbp.F8E4M3, 0)) == ALIAS and quantize(s=SC(2, 1)) == ALIAS and quantize(s=SC(2, 0)) == ALIAS
    assert quantize(s=sbp.SbpScales([0x300000008, 0x310000000])) == ALIGN
    assert quantize(s=sbp.SbpScales([None, 0x310000000])) == NULL
    assert quantize(x=sbp.SbpTensor([0x100000002, 0x200000000], 64, 256, sbp.BF16)) == ALIGN
    assert status(sbp.sbp_quantize, T(2, 64, 256), sbp.B, T(2, 64, 256, sbp.F8E4M3, 1), None, 2, STREAM) == NULL
    # a B output is k distinct buffers
    same = sbp.SbpTensor([0x300000000] * 2, 64, 256, sbp.F8E4M3)
    assert quantize(sx=sbp.B, q=same, s=SC(2, 4)) == ALIAS
    assert quantize(x=T(2, 2 ** 31, 8), q=T(2, 2 ** 31, 8, sbp.F8E4M3, 1)) == UNSUPPORTED
    for rows, cols in ((2 ** 31 - 1, 8), (8, 2 ** 31 - 1), (8, 2 ** 31 - 256)):      # the last tile's end would not be a 32-bit number
        assert quantize(x=T(2, rows, cols), q=T(2, rows, cols, sbp.F8E4M3, 1)) == UNSUPPORTED
    with pytest.raises(ValueError):
        sbp.sbp_quantize(T(1, 64, 256), sbp.S(0), T(2, 64, 256, sbp.F8E4M3, 1), SC(2, 2), 2, STREAM)


def test_dequantize_refusals():
    def call(q=None, s=None, sq=sbp.S(1), x=None, k=2, epi=sbp.EPI_NONE):
        return status(sbp.sbp_dequantize, q or T(2, 64, 256, sbp.F8E5M2), s or SC(2, 2), sq, x or T(2, 64, 256, sbp.F32, 1), k, STREAM, epi)
    assert call(k=-1) == K and call(sq=sbp.P_MAX) == SIGNATURE and call(sq=7) == AXIS
    assert call(q=T(2, 64, 256)) == DTYPE and call(x=T(2, 64, 256, sbp.F8E4M3, 1)) == DTYPE
    assert call(x=T(2, 64, 256, at=1, trans=1)) == UNSUPPORTED and call(x=T(2, 65, 256, at=1)) == SHAPE
    assert call(x=T(2, 64, 256, at=0)) == ALIAS and call(x=T(2, 64, 256, at=2)) == ALIAS
    assert call(epi=2) == UNSUPPORTED


def test_gelu_grad_refusals():
    def call(a=None, s=None, sa=sbp.S(1), dh=None, da=None, k=2):
        return status(sbp.sbp_gelu_grad, a or T(2, 64, 256), s, sa, dh or T(2, 64, 256, at=1), da or T(2, 64, 256, at=2), k, STREAM)
    assert call(sa=sbp.P_SUM) == SIGNATURE and call(k=0) == K
    assert call(s=SC(2, 3)) == DTYPE                                             # scales next to values that need none
    assert call(a=T(2, 64, 256, sbp.F8E4M3)) == NULL                             # and none next to values that do
    assert call(da=T(2, 64, 256, sbp.F32, 2)) == DTYPE
    assert call(dh=T(2, 64, 256, sbp.F8E4M3, 1), s=SC(2, 3)) == DTYPE
    assert call(da=T(2, 64, 256, at=1)) == ALIAS and call(da=T(2, 64, 256, at=0)) == ALIAS
    assert call(a=T(2, 64, 256, trans=1)) == UNSUPPORTED and call(dh=T(2, 32, 256, at=1)) == SHAPE


def test_layernorm_refusals():
    def call(x=None, sx=sbp.S(0), g=None, b=None, eps=1e-5, y=None, ys=None, mean=None, rstd=None, k=2):
        return status(sbp.sbp_layernorm, x or T(2, 64, 256), sx, g, b, eps, y or T(2, 64, 256, at=1), ys, mean, rstd, k, STREAM)
    assert call(sx=sbp.S(1)) == UNSUPPORTED and call(sx=sbp.P_SUM) == SIGNATURE and call(sx=9) == AXIS and call(k=0) == K
    assert call(x=T(33, 64, 256), y=T(33, 64, 256, at=1), k=33) == UNSUPPORTED
    assert call(x=T(2, 64, 16385), y=T(2, 64, 16385, at=1)) == UNSUPPORTED
    assert call(eps=-1.0) == UNSUPPORTED and call(eps=float("nan")) == UNSUPPORTED
    assert call(y=T(2, 64, 256, sbp.F8E4M3, 1)) == NULL and call(ys=SC(2, 4)) == DTYPE
    assert call(x=T(2, 64, 256, sbp.F8E4M3)) == DTYPE
    assert call(g=T(2, 255, 1, at=3)) == SHAPE and call(b=T(2, 256, 1, sbp.I32, 3)) == DTYPE
    assert call(g=T(2, 256, 1, at=3), b=T(2, 256, 1, sbp.F32, 4)) == DTYPE
    m, r = T(2, 64, 1, sbp.F32, 5), T(2, 64, 1, sbp.F32, 6)
    assert call(mean=m) == NULL and call(rstd=r) == NULL
    assert call(mean=m, rstd=T(2, 64, 1, sbp.F32, 5)) == ALIAS
    assert call(mean=T(2, 64, 1, sbp.BF16, 5), rstd=r) == DTYPE
    assert call(y=T(2, 64, 256, at=0)) == ALIAS and call(y=T(2, 64, 256, at=1, trans=1)) == UNSUPPORTED


def test_layernorm_grad_refusals():
    def call(x=None, xs=None, sx=sbp.S(0), g=None, mean=None, rstd=None, dy=None, dx=None, dg=None, db=None, room=None, k=2, rows=4096):
        return status(sbp.sbp_layernorm_grad, x or T(2, rows, 256), xs, sx, g, mean or T(2, rows, 1, sbp.F32, 1), rstd or T(2, rows, 1, sbp.F32, 2),
                      dy or T(2, rows, 256, at=3), dx or T(2, rows, 256, at=4), dg, db, room, k, STREAM)
    dg, db = T(2, 256, 1, sbp.F32, 5), T(2, 256, 1, sbp.F32, 6)
    assert call(sx=sbp.S(1)) == UNSUPPORTED and call(sx=sbp.P_SUM) == SIGNATURE
    assert call(dg=dg) == NULL and call(db=db) == NULL
    assert call(dg=dg, db=db) == NULL                                            # no workspace
    class Room:
        def __init__(self, n, at=0x900000000): self.n, self.at = n, at           # noqa: E704
        def numel(self): return self.n                                           # noqa: E704
        def element_size(self): return 1                                         # noqa: E704
        def data_ptr(self): return self.at                                       # noqa: E704
    need = sbp.sbp_layernorm_grad_workspace(4096, 256, sbp.S(0), 2)
    assert need > 0
    assert call(dg=dg, db=db, room=Room(need - 1)) == SHAPE
    assert call(dg=dg, db=db, room=Room(need, 0x900000004)) == ALIGN
    assert call(dg=dg, db=db, room=Room(need, 0x100000000)) == ALIAS
    assert call(dg=dg, db=T(2, 256, 1, sbp.F32, 5), room=Room(need)) == ALIAS
    assert call(dx=T(2, 4096, 256, sbp.F32, 4)) == DTYPE and call(x=T(2, 4096, 256, sbp.F8E4M3)) == NULL
    assert call(mean=T(2, 4095, 1, sbp.F32, 1)) == SHAPE
    assert sbp.sbp_layernorm_grad_workspace(1, 256, sbp.B, 1) == 0
    assert status(sbp.sbp_layernorm_grad_workspace, 8, 16385, sbp.S(0), 2) == UNSUPPORTED
    assert status(sbp.sbp_layernorm_grad_workspace, -1, 8, sbp.S(0), 2) == SHAPE


def test_matmul_f8_refusals():
    def call(x=None, xs=None, sx=sbp.B, w=None, ws=None, sw=sbp.S(1), y=None, sy=sbp.AUTO, k=2, epi=sbp.EPI_NONE):
        return status(sbp.sbp_matmul_f8, x or T(2, 64, 256, sbp.F8E4M3), xs or SC(2, 1), sx, w or T(2, 256, 96, sbp.F8E4M3, 2, trans=1), ws or SC(2, 3), sw,
                      y or T(2, 64, 96, sbp.BF16, 4), sy, k, STREAM, epi)
    assert call(k=0) == K and call(sx=sbp.S(0)) == SIGNATURE and call(sy=sbp.B) == SIGNATURE and call(sx=5) == AXIS
    assert call(sx=sbp.P_SUM, sw=sbp.B) == DTYPE
    assert call(x=T(2, 64, 256)) == DTYPE and call(w=T(2, 256, 96, sbp.F32, 2, trans=1)) == DTYPE
    assert call(w=T(2, 256, 96, sbp.F8E4M3, 2)) == UNSUPPORTED and call(x=T(2, 64, 256, sbp.F8E4M3, trans=1)) == UNSUPPORTED
    assert call(w=T(2, 255, 96, sbp.F8E4M3, 2, trans=1)) == SHAPE and call(y=T(2, 64, 97, at=4)) == SHAPE
    assert call(sx=sbp.S(1), sw=sbp.S(0)) == DTYPE                               # a P(sum) result is fp32
    f = T(2, 64, 96, sbp.F32, 4)
    assert call(sx=sbp.S(1), sw=sbp.S(0), y=f, epi=sbp.EPI_GELU) == SIGNATURE and call(epi=9) == UNSUPPORTED
    assert call(y=T(2, 64, 96, at=0)) == ALIAS and call(y=T(2, 64, 96, at=3)) == ALIAS
    assert call(xs=SC(2, 1, ld=1)) == SHAPE
    k = 33
    assert call(x=T(k, 64, 256, sbp.F8E4M3), xs=SC(k, 1), w=T(k, 256, 96, sbp.F8E4M3, 2, trans=1), ws=SC(k, 3), y=T(k, 64, 96, at=4), k=k) == UNSUPPORTED


def test_empty_tensors_are_fine():
    none = sbp.SbpTensor([None] * 2, 0, 256, sbp.BF16)
    none8 = sbp.SbpTensor([None] * 2, 0, 256, sbp.F8E4M3)
    s = sbp.SbpScales([None] * 2)
    sbp.sbp_quantize(none, sbp.S(0), none8, s, 2, STREAM)
    sbp.sbp_dequantize(none8, s, sbp.S(0), none, 2, STREAM)
    sbp.sbp_gelu_grad(none8, s, sbp.S(0), none, none, 2, STREAM)
    sbp.sbp_layernorm(none, sbp.S(0), None, None, 1e-5, none, None, None, None, 2, STREAM)
    sbp.sbp_matmul_f8(none8, s, sbp.S(0), T(2, 256, 96, sbp.F8E4M3, 2, trans=1), SC(2, 3), sbp.B, sbp.SbpTensor([None] * 2, 0, 96, sbp.BF16), sbp.AUTO, 2, STREAM)


def test_rows_without_elements_have_no_statistics():
    """the mean of nothing is not a number that a caller could go on with, and left unwritten it would be what the buffer held before"""
    x, y = T(2, 64, 0), T(2, 64, 0, at=1)
    m, r = T(2, 64, 1, sbp.F32, 5), T(2, 64, 1, sbp.F32, 6)
    assert status(sbp.sbp_layernorm, x, sbp.S(0), None, None, 1e-5, y, None, m, r, 2, STREAM) == SHAPE
    sbp.sbp_layernorm(x, sbp.S(0), None, None, 1e-5, y, None, None, None, 2, STREAM)
    none = sbp.SbpTensor([None] * 2, 0, 1, sbp.F32)
    sbp.sbp_layernorm(T(2, 0, 0), sbp.S(0), None, None, 1e-5, T(2, 0, 0, at=1), None, none, none, 2, STREAM)
