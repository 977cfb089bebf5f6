"""Refusals of the layer and of its epilogue's gradient (CPU): every call below must be rejected before a launch."""
import ctypes

import pytest

import paper_2110_15032_amd as sbp
from test_list_abi import ALIAS, ALIGN, AXIS, DTYPE, K, NULL, SHAPE, SIGNATURE, UNSUPPORTED, Room, T, status

M, KK, N = 64, 128, 256


def layer(x=None, sx=sbp.B, w=None, sw=sbp.S(1), bias="", residual="", pre="", y=None, sy=sbp.AUTO, k=2, epi=sbp.EPI_GELU):
    bias = T(2, N, 1, sbp.F32, 3) if bias == "" else bias
    residual, pre = T(2, M, N, sbp.F32, 4) if residual == "" else residual, T(2, M, N, sbp.BF16, 5) if pre == "" else pre
    args = (x or T(2, M, KK), sx, w or T(2, KK, N, at=1, trans=1), sw, bias, residual, pre, y or T(2, M, N, at=2), sy, k)
    with pytest.raises(sbp.SbpError) as e:
        sbp.sbp_linear(*args, 0, epi)
    return e.value.status


def test_layer_refusals():
    assert layer(k=0) == K and layer(sx=9) == AXIS and layer(sy=9) == AXIS and layer(sy=sbp.B) == SIGNATURE and layer(sx=sbp.S(0)) == SIGNATURE
    assert layer(sx=sbp.S(1), sw=sbp.S(0)) == SIGNATURE and layer(sx=sbp.P_SUM, sw=sbp.B) == SIGNATURE        # partial results
    assert layer(x=T(2, M, KK, sbp.F32)) == DTYPE and layer(x=T(2, M, KK, sbp.F8E4M3)) == DTYPE and layer(y=T(2, M, N, sbp.F8E4M3, 2)) == DTYPE
    assert layer(x=T(2, M, KK + 1)) == SHAPE and layer(y=T(2, M, N - 1, at=2)) == SHAPE and layer(residual=T(2, M, N + 1, sbp.F32, 4)) == SHAPE and layer(pre=T(2, M + 1, N, at=5)) == SHAPE
    assert layer(bias=T(2, N + 1, 1, sbp.F32, 3)) == SHAPE and layer(bias=T(2, 1, N, sbp.F32, 3)) == SHAPE and layer(bias=T(2, N, 1, sbp.I32, 3)) == DTYPE
    assert layer(residual=T(2, M, N, sbp.F8E4M3, 4)) == DTYPE
    assert layer(y=T(2, M, N, at=2, trans=1)) == UNSUPPORTED and layer(residual=T(2, M, N, sbp.F32, 4, trans=1)) == UNSUPPORTED and layer(pre=T(2, M, N, at=5, trans=1)) == UNSUPPORTED
    assert layer(epi=2) == UNSUPPORTED and layer(x=T(2, 2 ** 31 - 200, KK)) == UNSUPPORTED
    assert layer(y=T(2, M, N, at=0)) == ALIAS and layer(y=T(2, M, N, sbp.F32, 4)) == ALIAS and layer(pre=T(2, M, N, at=2)) == ALIAS and layer(pre=T(2, M, N, at=3)) == ALIAS
    assert layer(w=sbp.SbpTensor([0x200000004, 0x300000000], KK, N, sbp.BF16)) == ALIGN and layer(residual=T(2, M, N, sbp.F32, 4, ld=100)) == SHAPE
    same = sbp.SbpTensor([0x300000000] * 2, M, N, sbp.BF16)
    assert layer(sw=sbp.B, y=same) == ALIAS                                                        # a B result is two buffers
    with pytest.raises(ValueError):
        layer(bias=T(1, N, 1, sbp.F32, 3))
    L = sbp.lib()
    assert L.sbp_linear(None, sbp.B, T(1, 8, 8).ref(), sbp.B, None, None, None, T(1, 8, 8, at=1).ref(), sbp.B, 1, None, 0) == NULL


def grad(dy=None, s=sbp.S(1), pre="", ps=None, da="", db=None, room=Room(at=0x9000000000), k=2, epi=sbp.EPI_GELU):
    pre, da = T(2, M, N, at=1) if pre == "" else pre, T(2, M, N, at=2) if da == "" else da
    with pytest.raises(sbp.SbpError) as e:
        sbp.sbp_linear_grad(dy or T(2, M, N), s, pre, ps, da, db or T(2, N, 1, sbp.F32, 3), room, k, 0, epi)
    return e.value.status


def test_gradient_refusals():
    assert grad(k=0) == K and grad(s=sbp.P_SUM) == SIGNATURE and grad(s=6) == AXIS and grad(epi=5) == UNSUPPORTED
    assert grad(pre=None) == NULL and grad(da=None) == NULL and grad(pre=T(2, M, N, sbp.F8E4M3, 1)) == NULL
    assert grad(epi=sbp.EPI_NONE) == UNSUPPORTED and grad(epi=sbp.EPI_NONE, pre=None) == UNSUPPORTED
    assert grad(da=T(2, M, N, sbp.F32, 2)) == DTYPE and grad(dy=T(2, M, N, sbp.F8E4M3)) == DTYPE and grad(db=T(2, N, 1, sbp.BF16, 3)) == DTYPE
    assert grad(pre=T(2, M, N + 2, at=1)) == SHAPE and grad(da=T(2, M + 1, N, at=2)) == SHAPE and grad(db=T(2, N + 2, 1, sbp.F32, 3)) == SHAPE
    assert grad(dy=T(2, M, N, trans=1)) == UNSUPPORTED and grad(pre=T(2, M, N, at=1, trans=1)) == UNSUPPORTED
    assert grad(da=T(2, M, N, at=1)) == ALIAS and grad(db=T(2, N, 1, sbp.F32, 2)) == ALIAS
    assert grad(room=None) == NULL and grad(room=Room(size=16)) == SHAPE and grad(room=Room(at=0x9000000008)) == ALIGN and grad(room=Room(at=0x200000000)) == ALIAS
    assert grad(ps=sbp.SbpScales([0x9900000000, 0x9A00000000])) == DTYPE


def test_workspace():
    L, out = sbp.lib(), ctypes.c_int64()
    assert L.sbp_linear_grad_workspace(8, 8, sbp.B, 1, None) == NULL and L.sbp_linear_grad_workspace(8, 8, sbp.B, 0, ctypes.byref(out)) == K
    assert L.sbp_linear_grad_workspace(8, -8, sbp.B, 1, ctypes.byref(out)) == SHAPE and L.sbp_linear_grad_workspace(8, 8, sbp.P_SUM, 1, ctypes.byref(out)) == SIGNATURE
    assert sbp.sbp_linear_grad_workspace(32, 1000, sbp.B, 1) == 0                                   # one workgroup sums 32 rows
    assert sbp.sbp_linear_grad_workspace(33, 1001, sbp.B, 1) == (2 * 1001 * 4 + 15) // 16 * 16
