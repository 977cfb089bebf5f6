"""Refusals of the norms behind and in front of a block (CPU): every call below must be rejected before a launch."""
import ctypes

import pytest

import paper_2110_15032_amd as sbp
from test_list_abi import ALIAS, ALIGN, AXIS, DTYPE, K, NULL, SHAPE, SIGNATURE, UNSUPPORTED, Room, T, status

R, C = 64, 256


def V(n, at, dtype=sbp.F32, k=2):
    return T(k, n, 1, dtype, at)


def norm(kind=sbp.NORM_LAYER, eps=1e-5, at=20, stats=True, grads=False, dtype=sbp.F32, k=2, **over):
    layer = kind == sbp.NORM_LAYER
    f = dict(gamma=V(C, at, dtype, k), beta=V(C, at + 1, dtype, k) if layer else None, mean=V(R, at + 2, k=k) if layer and stats else None, rstd=V(R, at + 3, k=k) if stats else None,
             dgamma=V(C, at + 4, k=k) if grads else None, dbeta=V(C, at + 5, k=k) if grads and layer else None)
    f.update(over)
    return sbp.SbpNorm(kind, eps, **f)


def forward(x=None, sx=sbp.S(0), post="", gate="", r=None, h=None, pre="", y="", ys=None, k=2):
    post, pre = norm() if post == "" else post, norm(at=30) if pre == "" else pre
    gate, y = V(C, 9) if gate == "" else gate, T(2, R, C, sbp.BF16, 3) if y == "" else y
    return status(sbp.sbp_residual_norm, x or T(2, R, C), sx, post, gate, r or T(2, R, C, sbp.F32, 1), 1.0, h or T(2, R, C, sbp.F32, 2), pre, y, ys, k)


def test_forward_refusals():
    assert forward(k=0) == K and forward(sx=sbp.P_SUM) == SIGNATURE and forward(sx=9) == AXIS and forward(sx=sbp.S(1)) == UNSUPPORTED
    assert forward(x=T(2, R, C, sbp.F8E4M3)) == DTYPE and forward(r=T(2, R, C, sbp.BF16, 1)) == DTYPE and forward(x=T(2, R, C, sbp.I32)) == DTYPE
    assert forward(r=T(2, R, C + 1, sbp.F32, 1)) == SHAPE and forward(h=T(2, R + 1, C, sbp.F32, 2)) == SHAPE and forward(y=T(2, R, C + 8, sbp.BF16, 3)) == SHAPE
    assert forward(x=T(2, R, C, trans=1)) == UNSUPPORTED and forward(h=T(2, R, C, sbp.F32, 2, trans=1)) == UNSUPPORTED
    assert forward(y=T(2, R, C, sbp.F8E4M3, 3)) == NULL and forward(ys=sbp.SbpScales([0x9900000000, 0x9A00000000])) == DTYPE
    assert forward(y=None) == NULL and forward(pre=None) == NULL
    assert forward(gate=V(C - 1, 9)) == SHAPE and forward(gate=V(C, 9, sbp.BF16)) == DTYPE and forward(post=norm(dtype=sbp.BF16)) == DTYPE
    assert forward(post=norm(kind=2)) == UNSUPPORTED and forward(post=norm(eps=-1.0)) == UNSUPPORTED and forward(pre=norm(eps=float("nan"), at=30)) == UNSUPPORTED
    assert forward(post=norm(sbp.NORM_RMS, beta=V(C, 21))) == UNSUPPORTED and forward(post=norm(sbp.NORM_RMS, mean=V(R, 22))) == UNSUPPORTED
    assert forward(post=norm(mean=None)) == NULL and forward(post=norm(rstd=None)) == NULL and forward(post=norm(rstd=V(R + 1, 23))) == SHAPE
    assert forward(post=norm(rstd=V(R, 23, sbp.BF16))) == DTYPE
    assert forward(h=T(2, R, C, sbp.F32, 1)) == ALIAS and forward(y=T(2, R, C, sbp.BF16, 2)) == ALIAS and forward(pre=norm(at=20)) == ALIAS
    assert forward(pre=norm(at=30, rstd=V(R, 3))) == ALIAS
    assert forward(x=sbp.SbpTensor([0x100000008, 0x200000000], R, C, sbp.BF16)) == ALIGN and forward(x=T(2, R, C, ld=255)) == SHAPE
    wide = 16392
    assert status(sbp.sbp_residual_norm, T(1, 8, wide), sbp.B, None, None, T(1, 8, wide, at=1), 1.0, T(1, 8, wide, at=2), None, None, None, 1) == UNSUPPORTED
    assert status(sbp.sbp_residual_norm, T(33, 64, 8), sbp.S(0), None, None, T(33, 64, 8, at=1), 1.0, T(33, 64, 8, at=2), None, None, None, 33) == UNSUPPORTED
    none = sbp.SbpNorm(sbp.NORM_RMS, 1e-5, rstd=T(1, 8, 1, sbp.F32, 4))
    assert status(sbp.sbp_residual_norm, T(1, 8, 0), sbp.B, none, None, T(1, 8, 0, at=1), 1.0, T(1, 8, 0, at=2), None, None, None, 1) == SHAPE
    with pytest.raises(ValueError):
        forward(post=norm(k=1))


def grad(x=None, sx=sbp.S(0), post="", gate="", h="", pre="", dh="", dy="", dx=None, dr=None, dgate="", room=Room(at=0x9000000000, size=1 << 24), k=2):
    post, pre = norm(grads=True) if post == "" else post, norm(at=30, grads=True) if pre == "" else pre
    gate, dgate = V(C, 9) if gate == "" else gate, V(C, 10) if dgate == "" else dgate
    h, dh, dy = T(2, R, C, sbp.F32, 1) if h == "" else h, T(2, R, C, sbp.F32, 2) if dh == "" else dh, T(2, R, C, sbp.BF16, 3) if dy == "" else dy
    return status(sbp.sbp_residual_norm_grad, x or T(2, R, C), sx, post, gate, 1.0, h, pre, dh, dy, dx or T(2, R, C, sbp.BF16, 4), dr or T(2, R, C, sbp.F32, 5), dgate, room, k)


def test_gradient_refusals():
    assert grad(k=0) == K and grad(sx=sbp.P_SUM) == SIGNATURE and grad(sx=sbp.S(1)) == UNSUPPORTED
    assert grad(h=None) == NULL and grad(dy=None) == NULL and grad(pre=None) == NULL
    assert grad(pre=None, h=None, dy=None, dh=None) == NULL                                   # no gradient comes in
    assert grad(dx=T(2, R, C, sbp.F32, 4)) == DTYPE and grad(dr=T(2, R, C, sbp.BF16, 5)) == DTYPE and grad(dh=T(2, R, C, sbp.BF16, 2)) == DTYPE
    assert grad(dy=T(2, R, C, sbp.F8E4M3, 3)) == DTYPE
    assert grad(dy=T(2, R, C - 1, sbp.BF16, 3)) == SHAPE and grad(dgate=V(C + 1, 10)) == SHAPE and grad(dgate=V(C, 10, sbp.BF16)) == DTYPE
    assert grad(post=norm(mean=None)) == NULL and grad(post=norm(rstd=None)) == NULL and grad(post=norm(sbp.NORM_RMS, rstd=None)) == NULL
    assert grad(post=norm(sbp.NORM_RMS, dbeta=V(C, 25))) == UNSUPPORTED and grad(dy=T(2, R, C, sbp.BF16, 3, trans=1)) == UNSUPPORTED
    assert grad(room=None) == NULL and grad(room=Room(at=0x9000000000, size=16)) == SHAPE and grad(room=Room(at=0x9000000008, size=1 << 24)) == ALIGN
    assert grad(room=Room(at=0x100000000, size=1 << 24)) == ALIAS
    assert grad(dr=T(2, R, C, sbp.F32, 2)) == ALIAS and grad(dx=T(2, R, C, sbp.BF16, 0)) == ALIAS and grad(dgate=V(C, 9)) == ALIAS and grad(dgate=V(C, 24)) == ALIAS


def test_workspace():
    L, out = sbp.lib(), ctypes.c_int64()
    assert L.sbp_residual_norm_grad_workspace(8, 8, sbp.B, 1, None) == NULL
    assert L.sbp_residual_norm_grad_workspace(-1, 8, sbp.B, 1, ctypes.byref(out)) == SHAPE
    assert L.sbp_residual_norm_grad_workspace(8, 16385, sbp.B, 1, ctypes.byref(out)) == UNSUPPORTED
    assert L.sbp_residual_norm_grad_workspace(2 ** 31, 8, sbp.B, 1, ctypes.byref(out)) == UNSUPPORTED
    assert sbp.sbp_residual_norm_grad_workspace(1, 100, sbp.B, 1) == 4 * 100 * 4
    assert sbp.sbp_residual_norm_grad_workspace(0, 100, sbp.S(0), 2) == 2 * 4 * 100 * 4


def test_most_devices_fit_the_check():
    """32 devices with every tensor there is: refused for the last pair alone"""
    k, at = 32, lambda i: 0x100000000 * (64 * i + 1)  # noqa: E731

    def t(rows, cols, dtype, i):
        return sbp.SbpTensor([at(i) + j * 0x1000000 for j in range(k)], rows, cols, dtype)
    n = [sbp.SbpNorm(sbp.NORM_LAYER, 1e-5, t(C, 1, 0, i), t(C, 1, 0, i + 1), t(R, 1, 0, i + 2), t(R, 1, 0, i + 3), t(C, 1, 0, i + 4), t(C, 1, 0, i + 5)) for i in (20, 30)]
    assert status(sbp.sbp_residual_norm_grad, t(R, C, 0, 0), sbp.S(0), n[0], t(C, 1, 0, 1), 1.0, t(R, C, 0, 2), n[1], t(R, C, 0, 3), t(R, C, 0, 4), t(R, C, 0, 5), t(R, C, 0, 6),
                  t(C, 1, 0, 25), Room(at=at(40), size=1 << 24), k) == ALIAS
