"""Refusals of the operators on lists of tensors (CPU): every call below must be rejected before a launch."""
import ctypes

import pytest

import paper_2110_15032_amd as sbp

NULL, K, SHAPE, DTYPE, AXIS, SIGNATURE, ALIAS, ALIGN, UNSUPPORTED = -1, -2, -3, -4, -5, -6, -7, -8, -9
STREAM = 0


def T(k, rows, cols, dtype=sbp.BF16, at=0, trans=0, ld=0):
    """descriptor over made-up addresses, never dereferenced; `at`: buffers of another number lie elsewhere"""
    return sbp.SbpTensor([0x100000000 * (at + 1) + i * 0x1000000 for i in range(k)], rows, cols, dtype, trans, ld)


def scalar(k, at):
    return T(k, 1, 1, sbp.F32, at)


class Room:
    """a workspace at a made-up address"""

    def __init__(self, at=0x7000000000, size=1 << 20):
        self.at, self.size = at, size

    def data_ptr(self):
        return self.at

    def numel(self):
        return self.size

    def element_size(self):
        return 1


def status(fn, *a):
    with pytest.raises(sbp.SbpError) as e:
        fn(*a, STREAM)
    return e.value.status


def squares(tensors=None, sigs=None, out=None, room=Room(), k=2):
    tensors = [T(2, 64, 256), T(2, 32, 8, sbp.F32, 1)] if tensors is None else tensors
    sigs = [sbp.S(0), sbp.B][:len(tensors)] if sigs is None else sigs
    return status(sbp.sbp_square_sum, sbp.SbpList(tensors, sigs), out or scalar(2, 9), room, k)


def test_square_sum_refusals():
    assert squares(k=0) == K and squares(tensors=[T(65, 8, 8)], out=scalar(65, 9), k=65) == K
    assert squares(sigs=[sbp.P_SUM, sbp.B]) == SIGNATURE and squares(sigs=[5, sbp.B]) == AXIS
    assert squares(tensors=[T(2, 64, 256, sbp.F8E4M3)]) == DTYPE and squares(tensors=[T(2, 64, 256, sbp.I32)]) == DTYPE
    assert squares(tensors=[T(2, 64, 256, ld=255)]) == SHAPE and squares(tensors=[T(2, -1, 256)]) == SHAPE
    assert squares(tensors=[T(2, 2 ** 31, 8)]) == UNSUPPORTED and squares(tensors=[T(2, 8, 2 ** 31)]) == UNSUPPORTED
    assert squares(tensors=[T(1, 2 ** 31 - 1, 2 ** 31 - 1)], out=scalar(1, 9), k=1) == UNSUPPORTED
    assert squares(tensors=[sbp.SbpTensor([0x100000008, 0x200000000], 64, 256, sbp.BF16)]) == ALIGN
    assert squares(tensors=[sbp.SbpTensor([None, 0x200000000], 64, 256, sbp.BF16)]) == NULL
    assert squares(out=T(2, 2, 1, sbp.F32, 9)) == SHAPE and squares(out=T(2, 1, 1, sbp.BF16, 9)) == DTYPE
    assert squares(out=scalar(2, 0)) == ALIAS                                                 # inside the first tensor
    assert squares(out=sbp.SbpTensor([0x900000000] * 2, 1, 1, sbp.F32)) == ALIAS             # every device has its own part
    assert squares(room=None) == NULL and squares(room=Room(size=8)) == SHAPE and squares(room=Room(at=0x7000000008)) == ALIGN
    assert squares(room=Room(at=0x100000000)) == ALIAS and squares(room=Room(at=0xA00000000)) == ALIAS
    assert status(sbp.sbp_square_sum, sbp.SbpList([T(2, 8, 8)], [sbp.B]), sbp.SbpTensor([0x900000000, 0x900000040], 1, 1, sbp.F32, 1), Room(), 2) == UNSUPPORTED
    with pytest.raises(ValueError):
        sbp.sbp_square_sum(sbp.SbpList([T(1, 8, 8)], [sbp.B]), scalar(2, 9), Room(), 2, STREAM)
    with pytest.raises(ValueError):
        sbp.SbpList([T(1, 8, 8)], [])


def test_more_tensors_than_a_list_takes():
    one = T(1, 1, 1, sbp.F32)
    lst = sbp.SbpList([one], [sbp.B])
    lst.n = (1 << 20) + 1                      # refused before any of them is looked at
    with pytest.raises(sbp.SbpError) as e:
        sbp.sbp_square_sum_workspace(lst, 1)
    assert e.value.status == UNSUPPORTED
    assert status(sbp.sbp_square_sum, lst, scalar(1, 5), Room(), 1) == UNSUPPORTED
    assert status(sbp.sbp_clip, lst, scalar(1, 5), sbp.B, 1.0, lst, None, 1) == UNSUPPORTED


def test_square_sum_raw_entries():
    L, out = sbp.lib(), ctypes.c_int64()
    s = (ctypes.c_int32 * 1)(sbp.B)
    assert L.sbp_square_sum_workspace(None, s, 1, 1, ctypes.byref(out)) == NULL
    assert L.sbp_square_sum_workspace(T(1, 8, 8).ref(), None, 1, 1, ctypes.byref(out)) == NULL
    assert L.sbp_square_sum_workspace(T(1, 8, 8).ref(), s, -1, 1, ctypes.byref(out)) == SHAPE
    assert L.sbp_square_sum_workspace(T(1, 8, 8).ref(), s, 1, 1, None) == NULL
    assert L.sbp_square_sum_workspace(None, None, 0, 1, ctypes.byref(out)) == 0 and out.value == 0
    assert L.sbp_square_sum(T(1, 8, 8).ref(), s, 1, None, 0x7000000000, 1 << 20, 1, None) == NULL


def test_workspace_counts_partial_sums():
    def room(tensors, sigs, k):
        return sbp.sbp_square_sum_workspace(sbp.SbpList(tensors, sigs), k)
    # launches of 160 tensors, of 80 with rows at a pitch, one more of each; workgroups of 8192 elements, at most 2048
    assert room([T(1, 1, 1)], [sbp.B], 1) == 4 * 8 and room([T(1, 0, 8)], [sbp.B], 1) == 0 and room([], [], 1) == 0
    assert room([T(1, 8, 1024)], [sbp.B], 1) == 4 * 8 and room([T(1, 8, 1025)], [sbp.B], 1) == 4 * 2 * 8
    assert room([T(8, 1 << 16, 1 << 14)], [sbp.S(0)], 8) == 8 * 4 * 2048 * 8
    assert room([T(2, 1, 8)] * 161, [sbp.S(0)] * 161, 2) == 2 * (2 + 3 + 2) * 161 * 8


def clip(inp=None, sigs=None, sq=None, ssq=sbp.P_SUM, most=1.0, out=None, norm=None, k=2):
    sigs = [sbp.S(1), sbp.B] if sigs is None else sigs
    inp = [T(2, 64, 256), T(2, 32, 8, sbp.F32, 1)] if inp is None else inp
    out = [T(2, 64, 256, sbp.F32, 4), T(2, 32, 8, sbp.F32, 5)] if out is None else out
    return status(sbp.sbp_clip, sbp.SbpList(inp, sigs), sq or scalar(2, 9), ssq, most, sbp.SbpList(out, sigs), norm, k)


def test_clip_refusals():
    assert clip(k=0) == K and clip(sigs=[sbp.P_SUM, sbp.B]) == SIGNATURE and clip(sigs=[4, sbp.B]) == AXIS
    assert clip(ssq=sbp.S(0)) == SIGNATURE and clip(ssq=sbp.P_MAX) == SIGNATURE and clip(ssq=77) == AXIS
    assert clip(most=-1.0) == UNSUPPORTED and clip(most=float("nan")) == UNSUPPORTED
    assert clip(sq=T(2, 1, 1, sbp.BF16, 9)) == DTYPE and clip(sq=T(2, 1, 2, sbp.F32, 9)) == SHAPE
    assert clip(norm=T(2, 2, 1, sbp.F32, 8)) == SHAPE and clip(norm=scalar(2, 9)) == ALIAS and clip(norm=scalar(2, 4)) == ALIAS
    assert clip(out=[T(2, 64, 255, sbp.F32, 4), T(2, 32, 8, sbp.F32, 5)]) == SHAPE
    assert clip(out=[T(2, 64, 256, sbp.F32, 4, trans=1), T(2, 32, 8, sbp.F32, 5)]) == UNSUPPORTED
    assert clip(out=[T(2, 64, 256, sbp.F8E4M3, 4), T(2, 32, 8, sbp.F32, 5)]) == DTYPE
    assert clip(inp=[T(2, 2 ** 31 - 1, 2 ** 30), T(2, 32, 8, sbp.F32, 1)], out=[T(2, 2 ** 31 - 1, 2 ** 30, sbp.F32, 4), T(2, 32, 8, sbp.F32, 5)]) == UNSUPPORTED


def test_clip_in_place_is_one_tensor_in_its_own_place():
    two, one = T(2, 64, 256), T(2, 32, 8, sbp.F32, 1)
    assert clip(inp=[two, one], out=[T(2, 64, 256, sbp.F32, 0), one]) == ALIAS                # another type
    assert clip(inp=[two, one], out=[T(2, 64, 256, ld=136), one]) == ALIAS                    # another pitch
    assert clip(inp=[two, one], out=[T(2, 64, 256, at=4), T(2, 32, 8, sbp.F32, 0)]) == ALIAS  # another tensor's place
    shared = sbp.SbpTensor([0x200000000] * 2, 32, 8, sbp.F32)
    assert clip(inp=[two, shared], out=[two, shared]) == ALIAS                                # one buffer cannot be two outputs
    half = sbp.SbpTensor([0x200000000, 0x500000000], 32, 8, sbp.F32)
    assert clip(inp=[two, shared], out=[two, half]) == ALIAS                                  # device 1 reads what device 0 writes
    with pytest.raises(ValueError):
        sbp.sbp_clip(sbp.SbpList([two], [sbp.B]), scalar(2, 9), sbp.B, 1.0, sbp.SbpList([two], [sbp.S(0)]), None, 2, STREAM)
