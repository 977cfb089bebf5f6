"""Device buffers of tests of the operators around an MLP block's products: local tensors with poisoned surroundings."""
from __future__ import annotations

import torch

import paper_2110_15032_amd as sbp

TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
CODE = {"f32": sbp.F32, "bf16": sbp.BF16, "e4m3": sbp.F8E4M3, "e5m2": sbp.F8E5M2}
SIZE = {"f32": 4, "bf16": 2, "e4m3": 1, "e5m2": 1, "u8": 1}
#: half a rounding step, relative
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "e4m3": 2.0 ** -4, "e5m2": 2.0 ** -3}
SIG = {"S0": sbp.S(0), "S1": sbp.S(1), "B": sbp.B}
POISON = 0xA5


class Buf:
    """Rows `pitch` elements apart, 0xA5 in every byte between them, in 64 bytes behind them, and in the rows until something is written."""

    def __init__(self, rows, cols, kind, pitch=0, data=None):
        self.rows, self.cols, self.kind, self.pitch = rows, cols, kind, pitch or cols
        size = SIZE[kind]
        self.used = ((rows - 1) * self.pitch + cols) * size if rows and cols else 0
        self.raw = torch.full((self.used + 64,), POISON, dtype=torch.uint8, device="cuda")
        if data is not None and self.used:
            self.t.copy_(data.to(self.t.dtype) if kind != "u8" else data)

    @property
    def t(self):
        typed = self.raw[: self.used].view(TYPE[self.kind]) if self.kind != "u8" else self.raw[: self.used]
        return typed.as_strided((self.rows, self.cols), (self.pitch, 1)) if self.used else typed.view(-1)[:0].reshape(0, self.cols) if not self.rows else typed.view(self.rows, 0)

    def data_ptr(self):
        return self.raw.data_ptr() if self.used else 0   # an empty local tensor need not be anywhere

    def host(self):
        """The rows in 64 bits (8 bits: as they are), after a look that nothing else was written."""
        left = self.raw.clone()
        if self.used:
            size = SIZE[self.kind]
            cover = torch.as_strided(left, (self.rows, self.cols * size), (self.pitch * size, 1))
            cover.fill_(POISON)
        assert bool((left == POISON).all()), "bytes between or behind the rows were written"
        t = self.t.cpu()
        return t.double() if self.kind in ("f32", "bf16") else t.clone()


def split(n, k):
    """(begin, end) of the balanced split."""
    out, at = [], 0
    for i in range(k):
        m = n // k + (i < n % k)
        out.append((at, at + m))
        at += m
    return out


def slices(x, sig, k):
    """The k local tensors of a global one."""
    if sig == "S0":
        return [x[a:b] for a, b in split(x.shape[0], k)]
    if sig == "S1":
        return [x[:, a:b] for a, b in split(x.shape[1], k)]
    return [x] * k


class Dev:
    """A global tensor on k devices.  data: the global tensor on the host (an input), or None (an output of shape)."""

    def __init__(self, shape, kind, sig, k, pitch=0, trans=0, data=None, shared=False):
        self.kind, self.sig, self.k = kind, sig, k
        self.shape = tuple(shape)
        whole = torch.empty(shape, device="meta") if data is None else data
        local = slices(whole, sig, k)
        stored = [t.T if trans else t for t in local]
        widest = max(t.shape[1] for t in stored)
        self.pitch = widest + pitch if pitch >= 0 else 0          # pitch: that many elements between the longest row and the next
        if pitch == 0:
            self.pitch = 0
        self.bufs = [Buf(t.shape[0], t.shape[1], kind, self.pitch, None if data is None else t) for t in stored]
        if shared:
            self.bufs = [self.bufs[0]] * k
        self.trans = trans
        self.desc = sbp.SbpTensor(self.bufs, *shape, CODE[kind], trans, self.pitch)

    def host(self):
        """The local tensors."""
        got = [b.host() for b in self.bufs]
        return [t.T if self.trans else t for t in got]

    def ref(self):
        return self.desc.ref()


def column(n, kind, sig, k, data=None, shared=False):
    """A vector [n, 1]."""
    return Dev((n, 1), kind, sig, k, data=None if data is None else data.reshape(n, 1), shared=shared)


def room(n):
    """A workspace whose contents are poisoned: they do not matter."""
    return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") if n else None


def rounded(x, kind):
    """A host tensor in 64 bits with the values that `kind` can hold."""
    return x.to(TYPE[kind]).double()


def normal(*shape, seed=0, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return scale * torch.randn(*shape, generator=g, dtype=torch.float64)


def same(a, b):
    """Equal bit for bit (tensors in 64 bits)."""
    return torch.equal(a.contiguous().view(torch.int64), b.contiguous().view(torch.int64))


def close(got, want, bound, what=""):
    """|got - want| <= bound everywhere (tensors in 64 bits), and NaN where want is, there alone."""
    assert got.shape == want.shape, (what, got.shape, want.shape)
    if got.numel() == 0:
        return
    none = want.isnan()
    assert torch.equal(none, got.isnan()), f"{what}: NaN in other places"
    got, want, bound = got[~none], want[~none], bound.expand(none.shape)[~none]
    if got.numel() == 0:
        return
    excess = (got - want).abs() - bound
    assert bool((excess <= 0).all()), f"{what}: off by {float((got - want).abs().max()):.3g}, {int((excess > 0).sum())} of {got.numel()} outside, worst excess {float(excess.max()):.3g}"
