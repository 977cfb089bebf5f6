"""8-bit tensors, layer normalisation and products of 8-bit tensors on the GPU, element by element against the 64-bit implementation.

Half a rounding step: U below.  Every tolerance is written out where it is used; sums of n fp32 terms in any order are within n 2^-24 of the
sum of their magnitudes."""
import ctypes

import numpy as np
import pytest

import oracle as orc
import paper_2110_15032_amd as sbp
from oracle import block8_oracle as o8

pytestmark = pytest.mark.gpu

U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "e4m3": 2.0 ** -4, "e5m2": 2.0 ** -3}
CODE = {"f32": sbp.F32, "bf16": sbp.BF16, "e4m3": sbp.F8E4M3, "e5m2": sbp.F8E5M2}
SIG = {"S0": sbp.S(0), "S1": sbp.S(1), "B": sbp.B}
EPI = {False: sbp.EPI_NONE, True: sbp.EPI_GELU}
POISON = 0xA5


def torch_mod():
    import torch
    return torch


class Buf:
    """Rows of `bytes_` wide elements, `ld` apart, in poisoned device memory with 64 poisoned bytes behind the last row's last element; host() checks
    that nothing but the rows' elements was written."""

    def __init__(self, rows, cols, dtype, ld=0, data=None):
        torch = torch_mod()
        self.rows, self.cols, self.dtype, self.ld = rows, cols, np.dtype(dtype), ld or cols
        self.used = ((rows - 1) * self.ld + cols) * self.dtype.itemsize if rows and cols else 0
        raw = np.full(self.used + 64, POISON, np.uint8)
        if data is not None and self.used:
            self._view(raw)[...] = data
        self.t = torch.from_numpy(raw).cuda()

    def _view(self, raw):
        return np.lib.stride_tricks.as_strided(raw[:self.used].view(self.dtype) if self.used % self.dtype.itemsize == 0 else raw.view(self.dtype),
                                               (self.rows, self.cols), (self.ld * self.dtype.itemsize, self.dtype.itemsize))

    def host(self):
        raw = self.t.cpu().numpy()
        if not self.used:
            assert (raw == POISON).all()
            return np.zeros((self.rows, self.cols), self.dtype)
        got = self._view(raw).copy()
        left = raw.copy()
        self._view(left)[...] = np.full(1, POISON, np.uint8).repeat(self.dtype.itemsize).view(self.dtype)[0]
        assert (left == POISON).all(), "bytes between or behind the rows were written"
        return got

    def data_ptr(self):
        return self.t.data_ptr()


NP = {"f32": np.float32, "bf16": np.uint16, "e4m3": np.uint8, "e5m2": np.uint8}


def store(x, kind):
    """float64 -> stored words of f32 / bf16"""
    return x.astype(np.float32) if kind == "f32" else orc.f64_to_bf16(x) if hasattr(orc, "f64_to_bf16") else bf16_words(x)


def bf16_words(x):
    torch = torch_mod()
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).bfloat16().view(torch.int16).numpy().view(np.uint16).copy()


def value(w):
    return (w.astype(np.uint32) << 16).view(np.float32).astype(np.float64) if w.dtype == np.uint16 else w.astype(np.float64)


def parts(n, k):
    return [orc.split_range(n, k, i) for i in range(k)]


def split(a, sig, k):
    if sig == "S0":
        return [a[b:e] for b, e in parts(a.shape[0], k)]
    if sig == "S1":
        return [a[:, b:e] for b, e in parts(a.shape[1], k)]
    return [a] * k


def up(shards, kind, ld=0):
    return [Buf(*s.shape, NP[kind], ld, s) for s in shards]


def desc(bufs, rows, cols, kind, trans=0, ld=0):
    return sbp.SbpTensor(bufs, rows, cols, CODE[kind], trans, ld)


def sync():
    torch_mod().cuda.synchronize()


def blocks(n):
    return -(-n // 128)


def quantized(shards, kind, ld=0, lds=0):
    """stored rows -> device values and scales, and what they stand for"""
    enc = [o8.quantize(s, kind) if s.size else (np.zeros(s.shape, np.uint8), np.zeros((s.shape[0], blocks(s.shape[1])), np.uint8)) for s in shards]
    return ([Buf(*q.shape, np.uint8, ld, q) for q, _ in enc], [Buf(*s.shape, np.uint8, lds, s) for _, s in enc],
            [o8.dequantize(q, s, kind) if q.size else q.astype(np.float64) for q, s in enc])


def close(got, want, tol, what=""):
    assert got.shape == want.shape
    nan = np.isnan(want)
    assert (np.isnan(got) == nan).all(), f"{what}: NaN elsewhere"
    same = got == want
    with np.errstate(invalid="ignore"):
        bad = ~nan & ~same & ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: {got[bad][0]!r} for {want[bad][0]!r}, allowed {np.broadcast_to(tol, got.shape)[bad][0]:.3g}"


def activations(rng, rows, cols):
    x = rng.normal(size=(rows, cols)) * np.where(rng.random(cols) < 0.05, 30.0, 1.0)
    x[rng.random((rows, cols)) < 0.02] = 0.0
    return x


# ------------------------------------------------------------------ 8-bit tensors
SHAPES = [(1, 1, 1, "B"), (1, 7, 1, "S0"), (3, 128, 2, "S0"), (5, 129, 2, "B"), (1, 4096, 1, "B"), (300, 1001, 3, "S0"), (131, 1000, 3, "S1"), (257, 64, 8, "S0"),
          (128, 640, 4, "S1"), (3, 70, 8, "S0"), (513, 2049, 2, "S1")]


@pytest.mark.parametrize("trans", [0, 1])
@pytest.mark.parametrize("kind", ["e4m3", "e5m2"])
@pytest.mark.parametrize("xk", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,k,sig", SHAPES)
def test_quantize_bit_for_bit_and_back(rows, cols, k, sig, xk, kind, trans):
    rng = np.random.default_rng(rows * 1000 + cols)
    w = store(activations(rng, rows, cols), xk)
    shards = split(w, sig, k)
    widest = max(s.shape[1] for s in shards)
    longest = max(s.shape[0] for s in shards)
    pitch = rng.integers(0, 2) * (widest + int(rng.integers(1, 9)))
    qld = rng.integers(0, 2) * ((longest if trans else widest) + int(rng.integers(1, 17)))
    sld = rng.integers(0, 2) * (blocks(longest if trans else widest) + int(rng.integers(0, 5)))
    x = up(shards, xk, pitch)
    stored = [s.T if trans else s for s in shards]
    q = [Buf(*s.shape, np.uint8, qld) for s in stored]
    sc = [Buf(s.shape[0], blocks(s.shape[1]) if s.size else 0, np.uint8, sld) for s in stored]
    dq, ds = desc(q, rows, cols, kind, trans, qld), sbp.SbpScales(sc, sld)
    sbp.sbp_quantize(desc(x, rows, cols, xk, 0, pitch), SIG[sig], dq, ds, k)
    outs = {}
    for yk in ("f32", "bf16"):
        y = [Buf(*s.shape, NP[yk], pitch) for s in shards]
        sbp.sbp_dequantize(dq, ds, SIG[sig], desc(y, rows, cols, yk, 0, pitch), k)
        outs[yk] = y
    sync()
    for i, s in enumerate(stored):
        got, gots = q[i].host(), sc[i].host()
        if not s.size:
            continue
        want, wants = o8.quantize(value(np.ascontiguousarray(s)), kind)
        np.testing.assert_array_equal(gots, wants)
        np.testing.assert_array_equal(got, want)
        back = o8.dequantize(want, wants, kind)
        back = back.T if trans else back
        for yk in ("f32", "bf16"):
            np.testing.assert_array_equal(value(outs[yk][i].host()), back)   # exact in either type


@pytest.mark.parametrize("kind", ["e4m3", "e5m2"])
@pytest.mark.parametrize("xk", ["bf16", "f32"])
@pytest.mark.parametrize("trans", [0, 1])
def test_quantize_edges(kind, xk, trans):
    """the ends of the type, ties, the ends of the exponent range, blocks of zeros, infinities, NaN"""
    rng = np.random.default_rng(3)
    t = o8.decode_table(kind)[:128]
    t = t[np.isfinite(t)]
    rows = []
    for top in (448.0, 57344.0, 1.75, 1.7578125, 0.875, 3.3e38, 1e-30, 2.0 ** -100):
        r = rng.uniform(-1, 1, 256) * top
        r[0], r[128] = top, -top
        rows.append(r)
    ties = np.concatenate([(t[1:] + t[:-1]) / 2, t])
    r = np.resize(ties, 256)
    r[0] = r[128] = t[-1]
    rows.append(r)
    rows.append(np.zeros(256))
    r = rng.normal(size=256)
    r[3], r[130], r[131] = np.inf, np.nan, -np.inf
    rows.append(r)
    rows.append(np.full(256, np.nan))
    rows.append(np.full(256, np.inf))
    w = store(np.array(rows), xk)
    w = np.ascontiguousarray(w.T) if trans else w
    x = up([w], xk)
    s = w.T if trans else w
    q, sc = Buf(*s.shape, np.uint8), Buf(s.shape[0], blocks(s.shape[1]), np.uint8)
    y = Buf(*w.shape, np.float32)
    dq, ds = desc([q], *w.shape, kind, trans), sbp.SbpScales([sc])
    sbp.sbp_quantize(desc(x, *w.shape, xk), sbp.B, dq, ds, 1)
    sbp.sbp_dequantize(dq, ds, sbp.B, desc([y], *w.shape, "f32"), 1)
    sync()
    v = value(np.ascontiguousarray(s))
    want, wants = o8.quantize(v, kind)
    np.testing.assert_array_equal(sc.host(), wants)
    got = q.host()
    nan = np.isnan(o8.decode_table(kind)[want])
    np.testing.assert_array_equal(np.isnan(o8.decode_table(kind)[got]), nan)
    np.testing.assert_array_equal(got[~nan], want[~nan])
    # the largest fp32 numbers round up to 256 * 2^120 (or 8 * 2^125) = 2^128, which fp32 does not have: infinity
    with np.errstate(over="ignore"):
        back = o8.dequantize(want, wants, kind).astype(np.float32)
    np.testing.assert_array_equal(y.host(), back.T if trans else back)


@pytest.mark.parametrize("kind", ["e4m3", "e5m2"])
def test_smallest_scales(kind):
    """below 2^-119 (e4m3) or 2^-112 the scale stays 2^-127 and the values come nearer to zero; fp32 numbers throughout, subnormal ones too"""
    rng = np.random.default_rng(4)
    x = (rng.uniform(-1, 1, (6, 256)) * 2.0 ** np.array([[-110.0], [-118], [-120], [-126], [-130], [-140]])).astype(np.float32)
    q, sc, y = Buf(6, 256, np.uint8), Buf(6, 2, np.uint8), Buf(6, 256, np.float32)
    dq, ds = desc([q], 6, 256, kind), sbp.SbpScales([sc])
    sbp.sbp_quantize(desc(up([x], "f32"), 6, 256, "f32"), sbp.B, dq, ds, 1)
    sbp.sbp_dequantize(dq, ds, sbp.B, desc([y], 6, 256, "f32"), 1)
    sync()
    want, wants = o8.quantize(x.astype(np.float64), kind)
    np.testing.assert_array_equal(sc.host(), wants)
    # -0 and 0 stand for the same
    np.testing.assert_array_equal(o8.decode_table(kind)[q.host()], o8.decode_table(kind)[want])
    np.testing.assert_array_equal(y.host().astype(np.float64), o8.dequantize(want, wants, kind))


@pytest.mark.parametrize("trans", [0, 1])
@pytest.mark.parametrize("kind", ["e4m3", "e5m2"])
@pytest.mark.parametrize("xk", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,k,sig", [(1, 1, 1, "B"), (200, 333, 3, "S0"), (70, 512, 2, "S1")])
def test_quantize_and_restore_gelu(rows, cols, k, sig, xk, kind, trans):
    rng = np.random.default_rng(5)
    w = store(rng.normal(size=(rows, cols)) * 3, xk)
    shards = split(w, sig, k)
    x = up(shards, xk)
    stored = [s.T if trans else s for s in shards]
    q, sc = [Buf(*s.shape, np.uint8) for s in stored], [Buf(s.shape[0], blocks(s.shape[1]), np.uint8) for s in stored]
    sbp.sbp_quantize(desc(x, rows, cols, xk), SIG[sig], desc(q, rows, cols, kind, trans), sbp.SbpScales(sc), k, None, sbp.EPI_GELU)
    p8, ps, stands = quantized([value(np.ascontiguousarray(s)) for s in stored], kind)
    y = {yk: [Buf(*s.shape, NP[yk]) for s in shards] for yk in ("f32", "bf16")}
    for yk in y:
        sbp.sbp_dequantize(desc(p8, rows, cols, kind, trans), sbp.SbpScales(ps), SIG[sig], desc(y[yk], rows, cols, yk), k, None, sbp.EPI_GELU)
    sync()
    rel = 2.3e-5   # of the fit, and a rounding of the argument's scaling
    for i, s in enumerate(stored):
        want = o8.gelu(value(np.ascontiguousarray(s)))
        gots = sc[i].host()
        lo, hi = o8.scale_bytes(want * (1 - rel), kind), o8.scale_bytes(want * (1 + rel), kind)
        assert ((gots >= lo) & (gots <= hi)).all()
        scale = o8.spread(gots, s.shape[1])
        smallest = 2.0 ** (-6 - 3 if kind == "e4m3" else -14 - 2)   # step of the subnormal numbers
        back = o8.decode_table(kind)[q[i].host()] * scale
        close(back, want, np.maximum(np.abs(want) * (1 + rel) * U[kind], scale * smallest / 2) + rel * np.abs(want), "quantized gelu")
        w8 = o8.gelu(stands[i])
        w8 = w8.T if trans else w8
        # fp32: erfc, two products and their roundings, 1e-7 and 3 * 2^-24; an argument of erfc off by 2^-24 of itself moves it by up to z^2 2^-23 of its value
        z2 = np.minimum((stands[i].T if trans else stands[i]) ** 2 / 2, 100)
        close(y["f32"][i].host().astype(np.float64), w8, np.abs(w8) * (3e-7 + (2 * z2 + 4) * U["f32"]) + 1e-38, "restored gelu, fp32")
        close(value(y["bf16"][i].host()), w8, np.abs(w8) * (rel + z2 * 2 ** -22) * 1.01 + np.abs(w8) * 1.001 * U["bf16"] + 1e-37, "restored gelu, bf16")


@pytest.mark.parametrize("ak", ["e4m3", "e5m2", "bf16", "f32"])
@pytest.mark.parametrize("yk", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,k,sig", [(1, 1, 1, "B"), (3, 130, 2, "B"), (333, 1001, 3, "S0"), (64, 4096, 8, "S1"), (5, 9, 8, "S0")])
def test_gelu_grad(rows, cols, k, sig, ak, yk):
    rng = np.random.default_rng(6)
    a = rng.normal(size=(rows, cols)) * 2.5
    a.flat[::17] *= 6
    dh = store(rng.normal(size=(rows, cols)), yk)
    ld = int(rng.integers(0, 2)) * (cols + 3)
    if ak in ("e4m3", "e5m2"):
        da_, sc, vals = quantized(split(a, sig, k), ak, ld)
        scales = sbp.SbpScales(sc)
    else:
        w = store(a, ak)
        da_, scales, vals = up(split(w, sig, k), ak, ld), None, [value(s) for s in split(w, sig, k)]
    h = up(split(dh, sig, k), yk)
    out = [Buf(*s.shape, NP[yk], ld) for s in split(dh, sig, k)]
    sbp.sbp_gelu_grad(desc(da_, rows, cols, ak, 0, ld), scales, SIG[sig], desc(h, rows, cols, yk), desc(out, rows, cols, yk, 0, ld), k)
    sync()
    for o, v, d in zip(out, vals, split(value(dh), sig, k)):
        want = d * o8.gelu_slope(v)
        close(value(o.host()), want, np.abs(d) * 5e-7 + np.abs(want) * 1.001 * U[yk] + 1e-38, "gelu'")


def test_gelu_grad_specials_and_differences():
    a = np.array([[0.0, -0.0, 40.0, -40.0, np.inf, -np.inf, np.nan, 1.0, -1.0, 14.5, -14.5]]).astype(np.float32)
    one = np.ones_like(a)
    out = Buf(*a.shape, np.float32)
    sbp.sbp_gelu_grad(desc(up([a], "f32"), *a.shape, "f32"), None, sbp.B, desc(up([one], "f32"), *a.shape, "f32"), desc([out], *a.shape, "f32"), 1)
    x = np.linspace(-6, 6, 999).astype(np.float32)[None]
    o2 = Buf(*x.shape, np.float32)
    sbp.sbp_gelu_grad(desc(up([x], "f32"), *x.shape, "f32"), None, sbp.B, desc(up([np.ones_like(x)], "f32"), *x.shape, "f32"), desc([o2], *x.shape, "f32"), 1)
    sync()
    g = out.host()[0]
    np.testing.assert_allclose(g[:6], [0.5, 0.5, 1, 0, 1, 0], atol=1e-6)
    assert np.isnan(g[6])
    h = 1e-4
    v = x.astype(np.float64)
    # central differences: h^2 / 6 of the third derivative, at most 1.2
    np.testing.assert_allclose(o2.host(), (o8.gelu(v + h) - o8.gelu(v - h)) / (2 * h), atol=5e-7 + 2e-9 + 1e-8)


# ------------------------------------------------------------------ layer normalisation
NORMS = [(1, 1, 1, "B"), (1, 4096, 1, "B"), (3, 7, 2, "S0"), (2, 128, 8, "S0"), (77, 512, 3, "S0"), (65, 513, 2, "B"), (41, 1001, 3, "S0"), (300, 2048, 2, "S0"),
         (33, 4095, 1, "S0"), (19, 8192, 2, "S0"), (11, 8193, 2, "B"), (9, 16384, 1, "S0"), (1500, 96, 2, "S0")]


def norm_inputs(rng, rows, cols):
    x = activations(rng, rows, cols) + rng.normal(size=cols) * 0.3
    if rows > 2:
        x[1] = 0.0          # a row of zeros: xhat is 0, rstd 1 / sqrt(eps)
        x[2] += 100.0       # far from zero
    return x


def norm_tolerance(x, gamma, beta, mean, rstd):
    """mean: a tree over at most 32 elements a lane, 6 steps, 16 waves; xhat off by that times rstd and by rstd's own error; a rounding each for the rest"""
    a = np.abs(x).mean(1, keepdims=True)
    xhat = np.abs(x - mean[:, None]) * rstd[:, None]
    return U["f32"] * (64 * a * rstd[:, None] + 64 * xhat + 4 * np.abs(x) * rstd[:, None]) * np.abs(gamma) + 2 * U["f32"] * (xhat * np.abs(gamma) + np.abs(beta))


@pytest.mark.parametrize("wk", ["f32", "bf16", None])
@pytest.mark.parametrize("xk,yk", [("bf16", "bf16"), ("bf16", "e4m3"), ("f32", "f32"), ("f32", "e5m2"), ("bf16", "f32")])
@pytest.mark.parametrize("rows,cols,k,sig", NORMS)
def test_layernorm(rows, cols, k, sig, xk, yk, wk):
    rng = np.random.default_rng(rows + cols)
    w = store(norm_inputs(rng, rows, cols), xk)
    shards = split(w, sig, k)
    ld = int(rng.integers(0, 2)) * (cols + int(rng.integers(1, 9)))
    gamma, beta = np.ones(cols), np.zeros(cols)
    dg = db = None
    if wk:
        gw, bw = store(1 + 0.2 * rng.normal(size=(cols, 1)), wk), store(0.3 * rng.normal(size=(cols, 1)), wk)
        gamma, beta = value(gw)[:, 0], value(bw)[:, 0]
        dg, db = desc(up([gw], wk) * k, cols, 1, wk), desc(up([bw], wk) * k, cols, 1, wk)
    y = [Buf(*s.shape, NP[yk], ld) for s in shards]
    sc = [Buf(s.shape[0], blocks(cols) if s.size else 0, np.uint8) for s in shards]
    mean, rstd = [Buf(s.shape[0], 1, np.float32) for s in shards], [Buf(s.shape[0], 1, np.float32) for s in shards]
    sbp.sbp_layernorm(desc(up(shards, xk, ld), rows, cols, xk, 0, ld), SIG[sig], dg, db, 1e-5, desc(y, rows, cols, yk, 0, ld),
                      sbp.SbpScales(sc) if yk[0] == "e" else None, desc(mean, rows, 1, "f32"), desc(rstd, rows, 1, "f32"), k)
    sync()
    for i, s in enumerate(shards):
        got, m, r = y[i].host(), mean[i].host().astype(np.float64), rstd[i].host().astype(np.float64)
        gots = sc[i].host() if yk[0] == "e" else None
        if not s.size:
            continue
        v = value(s)
        want, wm, wr = o8.layernorm(v, gamma, beta, 1e-5)
        close(m[:, 0], wm, 48 * U["f32"] * np.abs(v).mean(1), "mean")
        # the variance's relative error: its sum's, and the mean's squared over it
        close(r[:, 0], wr, wr * (48 * U["f32"] + (48 * U["f32"] * np.abs(v).mean(1) * wr) ** 2), "rstd")
        tol = norm_tolerance(v, gamma, beta, wm, wr)
        if gots is None:
            close(value(got), want, tol + (np.abs(want) + tol) * U[yk], "y")
        else:
            most = o8.scale_bytes(np.abs(want) + tol, yk)
            least = o8.scale_bytes(np.maximum(np.abs(want) - tol, 0), yk)
            assert ((gots >= least) & (gots <= most)).all()
            scale = o8.spread(gots, cols)
            smallest = 2.0 ** (-9 if yk == "e4m3" else -16)
            close(o8.decode_table(yk)[got] * scale, want, tol + np.maximum((np.abs(want) + tol) * U[yk], scale * smallest / 2), "y in 8 bits")


def test_layernorm_without_statistics_and_nan_stays_in_its_row():
    rng = np.random.default_rng(8)
    x = rng.normal(size=(6, 600)).astype(np.float32)
    x[2, 17], x[4, 5] = np.nan, np.inf
    y = Buf(6, 600, np.float32)
    sbp.sbp_layernorm(desc(up([x], "f32"), 6, 600, "f32"), sbp.B, None, None, 1e-5, desc([y], 6, 600, "f32"), None, None, None, 1)
    sync()
    got = y.host()
    assert np.isnan(got[2]).all() and np.isnan(got[4]).any()
    keep = [0, 1, 3, 5]
    want, m, r = o8.layernorm(x[keep].astype(np.float64), 1.0, 0.0, 1e-5)
    close(got[keep].astype(np.float64), want, norm_tolerance(x[keep].astype(np.float64), 1.0, 0.0, m, r) + np.abs(want) * U["f32"])


@pytest.mark.parametrize("wk", ["f32", "bf16", None])
@pytest.mark.parametrize("xk,yk", [("bf16", "bf16"), ("f32", "f32"), ("e4m3", "bf16"), ("e5m2", "f32")])
@pytest.mark.parametrize("rows,cols,k,sig", NORMS + [(5000, 130, 1, "S0"), (2600, 600, 2, "B")])
def test_layernorm_grad(rows, cols, k, sig, xk, yk, wk):
    rng = np.random.default_rng(rows + 7 * cols)
    x = norm_inputs(rng, rows, cols)
    ld = int(rng.integers(0, 2)) * (cols + int(rng.integers(1, 9)))
    if xk[0] == "e":
        bx, bs, vals = quantized(split(x, sig, k), xk, ld)
        scales = sbp.SbpScales(bs)
    else:
        w = split(store(x, xk), sig, k)
        bx, scales, vals = up(w, xk, ld), None, [value(s) for s in w]
    gamma, dg = np.ones(cols), None
    if wk:
        gw = store(1 + 0.2 * rng.normal(size=(cols, 1)), wk)
        gamma, dg = value(gw)[:, 0], desc(up([gw], wk) * k, cols, 1, wk)
    dy = split(store(rng.normal(size=(rows, cols)) + 0.2, yk), sig, k)
    stats = [o8.layernorm(v, 1.0, 0.0, 1e-5)[1:] if v.size else (np.zeros(0), np.zeros(0)) for v in vals]
    mean = [m.astype(np.float32)[:, None] for m, _ in stats]
    rstd = [r.astype(np.float32)[:, None] for _, r in stats]
    dx = [Buf(*s.shape, NP[yk], ld) for s in dy]
    og, ob = [Buf(cols, 1, np.float32) for _ in range(k)], [Buf(cols, 1, np.float32) for _ in range(k)]
    need = sbp.sbp_layernorm_grad_workspace(rows, cols, SIG[sig], k)
    room = Buf(1, need, np.uint8)
    args = (desc(bx, rows, cols, xk, 0, ld), scales, SIG[sig], dg, desc(up(mean, "f32"), rows, 1, "f32"), desc(up(rstd, "f32"), rows, 1, "f32"),
            desc(up(dy, yk), rows, cols, yk))
    sbp.sbp_layernorm_grad(*args, desc(dx, rows, cols, yk, 0, ld), desc(og, cols, 1, "f32"), desc(ob, cols, 1, "f32"), room.t[:need] if need else None, k)
    again = [Buf(*s.shape, NP[yk], ld) for s in dy]
    sbp.sbp_layernorm_grad(*args, desc(again, rows, cols, yk, 0, ld), None, None, None, k)   # without the weights' gradients
    sync()
    room.host()
    for i, v in enumerate(vals):
        got, g1, b1 = dx[i].host(), og[i].host()[:, 0].astype(np.float64), ob[i].host()[:, 0].astype(np.float64)
        if not v.size:
            assert (g1 == 0).all() and (b1 == 0).all()
            again[i].host()
            continue
        np.testing.assert_array_equal(again[i].host(), got)
        m, r, d = mean[i].astype(np.float64)[:, 0], rstd[i].astype(np.float64)[:, 0], value(dy[i])
        want, wg, wb = o8.layernorm_grad(v, gamma, m, r, d)
        xhat, g = np.abs(v - m[:, None]) * r[:, None], np.abs(d * gamma)
        ex = 2 * U["f32"] * (np.abs(v) + np.abs(m)[:, None]) * r[:, None] + 2 * U["f32"] * xhat   # xhat's error
        s2 = np.abs((d * gamma * (v - m[:, None]) * r[:, None]).mean(1, keepdims=True))
        tol = r[:, None] * (64 * U["f32"] * (g + g.mean(1, keepdims=True) + xhat * (g * xhat).mean(1, keepdims=True)) + ex * s2 + xhat * (g * ex).mean(1, keepdims=True))
        close(value(got), want, tol + (np.abs(want) + tol) * U[yk], "dx")
        n = v.shape[0] + 16
        close(g1, wg, (np.abs(d) * ex).sum(0) + n * U["f32"] * (np.abs(d) * xhat).sum(0), "dgamma")
        close(b1, wb, n * U["f32"] * np.abs(d).sum(0), "dbeta")


# ------------------------------------------------------------------ products
def matmul_case(rng, M, K, N, k, sig, xk, wk, yk, gelu=False, dense=False, special=None, aligned=False):
    x, w = activations(rng, M, K), rng.normal(size=(N, K)) * 0.05     # w as it is stored: [N, K]
    if special is not None:
        special(x, w)
    xsig, wsig = {"S0": ("S0", "B"), "S1": ("B", "S0"), "P": ("S1", "S1"), "B": ("B", "B")}[sig]   # of the stored rows
    xs, ws = split(x, xsig, k), split(w, wsig, k)
    kl, r16 = max(s.shape[1] for s in xs), lambda n: -(-n // 16) * 16  # noqa: E731
    ldx, ldw = (0, 0) if dense else (r16(kl) + 16 * int(rng.integers(0, 3)), r16(kl) + 16 * int(rng.integers(0, 3)))
    lds = 0 if dense else blocks(kl) + int(rng.integers(0, 6))
    lds = -(-blocks(kl) // 4) * 4 if aligned else lds
    bx, bxs, vx = quantized(xs, xk, ldx, lds)
    bw, bws, vw = quantized(ws, wk, ldw, lds)
    a_sig, b_sig, y_sig = {"S0": (sbp.S(0), sbp.B, sbp.S(0)), "S1": (sbp.B, sbp.S(1), sbp.S(1)), "P": (sbp.S(1), sbp.S(0), sbp.P_SUM), "B": (sbp.B,) * 3}[sig]
    if sig in ("S0", "B"):
        bw, bws = [bw[0]] * k, [bws[0]] * k
    if sig in ("S1", "B"):
        bx, bxs = [bx[0]] * k, [bxs[0]] * k
    shapes = [(vx[i].shape[0], vw[i].shape[0]) for i in range(k)]
    ldy = int(rng.integers(0, 2)) * (max(s[1] for s in shapes) + int(rng.integers(1, 9)))
    y = [Buf(*s, NP[yk], ldy) for s in shapes]
    sbp.sbp_matmul_f8(desc(bx, M, K, xk, 0, ldx), sbp.SbpScales(bxs, lds), a_sig, desc(bw, K, N, wk, 1, ldw), sbp.SbpScales(bws, lds), b_sig,
                      desc(y, M, N, yk, 0, ldy), y_sig, k, None, EPI[gelu])
    sync()
    for i in range(k):
        got = value(y[i].host())
        if not got.size:
            continue
        want = vx[i] @ vw[i].T
        total = np.abs(vx[i]) @ np.abs(vw[i]).T
        tol = vx[i].shape[1] * U["f32"] * total
        if yk == "bf16":
            tol = tol + 2.0 ** -11 * total
        if gelu:
            tol = 1.13 * tol + 2.3e-5 * np.abs(o8.gelu(want))   # gelu' is at most 1.129
            want = o8.gelu(want)
        close(got, want, tol + (np.abs(want) + tol) * U[yk] + 1e-37, f"shard {i}")


@pytest.mark.parametrize("sig,k,yk", [("B", 1, "bf16"), ("B", 1, "f32"), ("S0", 2, "bf16"), ("S0", 2, "f32"), ("S1", 3, "bf16"), ("S1", 3, "f32"), ("P", 3, "f32")])
@pytest.mark.parametrize("M,K,N", [(1, 1, 1), (1, 128, 16), (1, 4096, 100), (3, 130, 5), (16, 384, 48), (17, 1000, 33), (64, 256, 256), (100, 640, 130), (129, 1001, 257),
                                   (300, 2048, 272), (513, 384, 515), (5, 515, 1030), (260, 128, 64)])
def test_matmul_f8(M, K, N, sig, k, yk):
    for dense in (False, True):
        matmul_case(np.random.default_rng(M + K + N), M, K, N, k, sig, "e4m3", "e4m3", yk, dense=dense)


@pytest.mark.parametrize("aligned", [True, False])
@pytest.mark.parametrize("yk", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N", [(9, 300, 9), (3, 650, 4200), (2, 520, 8300), (4200, 300, 7), (300, 1700, 500), (30, 300, 8300), (8300, 300, 5), (8300, 140, 30), (40, 1040, 8300),
                                   (200, 129, 9000), (3000, 2200, 2900), (4200, 2250, 4300), (7900, 300, 3900)])
def test_matmul_f8_every_tile(M, K, N, yk, aligned):
    """few rows, few columns, few and many of either: with 256 compute units each size has another tile, the last ones more tiles than workgroups; rows
    of operands and scales aligned for loads into shared memory, and not"""
    matmul_case(np.random.default_rng(M + K + N), M, K, N, 1, "B", "e4m3", "e4m3", yk, dense=not aligned, aligned=aligned)


@pytest.mark.parametrize("xk,wk", [("e4m3", "e5m2"), ("e5m2", "e4m3"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("yk,sig", [("bf16", "S1"), ("f32", "P"), ("f32", "S0")])
@pytest.mark.parametrize("M,K,N", [(2, 300, 40), (150, 777, 300), (300, 1024, 512)])
def test_matmul_f8_types(M, K, N, sig, yk, xk, wk):
    matmul_case(np.random.default_rng(11), M, K, N, 2, sig, xk, wk, yk)


@pytest.mark.parametrize("yk", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N", [(1, 256, 40), (140, 300, 270), (300, 512, 256)])
def test_matmul_f8_gelu(M, K, N, yk):
    matmul_case(np.random.default_rng(12), M, K, N, 2, "S1", "e4m3", "e4m3", yk, gelu=True)
    matmul_case(np.random.default_rng(13), M, K, N, 2, "S0", "e4m3", "e4m3", yk, gelu=True, dense=True)


@pytest.mark.parametrize("xk,wk", [("e4m3", "e5m2"), ("e5m2", "e4m3"), ("e5m2", "e5m2"), ("e4m3", "e4m3")])
@pytest.mark.parametrize("yk", ["bf16", "f32"])
def test_matmul_f8_largest_tile_types_and_gelu(yk, xk, wk):
    matmul_case(np.random.default_rng(14), 4000, 260, 4000, 1, "B", xk, wk, yk, gelu=True, aligned=True)
    matmul_case(np.random.default_rng(15), 4096, 390, 1100, 4, "S1", xk, wk, yk, aligned=True)


@pytest.mark.parametrize("yk", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N", [(3, 200, 20), (300, 400, 270), (64, 2300, 512)])
def test_matmul_f8_blocks_of_very_different_scale(M, K, N, yk):
    """scales from 2^-40 to 2^40, each row and block its own; a block of zeros; NaN stays in its row and column"""
    def special(x, w):
        rng = np.random.default_rng(14)
        for m in (x, w):
            nb = blocks(K)
            m *= o8.spread((127 + rng.integers(-40, 41, (m.shape[0], nb))).astype(np.uint8), K)
            m[:, :128] = 0.0 if m is x else m[:, :128]
        x[1, K - 1] = np.nan
        w[2, 5] = np.nan
    with np.errstate(invalid="ignore"):
        matmul_case(np.random.default_rng(15), M, K, N, 1, "B", "e4m3", "e4m3", yk, special=special)


# ------------------------------------------------------------------ together
def mlp_step(torch, seed, stream=None):
    """A training step of an MLP block in 8 bits on two devices, column- and then row-parallel, and its plain form in 64 bits from the same 8-bit tensors."""
    k, T, D, F = 2, 192, 256, 512
    g = torch.Generator(device="cuda").manual_seed(seed)
    bf = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    e = lambda *s, dtype=torch.bfloat16: torch.full(s, float("nan"), dtype=dtype, device="cuda")  # noqa: E731
    u8 = lambda *s: torch.full(s, 255, dtype=torch.uint8, device="cuda")  # noqa: E731
    S0, S1, B, P = sbp.S(0), sbp.S(1), sbp.B, sbp.P_SUM
    t = {}
    t["x"], t["dz"] = bf(T, D), bf(T, D)
    t["gamma"], t["beta"] = 1 + 0.1 * torch.randn(D, generator=g, device="cuda"), 0.1 * torch.randn(D, generator=g, device="cuda")
    w1, w2 = (0.05 * bf(D, F)), (0.05 * bf(F, D))
    fl = F // k
    t["w1"], t["w2"] = [w1[:, i * fl:(i + 1) * fl].contiguous() for i in range(k)], [w2[i * fl:(i + 1) * fl].contiguous() for i in range(k)]
    X = lambda ts, r, c, dt, trans=0: sbp.SbpTensor(ts, r, c, dt, trans)  # noqa: E731

    def q8(name, ts, sig, r, c, dt, trans, kind=sbp.F8E4M3, epi=sbp.EPI_NONE):
        n = k if ts[0] is not ts[-1] or len(ts) == 1 else 1
        shape = [(a.shape[1], a.shape[0]) if trans else tuple(a.shape) for a in ts]
        t[name] = [u8(*s) for s in shape]
        t[name + "_s"] = [u8(s[0], blocks(s[1])) for s in shape]
        d = (X(t[name], r, c, kind, trans), sbp.SbpScales(t[name + "_s"]))
        sbp.sbp_quantize(X(ts, r, c, dt), sig, *d, k, stream, epi)
        return d

    def step():
        # weights: both operands' reductions contiguous, forward and backward
        dw1, dw2 = q8("w1q", t["w1"], S1, D, F, sbp.BF16, 1), q8("w2q", t["w2"], S0, F, D, sbp.BF16, 1)
        # forward: every device normalises its copy
        t["y"], t["ys"] = [u8(T, D) for _ in range(k)], [u8(T, blocks(D)) for _ in range(k)]
        t["mean"], t["rstd"] = [e(T, dtype=torch.float32) for _ in range(k)], [e(T, dtype=torch.float32) for _ in range(k)]
        vec = lambda v: X([v] * k, v.numel(), 1, sbp.F32)  # noqa: E731
        stat = lambda n: X(t[n], T, 1, sbp.F32)  # noqa: E731
        y8 = (X(t["y"], T, D, sbp.F8E4M3), sbp.SbpScales(t["ys"]))
        sbp.sbp_layernorm(X([t["x"]] * k, T, D, sbp.BF16), B, vec(t["gamma"]), vec(t["beta"]), 1e-5, *y8, stat("mean"), stat("rstd"), k, stream)
        t["a"] = [e(T, fl) for _ in range(k)]
        sbp.sbp_matmul_f8(*y8, B, *dw1, S1, X(t["a"], T, F, sbp.BF16), S1, k, stream)
        a8 = q8("aq", t["a"], S1, T, F, sbp.BF16, 0)                                  # kept for the backward pass
        h8 = q8("hq", t["a"], S1, T, F, sbp.BF16, 0, epi=sbp.EPI_GELU)
        t["zp"] = [e(T, D, dtype=torch.float32) for _ in range(k)]
        sbp.sbp_matmul_f8(*h8, S1, *dw2, S0, X(t["zp"], T, D, sbp.F32), P, k, stream)
        t["z"] = [e(T, D, dtype=torch.float32) for _ in range(k)]
        sbp.sbp_boxing(X(t["zp"], T, D, sbp.F32), P, X(t["z"], T, D, sbp.F32), B, k, stream)
        # backward
        dz = [t["dz"].clone() for _ in range(k)]
        dz8 = q8("dzq", dz, B, T, D, sbp.BF16, 0, sbp.F8E5M2)
        w2r = q8("w2r", t["w2"], S0, F, D, sbp.BF16, 0)                               # [F, D] rows: dH = dZ W2^T reduces over D
        t["dh"] = [e(T, fl) for _ in range(k)]
        wt = X(t["w2r"], D, F, sbp.F8E4M3, 1)                                         # W2^T [D, F], S(1), stored transposed
        sbp.sbp_matmul_f8(*dz8, B, wt, w2r[1], S1, X(t["dh"], T, F, sbp.BF16), S1, k, stream)
        t["da"] = [e(T, fl) for _ in range(k)]
        sbp.sbp_gelu_grad(*a8, S1, X(t["dh"], T, F, sbp.BF16), X(t["da"], T, F, sbp.BF16), k, stream)
        # dW2 = H^T dZ from the kept pre-activation: H again, both operands transposed so that the tokens are contiguous
        t["h"] = [e(T, fl) for _ in range(k)]
        sbp.sbp_dequantize(*a8, S1, X(t["h"], T, F, sbp.BF16), k, stream, sbp.EPI_GELU)
        ht, dzt = q8("ht", t["h"], S1, T, F, sbp.BF16, 1), q8("dzt", dz, B, T, D, sbp.BF16, 1, sbp.F8E5M2)
        t["dw2"] = [e(fl, D, dtype=torch.float32) for _ in range(k)]
        sbp.sbp_matmul_f8(X(t["ht"], F, T, sbp.F8E4M3), ht[1], S0, X(t["dzt"], T, D, sbp.F8E5M2, 1), dzt[1], B, X(t["dw2"], F, D, sbp.F32), S0, k, stream)
        # dY = dA W1^T, P(sum) -> B, and through the norm
        da8 = q8("daq", t["da"], S1, T, F, sbp.BF16, 0, sbp.F8E5M2)
        q8("w1r", t["w1"], S1, D, F, sbp.BF16, 0)
        t["dyp"], t["dy"] = [e(T, D, dtype=torch.float32) for _ in range(k)], [e(T, D, dtype=torch.float32) for _ in range(k)]
        sbp.sbp_matmul_f8(*da8, S1, X(t["w1r"], F, D, sbp.F8E4M3, 1), sbp.SbpScales(t["w1r_s"]), S0, X(t["dyp"], T, D, sbp.F32), P, k, stream)
        sbp.sbp_boxing(X(t["dyp"], T, D, sbp.F32), P, X(t["dy"], T, D, sbp.F32), B, k, stream)
        t["dx"] = [e(T, D, dtype=torch.float32) for _ in range(k)]
        t["dgamma"], t["dbeta"] = [e(D, dtype=torch.float32) for _ in range(k)], [e(D, dtype=torch.float32) for _ in range(k)]
        t["room"] = u8(max(16, sbp.sbp_layernorm_grad_workspace(T, D, B, k)))
        sbp.sbp_layernorm_grad(X([t["x"]] * k, T, D, sbp.BF16), None, B, vec(t["gamma"]), stat("mean"), stat("rstd"), X(t["dy"], T, D, sbp.F32),
                               X(t["dx"], T, D, sbp.F32), X(t["dgamma"], D, 1, sbp.F32), X(t["dbeta"], D, 1, sbp.F32), t["room"], k, stream)
    return t, step


def stands_for(torch, t, name, kind):
    """64-bit values of every shard of an 8-bit tensor of the step"""
    return [o8.dequantize(q.cpu().numpy(), s.cpu().numpy(), kind) for q, s in zip(t[name], t[name + ("s" if name == "y" else "_s")])]


def test_a_training_step_of_an_mlp_block():
    """Every operator's output against the 64-bit formula on its own stored inputs, along the whole step."""
    torch = torch_mod()
    t, step = mlp_step(torch, 1)
    step()
    sync()
    f = lambda v: v.double().cpu().numpy()  # noqa: E731
    k = 2
    x, gamma, beta = f(t["x"]), f(t["gamma"]), f(t["beta"])
    y, m, r = o8.layernorm(x, gamma, beta, 1e-5)
    y8 = stands_for(torch, t, "y", "e4m3")
    assert (y8[0] == y8[1]).all()
    close(y8[0], y, np.abs(y) * (U["e4m3"] + 1e-5) + o8.spread(t["ys"][0].cpu().numpy(), 256) * 2.0 ** -10 + 1e-5, "y")
    w1, w2 = stands_for(torch, t, "w1q", "e4m3"), stands_for(torch, t, "w2q", "e4m3")
    a8, h8 = stands_for(torch, t, "aq", "e4m3"), stands_for(torch, t, "hq", "e4m3")
    dz8, w2r, ht, dzt = stands_for(torch, t, "dzq", "e5m2"), stands_for(torch, t, "w2r", "e4m3"), stands_for(torch, t, "ht", "e4m3"), stands_for(torch, t, "dzt", "e5m2")
    da8, w1r = stands_for(torch, t, "daq", "e5m2"), stands_for(torch, t, "w1r", "e4m3")

    def product(got, p, q, what):
        want, total = p @ q, np.abs(p) @ np.abs(q)
        tol = p.shape[1] * U["f32"] * total
        if got.dtype == torch.bfloat16:
            tol = tol + 2.0 ** -11 * total + (np.abs(want) + total * 2.0 ** -11) * U["bf16"]
        close(f(got), want, tol + np.abs(want) * U["f32"], what)
    for i in range(k):
        product(t["a"][i], y8[i], w1[i].T, "a")
        product(t["zp"][i], h8[i], w2[i].T, "z")
        product(t["dh"][i], dz8[i], w2r[i].T, "dh")
        product(t["dw2"][i], ht[i], dzt[i].T, "dw2")
        product(t["dyp"][i], da8[i], w1r[i].T, "dy")
        close(f(t["h"][i]), o8.gelu(a8[i]), np.abs(o8.gelu(a8[i])) * (U["bf16"] * 1.001 + 3e-5) + 1e-30, "h")
        dh = f(t["dh"][i])
        want = dh * o8.gelu_slope(a8[i])
        close(f(t["da"][i]), want, np.abs(dh) * 5e-7 + np.abs(want) * U["bf16"] * 1.001, "da")
        dx, dg, db = o8.layernorm_grad(x, gamma, f(t["mean"][i]), f(t["rstd"][i]), f(t["dy"][i]))
        close(f(t["dx"][i]), dx, 1e-5 * (np.abs(dx) + np.sqrt((dx ** 2).mean())), "dx")
        close(f(t["dgamma"][i]), dg, 300 * U["f32"] * (np.abs(f(t["dy"][i])) * np.abs((x - m[:, None]) * r[:, None])).sum(0), "dgamma")
        close(f(t["dbeta"][i]), db, 300 * U["f32"] * np.abs(f(t["dy"][i])).sum(0), "dbeta")
    for n in ("dx", "dgamma", "dbeta", "z"):
        assert torch.equal(t[n][0], t[n][1])


def test_the_step_in_a_graph_and_on_a_stream():
    """Captured once, replayed on new inputs with eager work in between: bit for bit the eager result.  The capture runs on a stream of its own."""
    torch = torch_mod()
    t, step = mlp_step(torch, 2)
    names = ("a", "zp", "z", "dh", "da", "dw2", "dy", "dx", "dgamma", "dbeta", "y", "ys", "aq", "aq_s")
    step()
    sync()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n in range(4):
        t["x"].copy_(torch.randn(t["x"].shape, device="cuda").bfloat16())
        t["dz"].mul_(1.25)
        sync()
        graph.replay()
        sync()
        got = {m: [v.clone() for v in t[m]] for m in names}
        held = {m: t[m] for m in t}          # the graph's own buffers
        step()                                # eager, into new buffers
        sync()
        for m in names:
            for p, q in zip(got[m], t[m]):
                assert torch.equal(p.view(torch.uint8), q.view(torch.uint8)), (n, m)
        t.update(held)


def test_two_steps_at_once_on_two_streams():
    """Calls that overlap in time share nothing."""
    torch = torch_mod()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    steps = [mlp_step(torch, 3 + i, streams[i]) for i in range(2)]
    sync()
    want = []
    for (t, step), s in zip(steps, streams):
        with torch.cuda.stream(s):
            step()
        sync()
        want.append([v.clone() for n in ("dx", "dw2", "dgamma") for v in t[n]])
    for _ in range(5):
        for (t, step), s in zip(steps, streams):
            with torch.cuda.stream(s):
                step()
    sync()
    for (t, _), w in zip(steps, want):
        for p, q in zip([v for n in ("dx", "dw2", "dgamma") for v in t[n]], w):
            assert torch.equal(p, q)


# ------------------------------------------------------------------ offsets past 32 bits
def big_and_tail(rows, cols, dtype, tail, seed):
    """A [rows, cols] tensor whose elements lie past 2^31, and a copy of its last `tail` rows."""
    torch = torch_mod()
    x = torch.randn(rows, cols, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda", dtype=dtype)
    assert x.numel() > 2 ** 31
    return x, x[-tail:].clone()


def one(t, dtype, trans=0):
    rows, cols = (t.shape[1], t.shape[0]) if trans else t.shape
    return sbp.SbpTensor([t], rows, cols, dtype, trans)


def test_elementwise_operators_past_32_bits():
    """every element of an elementwise operator and every block's scale depend on a block alone: the last rows are what a small tensor gives, bit for bit"""
    torch = torch_mod()
    rows, cols, tail = 34000, 65536, 128 + 34000 % 128      # whole blocks where the blocks run along the rows
    x, xt = big_and_tail(rows, cols, torch.bfloat16, tail, 1)
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8, device="cuda")  # noqa: E731
    q, s, qt, st = u8(rows, cols), u8(rows, blocks(cols)), u8(tail, cols), u8(tail, blocks(cols))
    sbp.sbp_quantize(one(x, sbp.BF16), sbp.B, one(q, sbp.F8E4M3), sbp.SbpScales([s]), 1)
    sbp.sbp_quantize(one(xt, sbp.BF16), sbp.B, one(qt, sbp.F8E4M3), sbp.SbpScales([st]), 1)
    assert torch.equal(q[-tail:], qt) and torch.equal(s[-tail:], st) and bool(qt.any())
    y, yt = torch.zeros_like(x), torch.zeros_like(xt)
    sbp.sbp_dequantize(one(q, sbp.F8E4M3), sbp.SbpScales([s]), sbp.B, one(y, sbp.BF16), 1)
    sbp.sbp_dequantize(one(qt, sbp.F8E4M3), sbp.SbpScales([st]), sbp.B, one(yt, sbp.BF16), 1)
    assert torch.equal(y[-tail:], yt) and bool(yt.any())
    sbp.sbp_gelu_grad(one(q, sbp.F8E4M3), sbp.SbpScales([s]), sbp.B, one(x, sbp.BF16), one(y, sbp.BF16), 1)
    sbp.sbp_gelu_grad(one(qt, sbp.F8E4M3), sbp.SbpScales([st]), sbp.B, one(xt, sbp.BF16), one(yt, sbp.BF16), 1)
    assert torch.equal(y[-tail:], yt)
    t, ts = u8(cols, rows), u8(cols, blocks(rows))
    tt, tts = u8(cols, tail), u8(cols, blocks(tail))
    sbp.sbp_quantize(one(x, sbp.BF16), sbp.B, one(t, sbp.F8E4M3, 1), sbp.SbpScales([ts]), 1)
    sbp.sbp_quantize(one(xt, sbp.BF16), sbp.B, one(tt, sbp.F8E4M3, 1), sbp.SbpScales([tts]), 1)
    assert torch.equal(t[:, -tail:], tt) and torch.equal(ts[:, -blocks(tail):], tts)
    sbp.sbp_dequantize(one(t, sbp.F8E4M3, 1), sbp.SbpScales([ts]), sbp.B, one(y, sbp.BF16), 1)
    sbp.sbp_dequantize(one(tt, sbp.F8E4M3, 1), sbp.SbpScales([tts]), sbp.B, one(yt, sbp.BF16), 1)
    assert torch.equal(y[-tail:], yt)


def test_layernorm_past_32_bits():
    """a row of y, dx and the statistics depends on the row alone"""
    torch = torch_mod()
    rows, cols, tail = 140000, 16000, 5
    x, xt = big_and_tail(rows, cols, torch.bfloat16, tail, 2)
    out = []
    for a in (x, xt):
        n = a.shape[0]
        y, mean, rstd = torch.zeros_like(a), torch.zeros(n, 1, device="cuda"), torch.zeros(n, 1, device="cuda")
        q, s = torch.zeros(n, cols, dtype=torch.uint8, device="cuda"), torch.zeros(n, blocks(cols), dtype=torch.uint8, device="cuda")
        sbp.sbp_layernorm(one(a, sbp.BF16), sbp.B, None, None, 1e-5, one(y, sbp.BF16), None, one(mean, sbp.F32), one(rstd, sbp.F32), 1)
        sbp.sbp_layernorm(one(a, sbp.BF16), sbp.B, None, None, 1e-5, one(q, sbp.F8E5M2), sbp.SbpScales([s]), None, None, 1)
        dx, dg, db = torch.zeros_like(a), torch.zeros(cols, 1, device="cuda"), torch.zeros(cols, 1, device="cuda")
        need = sbp.sbp_layernorm_grad_workspace(n, cols, sbp.B, 1)
        room = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
        sbp.sbp_layernorm_grad(one(a, sbp.BF16), None, sbp.B, None, one(mean, sbp.F32), one(rstd, sbp.F32), one(y, sbp.BF16), one(dx, sbp.BF16),
                               one(dg, sbp.F32), one(db, sbp.F32), room, 1)
        out.append([v[-tail:].clone() for v in (y, mean, rstd, q, s, dx)])
        if n == rows:   # the sum over rows of xhat^2 but for dy's rounding: n, to sqrt(2 / 140000) = 0.004, 12 of which are 0.05
            assert bool((dg / rows - 1).abs().max() < 0.05)
    for a, b in zip(*out):
        assert torch.equal(a, b) and bool(a.any())


@pytest.mark.parametrize("rows,K,N", [(140000, 16000, 32), (34000, 128, 65536)])
def test_matmul_f8_past_32_bits(rows, K, N):
    """operands, and results, past 2^31 elements: the last rows against the 64-bit product of what they stand for"""
    torch = torch_mod()
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randint(0, 120, (rows, K), generator=g, device="cuda", dtype=torch.uint8)     # finite e4m3
    w = torch.randint(0, 120, (N, K), generator=g, device="cuda", dtype=torch.uint8) | 128 * torch.randint(0, 2, (N, K), generator=g, device="cuda", dtype=torch.uint8)
    sx = torch.randint(117, 122, (rows, blocks(K)), generator=g, device="cuda", dtype=torch.uint8)
    sw = torch.randint(117, 122, (N, blocks(K)), generator=g, device="cuda", dtype=torch.uint8)
    y = torch.zeros(rows, N, device="cuda", dtype=torch.bfloat16)
    assert max(x.numel(), y.numel()) > 2 ** 31
    sbp.sbp_matmul_f8(one(x, sbp.F8E4M3), sbp.SbpScales([sx]), sbp.B, one(w, sbp.F8E4M3, 1), sbp.SbpScales([sw]), sbp.B, one(y, sbp.BF16), sbp.B, 1)
    sync()
    a = o8.dequantize(x[-7:].cpu().numpy(), sx[-7:].cpu().numpy(), "e4m3")
    b = o8.dequantize(w.cpu().numpy(), sw.cpu().numpy(), "e4m3")
    want, total = a @ b.T, np.abs(a) @ np.abs(b).T
    tol = (K * U["f32"] + 2.0 ** -11) * total
    close(y[-7:].float().cpu().numpy().astype(np.float64), want, tol + (np.abs(want) + tol) * U["bf16"])


# ------------------------------------------------------------------ rows far from zero
@pytest.mark.parametrize("xk", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [1, 5, 64, 384, 512, 1000, 1024, 1001, 2048, 4095, 4096, 8192, 8200, 16384])
def test_layernorm_rows_of_equal_values(cols, xk):
    """A row of one value of bf16 (8 bits, so that sums of up to 2^16 of them are exact) has that value as its mean and no distance to it: y is beta, exactly."""
    rng = np.random.default_rng(cols)
    each = np.array([1000.0, 3008.0, -0.1015625, 1.0, 2.0 ** -20, -57344.0, 123.5])
    w = store(np.repeat(each[:, None], cols, 1), xk)
    assert (value(w) == each[:, None]).all()
    rows = len(each)
    gw, bw = (1 + 0.2 * rng.normal(size=(cols, 1))).astype(np.float32), (0.3 * rng.normal(size=(cols, 1))).astype(np.float32)
    y, mean, rstd = Buf(rows, cols, np.float32), Buf(rows, 1, np.float32), Buf(rows, 1, np.float32)
    sbp.sbp_layernorm(desc(up([w], xk), rows, cols, xk), sbp.B, desc(up([gw], "f32"), cols, 1, "f32"), desc(up([bw], "f32"), cols, 1, "f32"), 1e-5,
                      desc([y], rows, cols, "f32"), None, desc([mean], rows, 1, "f32"), desc([rstd], rows, 1, "f32"), 1)
    sync()
    np.testing.assert_array_equal(mean.host()[:, 0], each)
    np.testing.assert_array_equal(y.host(), np.repeat(bw.T, rows, 0))
    np.testing.assert_allclose(rstd.host()[:, 0], 1e-5 ** -0.5, rtol=2 * 2.0 ** -23)   # eps's rounding halved, the root's last place


@pytest.mark.parametrize("cols", [64, 1001, 4096, 16384])
@pytest.mark.parametrize("far,deviation", [(1000.0, 0.1), (-3000.0, 1.0), (10.0, 1.0)])
def test_layernorm_is_the_distance_to_its_mean(cols, far, deviation):
    """y = (x - mean) rstd gamma + beta of the mean and rstd that the call returns: a rounding of the distance, of its product with rstd and of the rest
    each, all relative to the distance, however far the row is from zero."""
    rng = np.random.default_rng(cols)
    x = (far + deviation * rng.normal(size=(9, cols))).astype(np.float32)
    gw, bw = (1 + 0.2 * rng.normal(size=(cols, 1))).astype(np.float32), (0.3 * rng.normal(size=(cols, 1))).astype(np.float32)
    y, mean, rstd = Buf(9, cols, np.float32), Buf(9, 1, np.float32), Buf(9, 1, np.float32)
    sbp.sbp_layernorm(desc(up([x], "f32"), 9, cols, "f32"), sbp.B, desc(up([gw], "f32"), cols, 1, "f32"), desc(up([bw], "f32"), cols, 1, "f32"), 1e-5,
                      desc([y], 9, cols, "f32"), None, desc([mean], 9, 1, "f32"), desc([rstd], 9, 1, "f32"), 1)
    sync()
    part = (x.astype(np.float64) - mean.host().astype(np.float64)) * rstd.host().astype(np.float64) * gw[:, 0].astype(np.float64)
    want = part + bw[:, 0]
    close(y.host().astype(np.float64), want, 2.001 * U["f32"] * np.abs(part) + 1.001 * U["f32"] * np.abs(want), "y")


# ------------------------------------------------------------------ NaN whose quiet bit is not set
@pytest.mark.parametrize("kind", ["e4m3", "e5m2"])
@pytest.mark.parametrize("xk,word", [("bf16", 0x7F81), ("bf16", 0xFFA0), ("bf16", 0x7FC0), ("f32", 0x7F800001), ("f32", 0xFFBFFFFF), ("f32", 0x7FC00000)])
@pytest.mark.parametrize("trans", [0, 1])
@pytest.mark.parametrize("gelu", [False, True])
def test_quantize_any_nan_leaves_its_block_alone(gelu, trans, xk, word, kind):
    """One NaN, quiet or signalling, and the block's largest number at every pair of places of eight neighbours: scale and values are those of the other
    127 (GeLU of the largest is that number itself).  Eight blocks of a kind side by side, so that none is gone through again for the sake of another's."""
    rng = np.random.default_rng(9)
    rows = 8 * 256
    v = rng.uniform(-1, 1, (rows, 128))
    case = np.arange(rows) // 8
    place, largest = case % 128, case // 16 % 8 + case % 128 // 8 * 8
    assert len(set(zip(place % 8, largest % 8))) == 64
    v[np.arange(rows), largest] = 300.0 + case
    w = store(v, xk).copy()
    clear = place != largest
    bits = w.view(np.uint32 if xk == "f32" else np.uint16)
    bits[np.arange(rows)[clear], place[clear]] = word
    with np.errstate(invalid="ignore"):
        v = value(w.view(NP[xk]))
    assert np.isnan(v).sum() == clear.sum()
    stored = np.ascontiguousarray(w.T) if trans else w
    x = up([stored], xk)
    q, sc = Buf(rows, 128, np.uint8), Buf(rows, 1, np.uint8)
    sbp.sbp_quantize(desc(x, *stored.shape, xk), sbp.B, desc([q], *stored.shape, kind, trans), sbp.SbpScales([sc]), 1, None, EPI[gelu])
    sync()
    want, wants = o8.quantize(v, kind)
    np.testing.assert_array_equal(sc.host(), wants)
    got, nan = q.host(), np.isnan(v)
    assert np.isnan(o8.decode_table(kind)[got[nan]]).all() and not np.isnan(o8.decode_table(kind)[got[~nan]]).any()
    same = v > 2 if gelu else ~nan
    np.testing.assert_array_equal(got[same], want[same])


# ------------------------------------------------------------------ every kind of tile, every element, on the GPU in 64 bits
#: M, K, N, devices, signature, result, aligned rows; 16s of rows of the tile that the sizes lead to on 256 compute units (asked of the choice itself on the
#: CPU); what the sizes are for
F8_TILES = [
    (4096, 2200, 8192, 1, "B", "bf16", True, 16),      # two tiles a workgroup, scales read in two parts, a cut block
    (4096, 2200, 8192, 1, "B", "f32", True, 16),
    (2048, 2100, 16384, 8, "S1", "bf16", True, 16),    # tiles of several devices one after another
    (4096, 513, 4096, 2, "P", "f32", True, 16),        # reductions of three and of two blocks
    (8000, 260, 4000, 2, "S0", "bf16", True, 16),      # a cut block of four elements
    (2000, 2200, 2000, 1, "B", "bf16", True, 8),
    (2000, 2200, 1990, 1, "B", "f32", True, 8),
    (777, 3001, 1501, 3, "P", "f32", True, 8),
    (2500, 383, 2500, 3, "P", "f32", True, 8),         # several tiles a workgroup, of devices with one block, the last one cut
    (2500, 385, 2500, 3, "P", "f32", True, 8),         # with one whole block and one element, and with one block
    (1111, 1531, 1777, 1, "B", "bf16", False, 8),      # through registers
    (1111, 1531, 1777, 1, "B", "f32", False, 8),
    (3000, 2201, 3000, 1, "B", "bf16", False, 8),      # several tiles a workgroup
    (2500, 385, 2500, 3, "P", "f32", False, 8),
]


def f8_pitches(k, aligned):
    """pitches of rows of k values and of their scales"""
    return (-(-k // 16) * 16 + 16, -(-blocks(k) // 4) * 4 + 4) if aligned else (k | 1, blocks(k))


def f8_on_the_gpu(M, K, N, k, sig, xk, wk, yk, aligned, gelu, seed):
    """Random codes of every finite value; scales from 2^-40 to 2^40 and three NaN an operand (moderate scales and no NaN with GeLU); what lies between and behind
    the rows is NaN, and no scale.  Every element against the 64-bit product on the same card.

    bf16 results: the instruction for 8 bits cuts the products of eight consecutive values at 2^-13 of the power of two that is the largest of their exponents'
    sums (subnormal numbers' being the smallest normal one's), so eight of them lose less than 2^-10 of it."""
    torch = torch_mod()
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=g, device="cuda", dtype=torch.int32).to(torch.uint8)  # noqa: E731
    table = {t: torch.from_numpy(o8.decode_table(t)).cuda() for t in (xk, wk)}

    parts_ = lambda n: [e - b for b, e in parts(n, k)]  # noqa: E731
    ld, lds = f8_pitches(max(parts_(K)) if sig == "P" else K, aligned)   # one pitch for all devices

    def operand(rows, cols, kind):
        v, s = (torch.full((rows * p,), 255, dtype=torch.uint8, device="cuda").view(rows, p) for p in (ld, lds))
        v[:, :cols] = rand(0, 120, rows, cols) | 128 * rand(0, 2, rows, cols)
        s[:, :blocks(cols)] = rand(118, 123, rows, blocks(cols)) if gelu else rand(87, 168, rows, blocks(cols))
        if not gelu:
            for r, c in ((rows // 3, 0), (rows - 1, cols - 1), (rows // 2, cols // 2)):
                v[r, c] = 255
        power = torch.exp2(s[:, :blocks(cols)].double() - 127).repeat_interleave(128, 1)[:, :cols]
        value_ = table[kind][v[:, :cols].long()]
        most = torch.nn.functional.pad(value_.abs().nan_to_num(0.0), (0, -cols % 8)).unflatten(1, (-1, 8)).amax(2).clamp(min=2.0 ** (-6 if kind == "e4m3" else -14))
        return v, s, value_ * power, torch.exp2(torch.floor(torch.log2(most))) * power[:, ::8]

    if sig == "P":
        x, w = [operand(M, n, xk) for n in parts_(K)], [operand(N, n, wk) for n in parts_(K)]
    else:
        x = [operand(n, K, xk) for n in parts_(M)] if sig == "S0" else [operand(M, K, xk)] * k
        w = [operand(n, K, wk) for n in parts_(N)] if sig == "S1" else [operand(N, K, wk)] * k
    ldy = max(o[0].shape[0] for o in w) + 3
    y = [torch.full((a[0].shape[0], ldy), -7.0, dtype=torch.float32 if yk == "f32" else torch.bfloat16, device="cuda") for a in x]
    a_sig, b_sig, y_sig = {"S0": (sbp.S(0), sbp.B, sbp.S(0)), "S1": (sbp.B, sbp.S(1), sbp.S(1)), "P": (sbp.S(1), sbp.S(0), sbp.P_SUM), "B": (sbp.B,) * 3}[sig]
    sbp.sbp_matmul_f8(desc([o[0] for o in x], M, K, xk, 0, ld), sbp.SbpScales([o[1] for o in x], lds), a_sig,
                      desc([o[0] for o in w], K, N, wk, 1, ld), sbp.SbpScales([o[1] for o in w], lds), b_sig, desc(y, M, N, yk, 0, ldy), y_sig, k, None, EPI[gelu])
    for i in range(k):
        xv, wv, n = x[i][2], w[i][2], w[i][2].shape[0]
        assert bool((y[i][:, n:] == -7).all())
        got, want, total = y[i][:, :n].double(), xv @ wv.T.contiguous(), xv.abs() @ wv.abs().T.contiguous()
        tol = xv.shape[1] * U["f32"] * total + (2.0 ** -10 * (x[i][3] @ w[i][3].T.contiguous()) if yk == "bf16" else 0.0)
        if gelu:
            want = 0.5 * want * torch.special.erfc(-want * 0.5 ** 0.5)
            tol = 1.13 * tol + 2.3e-5 * want.abs()
        nan = want.isnan()
        assert bool((got.isnan() == nan).all()) and int(nan.sum()) == (0 if gelu else 3 * n + 3 * got.shape[0] - 9)
        bad = ~nan & ~((got - want).abs() <= tol + (want.abs() + tol) * U[yk] + 1e-37)
        assert not bool(bad.any()), f"shard {i}: {int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}"


@pytest.mark.parametrize("M,K,N,k,sig,yk,aligned,tile", F8_TILES)
def test_matmul_f8_tiles_with_scales_far_apart(M, K, N, k, sig, yk, aligned, tile):
    f8_on_the_gpu(M, K, N, k, sig, "e4m3", "e4m3", yk, aligned, False, 21)


@pytest.mark.parametrize("xk,wk", [("e4m3", "e5m2"), ("e5m2", "e4m3"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("M,K,N,k,sig,yk,aligned,tile", [c for c in F8_TILES if not c[6]] + F8_TILES[:2] + F8_TILES[5:8])
def test_matmul_f8_tiles_of_either_type(M, K, N, k, sig, yk, aligned, tile, xk, wk):
    f8_on_the_gpu(M, K, N, k, sig, xk, wk, yk, aligned, False, 22)


@pytest.mark.parametrize("M,K,N,k,sig,yk,aligned,tile", [c for c in F8_TILES if c[4] != "P"])
def test_matmul_f8_tiles_with_gelu(M, K, N, k, sig, yk, aligned, tile):
    f8_on_the_gpu(M, K, N, k, sig, "e4m3", "e5m2", yk, aligned, True, 23)


@pytest.mark.parametrize("M,K,N", [(1, 260, 16), (300, 900, 272), (2000, 2200, 2000), (4096, 2200, 8192)])
def test_matmul_f8_the_most_that_an_eight_of_products_loses(M, K, N):
    """In every eight of the reduction 2^7 and -2^7 times the smallest subnormal number, 2^-9, whose exponent counts as -6, and six products below 2^(7 - 6 - 13):
    bf16 results may lose the six, which are 2^-8.6 of the products' magnitudes and all of the result, but less than 2^-10 2^(7 - 6).  fp32 results
    have them."""
    torch = torch_mod()
    kp, nb = -(-K // 16) * 16, -(-blocks(K) // 4) * 4
    place = torch.arange(kp, device="cuda")
    row = lambda first, second, rest: torch.where(place >= K, 0, torch.where(place % 8 == 0, first, torch.where(place % 8 == 1, second, rest))).to(torch.uint8)  # noqa: E731
    rx, rw = row(0x70, 0xF0, 0x07), row(0x01, 0x01, 0x08)
    x, w = rx.repeat(M, 1), rw.repeat(N, 1)
    one = lambda n: torch.full((n, nb), 127, dtype=torch.uint8, device="cuda")  # noqa: E731
    sx, sw = one(M), one(N)
    table = torch.from_numpy(o8.decode_table("e4m3")).cuda()
    p = table[rx.long()] * table[rw.long()]
    want, total = float(p.sum()), float(p.abs().sum())
    for yk, dt, tol in (("f32", torch.float32, K * U["f32"] * total), ("bf16", torch.bfloat16, -(-K // 8) * 2.0 ** -9 + K * U["f32"] * total + 2 * U["bf16"] * want)):
        y = torch.zeros(M, N, dtype=dt, device="cuda")
        sbp.sbp_matmul_f8(desc([x], M, K, "e4m3", 0, kp), sbp.SbpScales([sx], nb), sbp.B, desc([w], K, N, "e4m3", 1, kp), sbp.SbpScales([sw], nb), sbp.B,
                          desc([y], M, N, yk), sbp.B, 1)
        assert float((y.double() - want).abs().max()) <= tol, yk


def test_gelu_grad_of_fp32_is_as_good_as_its_roundings():
    """gelu' lies in -0.13 .. 1.13: four roundings (the tail's two products, the distance to 1, the sum) of numbers up to 1 are 2^-25 / sqrt 3 each, root mean
    square, 3.5e-8 together; half as much again for the exponential, the reciprocal and the fit would be 5.2e-8."""
    x = np.linspace(-4, 4, 1 << 20).astype(np.float32)[None]
    out = Buf(*x.shape, np.float32)
    sbp.sbp_gelu_grad(desc(up([x], "f32"), *x.shape, "f32"), None, sbp.B, desc(up([np.ones_like(x)], "f32"), *x.shape, "f32"), desc([out], *x.shape, "f32"), 1)
    sync()
    off = out.host().astype(np.float64) - o8.gelu_slope(x.astype(np.float64))
    assert np.sqrt((off ** 2).mean()) < 5.2e-8 and np.abs(off).max() < 5e-7
    # far out on the left what is left is a phi(a) and the tail, which a bf16 result still has to 2^-8 of itself
    far = out.host()[0] < 0
    far &= x[0] < -3
    assert (np.abs(off[0][far]) < 1e-4 * np.abs(o8.gelu_slope(x[0][far].astype(np.float64)))).all()


@pytest.mark.parametrize("yk", ["bf16", "f32"])
def test_gelu_of_infinities(yk):
    """0 on the left and infinity on the right, in every form: of values restored from 8 bits (e5m2 has infinities), and of a product's results"""
    x = np.zeros((3, 130), np.float32)
    x[0, [0, 64, 129]], x[1, 5], x[2, 7] = [np.inf, -np.inf, 3.0], -np.inf, np.nan
    q, sc, y = Buf(3, 130, np.uint8), Buf(3, 2, np.uint8), Buf(3, 130, NP[yk])
    dq, ds = desc([q], 3, 130, "e5m2"), sbp.SbpScales([sc])
    sbp.sbp_quantize(desc(up([x], "f32"), 3, 130, "f32"), sbp.B, dq, ds, 1)
    sbp.sbp_dequantize(dq, ds, sbp.B, desc([y], 3, 130, yk), 1, None, sbp.EPI_GELU)
    w = Buf(20, 130, np.uint8, 0, np.full((20, 130), 0x38, np.uint8))             # ones
    ws, p = Buf(20, 2, np.uint8, 0, np.full((20, 2), 127, np.uint8)), Buf(3, 20, NP[yk])
    x2 = x.copy()
    x2[0, 64] = 0.0
    q2, sc2 = Buf(3, 130, np.uint8), Buf(3, 2, np.uint8)
    dq2, ds2 = desc([q2], 3, 130, "e5m2"), sbp.SbpScales([sc2])
    sbp.sbp_quantize(desc(up([x2], "f32"), 3, 130, "f32"), sbp.B, dq2, ds2, 1)
    sbp.sbp_matmul_f8(dq2, ds2, sbp.B, desc([w], 130, 20, "e4m3", 1), sbp.SbpScales([ws]), sbp.B, desc([p], 3, 20, yk), sbp.B, 1, None, sbp.EPI_GELU)
    sync()
    got, want = value(y.host()), x.astype(np.float64)
    want[want == -np.inf] = 0.0
    keep = ~((want == 3.0))
    np.testing.assert_array_equal(got[keep], want[keep])
    got = value(p.host())
    assert (got[0] == np.inf).all() and (got[1] == 0).all() and np.isnan(got[2]).all()


# ------------------------------------------------------------------ the ends of what the calls allow
@pytest.mark.parametrize("which", ["gamma", "beta"])
@pytest.mark.parametrize("wk", ["f32", "bf16"])
def test_layernorm_with_one_weight(wk, which):
    rng = np.random.default_rng(31)
    x, v = (rng.normal(size=(5, 700))).astype(np.float32), store(rng.normal(size=(700, 1)), wk)
    d = desc(up([v], wk), 700, 1, wk)
    y = Buf(5, 700, np.float32)
    sbp.sbp_layernorm(desc(up([x], "f32"), 5, 700, "f32"), sbp.B, d if which == "gamma" else None, d if which == "beta" else None, 1e-5, desc([y], 5, 700, "f32"),
                      None, None, None, 1)
    sync()
    g, b = (value(v)[:, 0], 0.0) if which == "gamma" else (1.0, value(v)[:, 0])
    want, m, r = o8.layernorm(x.astype(np.float64), g, b, 1e-5)
    close(y.host().astype(np.float64), want, norm_tolerance(x.astype(np.float64), np.broadcast_to(g, 700), np.broadcast_to(b, 700), m, r) + np.abs(want) * U["f32"])


def test_layernorm_grad_of_no_rows_is_zero():
    og, ob = [Buf(300, 1, np.float32) for _ in range(2)], [Buf(300, 1, np.float32) for _ in range(2)]
    none = lambda cols, kind: sbp.SbpTensor([None, None], 0, cols, CODE[kind])  # noqa: E731
    assert sbp.sbp_layernorm_grad_workspace(0, 300, sbp.S(0), 2) == 0
    sbp.sbp_layernorm_grad(none(300, "bf16"), None, sbp.S(0), None, none(1, "f32"), none(1, "f32"), none(300, "bf16"), none(300, "bf16"), desc(og, 300, 1, "f32"),
                           desc(ob, 300, 1, "f32"), None, 2)
    sync()
    assert all((b.host() == 0).all() for b in og + ob)


@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("yk", ["bf16", "f32"])
def test_matmul_f8_of_no_reduction_is_zero(yk, gelu):
    none, s = sbp.SbpTensor([None], 70, 0, sbp.F8E4M3), sbp.SbpScales([None])
    y = Buf(70, 33, NP[yk], 40)
    sbp.sbp_matmul_f8(none, s, sbp.B, sbp.SbpTensor([None], 0, 33, sbp.F8E5M2, 1), s, sbp.B, desc([y], 70, 33, yk, 0, 40), sbp.B, 1, None, EPI[gelu])
    sync()
    assert (y.host() == 0).all()


@pytest.mark.parametrize("sig", ["S0", "S1", "B"])
def test_as_many_devices_as_there_may_be(sig):
    """64 for the elementwise operators, 32 for the others; more devices than rows or columns among them"""
    rng = np.random.default_rng(33)
    for rows, cols in ((50, 300), (130, 40), (200, 260)):
        w = store(rng.normal(size=(rows, cols)), "bf16")
        shards, k = split(w, sig, 64), 64
        x, dh = up(shards, "bf16"), up(shards, "bf16")
        q, sc = [Buf(*s.shape, np.uint8) for s in shards], [Buf(s.shape[0], blocks(s.shape[1]) if s.size else 0, np.uint8) for s in shards]
        y, da = [Buf(*s.shape, np.float32) for s in shards], [Buf(*s.shape, np.uint16) for s in shards]
        dq, ds = desc(q, rows, cols, "e4m3"), sbp.SbpScales(sc)
        sbp.sbp_quantize(desc(x, rows, cols, "bf16"), SIG[sig], dq, ds, k)
        sbp.sbp_dequantize(dq, ds, SIG[sig], desc(y, rows, cols, "f32"), k)
        sbp.sbp_gelu_grad(dq, ds, SIG[sig], desc(dh, rows, cols, "bf16"), desc(da, rows, cols, "bf16"), k)
        sync()
        for i, s in enumerate(shards):
            if not s.size:
                continue
            want, wants = o8.quantize(value(np.ascontiguousarray(s)), "e4m3")
            stands = o8.dequantize(want, wants, "e4m3")
            np.testing.assert_array_equal(q[i].host(), want)
            np.testing.assert_array_equal(y[i].host(), stands)
            grad = value(s) * o8.gelu_slope(stands)
            close(value(da[i].host()), grad, np.abs(value(s)) * 5e-7 + np.abs(grad) * 1.001 * U["bf16"] + 1e-38)


@pytest.mark.parametrize("sig,yk", [("S0", "bf16"), ("S1", "f32"), ("P", "f32"), ("B", "bf16")])
@pytest.mark.parametrize("M,K,N", [(20, 300, 20), (70, 40, 90), (300, 33 * 128, 260)])
def test_matmul_f8_on_32_devices(M, K, N, sig, yk):
    matmul_case(np.random.default_rng(34), M, K, N, 32, sig, "e4m3", "e5m2", yk)


@pytest.mark.parametrize("rows,cols", [(20, 600), (2000, 130)])
def test_layernorm_on_32_devices(rows, cols):
    test_layernorm(rows, cols, 32, "S0", "bf16", "e4m3", "f32")
    test_layernorm_grad(rows, cols, 32, "S0", "e4m3", "bf16", "bf16")


@pytest.mark.parametrize("xk,yk", [("f32", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("cols", [5, 100, 129])
def test_layernorm_grad_of_rows_whose_mean_times_rstd_overflows(cols, xk, yk):
    """rows of one large value: their elements are at no distance, and what is behind their end counts for nothing"""
    rng = np.random.default_rng(35)
    w = store(np.full((4, cols), 2.0 ** 120), xk)
    dy = store(rng.normal(size=(4, cols)), yk)
    mean, rstd = Buf(4, 1, np.float32), Buf(4, 1, np.float32)
    y, dx = Buf(4, cols, np.float32), Buf(4, cols, NP[yk])
    og, ob = Buf(cols, 1, np.float32), Buf(cols, 1, np.float32)
    x, room = desc(up([w], xk), 4, cols, xk), torch_mod().zeros(1 << 20, dtype=torch_mod().uint8, device="cuda")
    sbp.sbp_layernorm(x, sbp.B, None, None, 1e-5, desc([y], 4, cols, "f32"), None, desc([mean], 4, 1, "f32"), desc([rstd], 4, 1, "f32"), 1)
    sbp.sbp_layernorm_grad(x, None, sbp.B, None, desc([mean], 4, 1, "f32"), desc([rstd], 4, 1, "f32"), desc(up([dy], yk), 4, cols, yk), desc([dx], 4, cols, yk),
                           desc([og], cols, 1, "f32"), desc([ob], cols, 1, "f32"), room, 1)
    sync()
    assert (y.host() == 0).all() and (og.host() == 0).all()
    d, r = value(dy), float(rstd.host()[0, 0])
    want = r * (d - d.mean(1, keepdims=True))
    close(value(dx.host()), want, r * 16 * U["f32"] * (np.abs(d) + np.abs(d).mean(1, keepdims=True)) + np.abs(want) * 1.001 * U[yk], "dx")
