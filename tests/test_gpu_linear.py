"""sbp_linear and the gradient of its epilogue against plain products in 64 bits.

Bounds.  A sum of K products in fp32, in any order and with steps of 2^-23 at worst, is within 2 (K + 64) E of the sum of their magnitudes (E = 2^-24; fp32 operands as
bf16 terms leave out less than 3 E of each, inside the 64).  GeLU: 2.2e-5 of its value in front of a rounding to bf16; in fp32 erfc's few units and the rounding of its
argument, which a^2 magnifies: (8 + 2 a^2) E.  Its slope is at most 1.13."""
import itertools

import pytest
import torch

import paper_2110_15032_amd as sbp
import train_reference as ref
from train_harness import SIG, Buf, Dev, U, close, column, normal, room, rounded, same, slices

pytestmark = pytest.mark.gpu
E = 2.0 ** -24
EPI = {False: sbp.EPI_NONE, True: sbp.EPI_GELU}
SIGS = {"S0": ("S0", "B", "S0", "B"), "S1": ("B", "S1", "S1", "S0"), "B": ("B", "B", "B", "B")}      # x, w, y, bias


class Layer:
    def __init__(self, m, kk, n, k=1, sig="B", x="bf16", y="bf16", bias="f32", residual="", pre="", gelu=False, x_trans=0, w_trans=1, pitch=0, seed=0):
        self.__dict__.update(m=m, kk=kk, n=n, k=k, sig=sig, kx=x, ky=y, kb=bias, kr=residual, kp=pre, gelu=gelu, pitch=pitch)
        sx, sw, self.sy, sb = SIGS[sig]
        self.sx, self.sw = SIG[sx], SIG[sw]
        self.x, self.w = rounded(normal(m, kk, seed=seed), x), rounded(normal(kk, n, seed=seed + 1, scale=max(kk, 1) ** -0.5), x)
        self.X = Dev((m, kk), x, sx, k, pitch, x_trans, self.x)
        self.W = Dev((kk, n), x, sw, k, pitch, w_trans, self.w)
        self.b = rounded(normal(n, seed=seed + 2), bias) if bias else None
        self.Bias = column(n, bias, sb, k, self.b, shared=sb == "B") if bias else None
        self.r = rounded(normal(m, n, seed=seed + 3), residual) if residual else None
        self.R = Dev((m, n), residual, self.sy, k, pitch and pitch + 1, data=self.r) if residual else None
        self.P = Dev((m, n), pre, self.sy, k, pitch and pitch + 2) if pre else None
        self.Y = Dev((m, n), y, self.sy, k, pitch)

    def run(self, stream=None):
        d = lambda t: None if t is None else t.desc  # noqa: E731
        sbp.sbp_linear(self.X.desc, self.sx, self.W.desc, self.sw, d(self.Bias), d(self.R), d(self.P), self.Y.desc, sbp.AUTO, self.k, stream, EPI[self.gelu])

    def want(self):
        x, w = self.x.cuda(), self.w.cuda()
        a, size = (x @ w).cpu(), (x.abs() @ w.abs()).cpu()
        da = 2 * (self.kk + 64) * E * size
        if self.b is not None:
            a = a + self.b
            da = da + 2 * E * (a.abs() + self.b.abs())
        y, dy = a, da
        if self.gelu:
            y = ref.gelu(a)
            dy = 1.13 * da + (2.2e-5 if self.ky == "bf16" else (8 + 2 * a ** 2) * E) * (y.abs() + 1.13 * da) + 1e-37
        if self.r is not None:
            y = y + self.r
            dy = dy + 2 * E * (y.abs() + self.r.abs())
        return a, da, y, dy

    def check(self):
        self.run()
        a, da, y, dy = self.want()
        cut = lambda t: slices(t, self.sy, self.k)  # noqa: E731
        for got, v, b in zip(self.Y.host(), cut(y), cut(dy)):
            close(got, v, 1.01 * b + U[self.ky] * (v.abs() + b), "y")
        if self.P:
            for got, v, b in zip(self.P.host(), cut(a), cut(da)):
                close(got, v, 1.01 * b + U[self.kp] * (v.abs() + b), "pre")


# one shape at least for every kernel that has the epilogue: single elements; waves splitting the reduction (32, 64, 128 rows); two groups of waves; 128 and 256 tiles;
# rows of any pitch with 64 and 128 tiles and with the reduction split
BF16 = [(5, 3, 7), (1, 4096, 300), (17, 520, 130), (33, 1024, 260), (1000, 520, 1500), (1000, 600, 1500), (1000, 200, 1500), (520, 64, 520), (4000, 104, 3900), (2304, 1024, 2048),
        (257, 777, 129), (1500, 77, 1500), (9, 4099, 100)]
FLAVOURS = [dict(y="bf16", bias="f32", residual="bf16", pre="bf16", gelu=True), dict(y="f32", bias="bf16", residual="f32", pre="f32", gelu=True),
            dict(y="bf16", bias="", residual="f32", gelu=False), dict(y="f32", bias="f32", pre="bf16", gelu=False)]


@pytest.mark.parametrize("shape", BF16)
@pytest.mark.parametrize("flavour", range(4))
def test_bf16(shape, flavour):
    i = BF16.index(shape)
    layouts = list(itertools.product((0, 1), (0, 1)))
    for x_trans, w_trans in layouts if min(shape) < 200 else layouts[(i + flavour) % 4::4] + [(0, 1)]:
        Layer(*shape, **FLAVOURS[flavour], x_trans=x_trans, w_trans=w_trans, seed=i).check()


@pytest.mark.parametrize("shape", [(5, 3, 7), (8, 300, 1000), (200, 300, 200), (1000, 100, 1000), (2100, 60, 2100), (2100, 300, 2100), (2600, 300, 2600), (65, 1001, 131)])
@pytest.mark.parametrize("flavour", range(4))
def test_f32(shape, flavour):
    i = shape[0] + flavour
    layouts = list(itertools.product((0, 1), (0, 1)))
    for x_trans, w_trans in layouts if min(shape) < 100 else layouts[i % 4::4]:
        Layer(*shape, x="f32", **FLAVOURS[flavour], x_trans=x_trans, w_trans=w_trans, seed=i).check()


@pytest.mark.parametrize("shape", [(130, 264, 200), (37, 1032, 77), (300, 96, 515), (1300, 80, 1290)])
@pytest.mark.parametrize("pitch", [1, 3, 8])
@pytest.mark.parametrize("x", ["bf16", "f32"])
def test_pitches(shape, pitch, x):
    for x_trans, w_trans in itertools.product((0, 1), (0, 1)):
        Layer(*shape, x=x, y=("bf16", "f32")[pitch % 2], residual="bf16", pre="f32", gelu=pitch == 3, x_trans=x_trans, w_trans=w_trans, pitch=pitch).check()


@pytest.mark.parametrize("m", [1, 2, 3, 4])
@pytest.mark.parametrize("kk,n", [(1, 9000), (7, 40), (512, 64), (1000, 1504), (1500, 130), (4099, 100), (520, 9001)])
@pytest.mark.parametrize("x", ["bf16", "f32"])
def test_a_few_rows(m, kk, n, x):
    """the weight in rows or in columns, whole pieces and cut ones, one wave a row or several"""
    for w_trans, pitch in ((1, 0), (1, 1), (0, 0), (0, 3)):
        Layer(m, kk, n, x=x, residual="bf16" if m % 2 else "", pre="f32", gelu=m > 2, w_trans=w_trans, pitch=pitch).check()


@pytest.mark.parametrize("m", [5, 15, 16, 17, 31, 32])
@pytest.mark.parametrize("kk,n", [(1, 40), (7, 16), (8, 17), (127, 130), (128, 64), (2047, 300), (2048, 65), (2200, 1000), (4099, 15), (9000, 257)])
def test_up_to_thirty_two_rows(m, kk, n):
    """pieces of the reduction for some of the waves, for all, and for some again, whole and cut; rows at any alignment"""
    for pitch in (0, 1, 8):
        Layer(m, kk, n, residual="bf16" if m % 2 else "", pre="f32", gelu=m > 16, pitch=pitch).check()
    Layer(m, kk, n, 3, "S1", pitch=5).check()
    Layer(m, kk, n, 20, "S0", y="f32", residual="f32").check()


def test_one_row_with_many_columns():
    for w_trans, pitch, x in ((0, 0, "bf16"), (0, 1, "bf16"), (1, 0, "f32"), (0, 0, "f32")):
        Layer(1, 300, 20000, x=x, residual="f32", gelu=True, w_trans=w_trans, pitch=pitch).check()
        Layer(1, 2050, 17000, 3, "S1", x=x, w_trans=w_trans, pitch=pitch).check()
    Layer(2, 4096, 16500, residual="f32", gelu=True).check()               # past the caches


@pytest.mark.parametrize("m,k", [(3, 4), (1, 2), (5, 8), (2, 40)])
@pytest.mark.parametrize("x", ["bf16", "f32"])
def test_fewer_rows_than_devices(m, k, x):
    """devices without rows, whose x, residual, pre and y are null"""
    for w_trans, kk, n in ((1, 461, 1189), (1, 1500, 130), (1, 300, 9000), (0, 300, 20000), (0, 40, 64), (0, 777, 130)):
        Layer(m, kk, n, k, "S0", x=x, residual="f32", pre="bf16", gelu=kk == 300, w_trans=w_trans, pitch=3).check()


@pytest.mark.parametrize("k,sig,m,n", [(2, "B", 30, 100), (3, "S0", 100, 70), (8, "S0", 5, 64), (3, "S1", 50, 100), (8, "S1", 1, 2048), (9, "S1", 20, 180), (20, "S0", 70, 40), (64, "S1", 3, 640)])
@pytest.mark.parametrize("x", ["bf16", "f32"])
def test_on_devices(k, sig, m, n, x):
    for kk in (40, 640):
        Layer(m, kk, n, k, sig, x=x, residual="f32", pre="bf16", gelu=True, w_trans=kk % 3 == 1).check()
        Layer(m, kk, n, k, sig, x=x, y="f32", bias="bf16").check()


@pytest.mark.parametrize("shape", [(1, 1, 1), (3, 0, 5), (0, 8, 4), (4, 8, 0), (1, 512, 1), (2, 33, 9), (129, 8, 1), (1, 7, 129)])
@pytest.mark.parametrize("x", ["bf16", "f32"])
def test_smallest(shape, x):
    for gelu in (False, True):
        Layer(*shape, x=x, y="f32", residual="f32", pre="f32", gelu=gelu).check()
        Layer(*shape, x=x, gelu=gelu).check()


@pytest.mark.parametrize("y", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(5, 3, 16), (200, 64, 520), (4, 1024, 64), (1000, 600, 1500)])
def test_gelu_of_infinities_and_nan(shape, y):
    t = Layer(*shape, y=y, residual="f32", gelu=True)
    inf, nan = float("inf"), float("nan")
    t.Bias.bufs[0].t[:3, 0] = torch.tensor([-inf, inf, nan], device="cuda")
    t.run()
    got = t.Y.host()[0]
    assert torch.equal(got[:, 0], rounded(t.r, y)[:, 0]) and bool((got[:, 1] == inf).all()) and bool(got[:, 2].isnan().all())
    assert bool(got[:, 3:].isfinite().all())


def test_a_graph_replays_the_layer_on_new_inputs():
    t = Layer(300, 520, 200, 2, "S1", residual="bf16", pre="bf16", gelu=True)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        t.run()
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            t.run()
    for _ in range(3):
        t.X.bufs[0].t.mul_(-0.5)
        for b in t.Y.bufs + t.P.bufs:
            b.t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in t.Y.host() + t.P.host()]
        t.run()
        assert all(torch.equal(a, b) and float(a.abs().max()) > 0 for a, b in zip(t.Y.host() + t.P.host(), got))


def test_results_past_two_to_the_31_elements():
    """the last rows of results, pre-activations and a residual whose offsets need more than 32 bits"""
    m, n, kk = 33000, 66000, 16
    x = torch.zeros(m, kk, dtype=torch.bfloat16, device="cuda")
    w = torch.zeros(n, kk, dtype=torch.bfloat16, device="cuda")
    x[-2:, 0], w[-3:, 0] = 2.0, 3.0
    res = torch.zeros(m, n, dtype=torch.bfloat16, device="cuda")
    res[-1, -3:] = 1.0
    pre, y = torch.empty_like(res), torch.empty_like(res)
    d = lambda t, r, c, tr=0: sbp.SbpTensor([t], r, c, sbp.BF16, tr)  # noqa: E731
    sbp.sbp_linear(d(x, m, kk), sbp.B, d(w, kk, n, 1), sbp.B, None, d(res, m, n), d(pre, m, n), d(y, m, n), sbp.AUTO, 1)
    assert int(pre.count_nonzero()) == 6 and int(y.count_nonzero()) == 6
    assert bool((pre[-2:, -3:] == 6).all()) and bool((y[-1, -3:] == 7).all()) and bool((y[-2, -3:] == 6).all())


@pytest.mark.parametrize("w_trans", [0, 1])
def test_one_row_with_more_columns_than_a_grid_of_the_fast_kernels(w_trans):
    n = 2 ** 28 + 2 ** 12 + 37
    x = torch.tensor([[1.0, 2.0]], dtype=torch.bfloat16, device="cuda")
    w = (torch.arange(2 * n, device="cuda", dtype=torch.int32) % 61).to(torch.bfloat16)      # whole numbers, whose sums bf16 holds
    w = w.view(n, 2) if w_trans else w.view(2, n)
    y = torch.full((1, n), float("nan"), dtype=torch.bfloat16, device="cuda")
    d = lambda t, r, c, tr=0: sbp.SbpTensor([t], r, c, sbp.BF16, tr)  # noqa: E731
    sbp.sbp_linear(d(x, 1, 2), sbp.B, d(w, 2, n, w_trans), sbp.B, None, None, None, d(y, 1, n), sbp.AUTO, 1)
    a, b = (w[:, 0], w[:, 1]) if w_trans else (w[0], w[1])
    assert torch.equal(y[0], a + 2 * b)


# ---- the epilogue's gradient ----------------------------------------------------------------------
def check_grad(rows, cols, k=1, sig="B", y="bf16", pre="bf16", gelu=True, pitch=0, seed=0):
    dy = rounded(normal(rows, cols, seed=seed), y)
    Scales = None
    if not gelu:
        a, A = None, None
    elif pre in ("f32", "bf16"):
        a = rounded(2.0 * normal(rows, cols, seed=seed + 1), pre)
        A = Dev((rows, cols), pre, sig, k, pitch, data=a)
    else:
        code = rounded(100.0 * normal(rows, cols, seed=seed + 1), pre)
        A = Dev((rows, cols), pre, sig, k, pitch, data=code)
        cut = slices(code, sig, k)
        blocks = [(c.shape[1] + 127) // 128 for c in cut]
        gen = torch.Generator().manual_seed(seed)
        bytes_ = [torch.randint(119, 122, (c.shape[0], n), generator=gen, dtype=torch.uint8) for c, n in zip(cut, blocks)]
        if sig == "B":
            bytes_ = bytes_[:1] * k
        parts = [c * torch.exp2(e.double() - 127)[:, torch.arange(c.shape[1]) // 128] for c, e in zip(cut, bytes_)]
        a = parts[0] if sig == "B" else torch.cat(parts, 0 if sig == "S0" else 1)
        Scales = sbp.SbpScales([Buf(e.shape[0], e.shape[1], "u8", max(blocks) + 3, e) for e in bytes_], max(blocks) + 3)
    DY = Dev((rows, cols), y, sig, k, pitch and pitch + 1, data=dy)
    DA = Dev((rows, cols), y, sig, k, pitch) if gelu else None
    DB = column(cols, "f32", {"S0": "B", "S1": "S0", "B": "B"}[sig], k)
    work = room(sbp.sbp_linear_grad_workspace(rows, cols, SIG[sig], k))
    d = lambda t: None if t is None else t.desc  # noqa: E731

    def call():
        sbp.sbp_linear_grad(DY.desc, SIG[sig], d(A), Scales, d(DA), DB.desc, work, k, None, EPI[gelu])
    call()
    slope = ref.gelu_slope(a) if gelu else torch.ones_like(dy)
    da = dy * slope
    off = dy.abs() * (5e-7 if y == "bf16" else 3e-7) + 2 * E * da.abs() if gelu else torch.zeros_like(dy)
    got, sums = (DA.host() if gelu else []), [t.clone() for t in DB.host()]
    for t, v, b in zip(got, slices(da, sig, k), slices(off, sig, k)):
        close(t, v, 1.01 * b + U[y] * (v.abs() + b) + 1e-37, "da")
    for t, v, b in zip(sums, slices(da, sig, k), slices(off, sig, k)):
        close(t[:, 0], v.sum(0), 1.01 * (b.sum(0) + (v.shape[0] + 16) * E * v.abs().sum(0)) + 1e-37, "dbias")
    call()
    assert all(same(p, q) for p, q in zip(DB.host(), sums))


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (3, 8), (31, 255), (32, 256), (33, 257), (100, 1000), (1000, 130), (5000, 64), (70, 5001), (0, 40)])
@pytest.mark.parametrize("y,pre,gelu", [("bf16", "bf16", True), ("f32", "f32", True), ("f32", "bf16", True), ("bf16", "f32", True), ("bf16", "e4m3", True), ("f32", "e5m2", True),
                                         ("bf16", "", False), ("f32", "", False)])
def test_gradient(rows, cols, y, pre, gelu):
    check_grad(rows, cols, y=y, pre=pre, gelu=gelu, pitch=rows % 4)


@pytest.mark.parametrize("k,sig,rows,cols", [(2, "B", 50, 100), (3, "S0", 100, 300), (8, "S0", 5, 64), (8, "S1", 300, 1024), (3, "S1", 40, 100), (9, "S0", 400, 20), (64, "S1", 10, 640)])
@pytest.mark.parametrize("gelu", [False, True])
def test_gradient_on_devices(k, sig, rows, cols, gelu):
    check_grad(rows, cols, k, sig, gelu=gelu)
    check_grad(rows, cols, k, sig, y="f32", pre="e4m3", gelu=gelu, pitch=1)


def test_gradient_of_long_columns():
    check_grad(40000, 200, y="f32", pre="f32")
    check_grad(40000, 300, k=2, sig="S0", gelu=False)
