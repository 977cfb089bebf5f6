"""sbp_residual_norm and its gradient against the 64-bit forms of train_reference.py, whose bounds count the roundings of fp32; results in a narrower type have one
rounding more, U of the value."""
import itertools

import pytest
import torch

import paper_2110_15032_amd as sbp
import train_reference as ref
from train_harness import SIG, TYPE, Buf, Dev, U, close, column, normal, room, rounded, slices, split

pytestmark = pytest.mark.gpu
KIND = {"layer": (sbp.NORM_LAYER, ref.LAYER), "rms": (sbp.NORM_RMS, ref.RMS)}
TINY = 1e-37   # below it fp32 numbers are subnormal, and a relative bound says nothing


class Case:
    """Inputs on the host (as fp32 or bf16 hold them) and on k devices."""

    def __init__(self, rows, cols, k=1, sig="S0", x="f32", r="f32", y="f32", w="f32", post="layer", pre="layer", gate=True, alpha=0.75, eps=1e-5, pitch=0, bare=False, seed=0,
                 offset=0.0, size=1.0):
        self.__dict__.update(rows=rows, cols=cols, k=k, sig=sig, kx=x, kr=r, ky=y, kw=w, alpha=float(torch.tensor(alpha).float()), eps=float(torch.tensor(eps).float()), pitch=pitch)
        strong = 1.0 + 7.0 * (normal(cols, seed=seed + 50).abs() > 2.0)
        self.x = rounded(size * normal(rows, cols, seed=seed) * strong + offset, x)
        self.r = rounded(size * normal(rows, cols, seed=seed + 1) + offset, r)
        self.gate = rounded(0.5 + 0.3 * normal(cols, seed=seed + 2), w) if gate else None
        self.post = self._norm(post, bare, seed + 3)
        self.pre = self._norm(pre, bare, seed + 5)
        self.posts, self.pres = post, pre
        self.X, self.R = self.dev(self.x, x), self.dev(self.r, r)
        self.weights = {}

    def _norm(self, name, bare, seed):
        if not name:
            return None
        gamma, beta = rounded(1.0 + 0.2 * normal(self.cols, seed=seed), self.kw), rounded(0.3 * normal(self.cols, seed=seed + 1), self.kw)
        return ref.Norm(KIND[name][1], self.eps, None if bare else gamma, None if bare or name == "rms" else beta)

    def dev(self, data, kind, pitch=None):
        return Dev((self.rows, self.cols), kind, self.sig, self.k, self.pitch if pitch is None else pitch, data=data)

    def out(self, kind):
        return Dev((self.rows, self.cols), kind, self.sig, self.k, self.pitch and self.pitch + 1)

    def weight(self, data):
        if data is None:
            return None
        dev = column(self.cols, self.kw, "B", self.k, data, shared=True)
        self.weights[id(dev)] = dev
        return dev.desc

    def stat(self, data=None):
        return column(self.rows, "f32", self.sig, self.k, data)

    def norm(self, which, stats, grads=(None, None)):
        m, name = (self.post, self.posts) if which == 1 else (self.pre, self.pres)
        if m is None:
            return None
        d = lambda t: None if t is None else t.desc  # noqa: E731
        return sbp.SbpNorm(KIND[name][0], self.eps, self.weight(m.gamma), self.weight(m.beta), d(stats[0]) if name == "layer" else None, d(stats[1]), *(d(g) for g in grads))


def run_forward(c, stats=True):
    h, y = c.out(c.kr), c.out(c.ky) if c.pre else None
    st = {w: (c.stat(), c.stat()) if stats else (None, None) for w in (1, 2)}
    scales = None
    if c.pre and c.ky in ("e4m3", "e5m2"):
        blocks = (c.cols + 127) // 128
        scales = [Buf(b.rows, blocks, "u8", blocks + 3) for b in y.bufs]
    sbp.sbp_residual_norm(c.X.desc, SIG[c.sig], c.norm(1, st[1]), c.weight(c.gate), c.R.desc, c.alpha, h.desc, c.norm(2, st[2]), y.desc if y else None,
                          sbp.SbpScales(scales, blocks + 3) if scales else None, c.k)
    return h, y, scales, st


def check_forward(c, stats=True):
    h, y, scales, st = run_forward(c, stats)
    hs, ys = h.host(), y.host() if y else None
    for i, (x, r) in enumerate(zip(slices(c.x, c.sig, c.k), slices(c.r, c.sig, c.k))):
        if x.shape[0] == 0:
            continue
        want = ref.residual_norm(x, r, c.post, c.gate, c.alpha, c.pre)
        v, b = want["h"]
        close(hs[i], v, 1.01 * b + U[c.kr] * (v.abs() + b) + TINY, "h")
        if y and scales is None:
            v, b = want["y"]
            close(ys[i], v, 1.01 * b + U[c.ky] * (v.abs() + b) + TINY, "y")
        elif y:
            check8(ys[i], scales[i].host(), *want["y"], c.ky)
        if stats:
            for w, norm in ((1, c.post), (2, c.pre)):
                if norm is None:
                    continue
                for name, dev in zip(("mean", "rstd"), st[w]):
                    if name == "mean" and norm.kind == ref.RMS:
                        continue
                    v, b = want[f"{name}{w}"]
                    close(dev.host()[i], v, 1.01 * b + 2 * ref.E * v.abs() + TINY, f"{name}{w}")


def check8(codes, scales, value, bound, kind):
    """8 bits: nothing saturates, the scale is the smallest that fits (where the bound leaves that open, either), values are to half a step."""
    top = {"e4m3": 448.0, "e5m2": 57344.0}[kind]
    least = {"e4m3": 2.0 ** -10, "e5m2": 2.0 ** -17}[kind]      # half of the smallest step
    power = torch.exp2(scales.double() - 127)
    for j in range(scales.shape[1]):
        v, b = value[:, 128 * j:128 * (j + 1)], 1.01 * bound[:, 128 * j:128 * (j + 1)]
        p = power[:, j:j + 1]
        most, off = v.abs().amax(1, keepdim=True), b.amax(1, keepdim=True)
        assert bool((most - off <= top * p).all()) and bool(((most + off > top * p / 2) | (p <= 2.0 ** -127)).all())
        close(codes[:, 128 * j:128 * (j + 1)].double() * p, v, b + torch.maximum(U[kind] * (v.abs() + b), least * p), "y in 8 bits")


FORMS = [("layer", "layer"), ("rms", "rms"), ("", "layer"), ("", "rms"), ("rms", ""), ("layer", "rms"), ("layer", "")]
SIZES = [(1, 1), (3, 7), (5, 8), (4, 100), (7, 511), (9, 512), (5, 515), (3, 1024), (6, 1030), (5, 2048), (3, 2100), (4, 4096), (3, 4099), (3, 8192), (2, 8200), (3, 16384), (2, 16377)]


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("post,pre", FORMS[:5])
def test_forward_sizes(rows, cols, post, pre):
    i = SIZES.index((rows, cols))
    x, r, y, w = ("f32", "bf16")[i % 2], ("bf16", "f32")[i // 2 % 2], ("f32", "bf16", "e4m3", "e5m2")[i % 4], ("f32", "bf16")[i // 3 % 2]
    check_forward(Case(rows, cols, x=x, r=r, y=y, w=w, post=post, pre=pre, gate=i % 3 != 0, pitch=i % 4, seed=i))


@pytest.mark.parametrize("x,r,y", list(itertools.product(("f32", "bf16"), ("f32", "bf16"), ("f32", "bf16", "e4m3", "e5m2"))))
def test_forward_types(x, r, y):
    for cols, w in ((300, "f32"), (1000, "bf16"), (1500, "f32"), (3001, "bf16"), (5000, "f32"), (9001, "bf16")):
        check_forward(Case(5, cols, x=x, r=r, y=y, w=w, pitch=3))


@pytest.mark.parametrize("k,sig,rows", [(2, "B", 3), (3, "S0", 100), (8, "S0", 5), (9, "S0", 40), (32, "S0", 70)])
@pytest.mark.parametrize("post,pre", FORMS)
def test_forward_on_devices(k, sig, rows, post, pre):
    check_forward(Case(rows, 200, k=k, sig=sig, x="bf16", r="f32", y="bf16", post=post, pre=pre, pitch=2), stats=k != 8)


def test_forward_many_rows_and_no_weights():
    check_forward(Case(5000, 130, k=2, x="bf16", r="bf16", y="bf16", bare=True, gate=False, alpha=1.0))
    check_forward(Case(3000, 1100, x="bf16", r="bf16", y="e4m3", post="rms", pre="rms", bare=True))


def test_forward_rows_far_from_zero():
    """the distances to the mean, not the squares of the elements, make the variance"""
    check_forward(Case(6, 2000, offset=1000.0))
    check_forward(Case(6, 4096, offset=-300.0, size=0.01))
    check_forward(Case(3, 600, size=1e-18, eps=0.0))
    check_forward(Case(3, 600, size=1e15))


def test_forward_keeps_rows_apart():
    """NaN and infinity of a row stay in that row, and behind no row's end is anything read that counts"""
    c = Case(5, 1001, x="bf16", r="f32", y="bf16", pitch=5)
    bad = c.x.clone()
    bad[1, 3], bad[3, 1000] = float("nan"), float("inf")
    for buf, part in zip(c.X.bufs, slices(bad, "S0", 1)):
        buf.raw.fill_(0xFF)            # NaN between the rows
        buf.t.copy_(part)
    h, y, _, st = run_forward(c)
    ok = [0, 2, 4]
    want = ref.residual_norm(c.x, c.r, c.post, c.gate, c.alpha, c.pre)
    got_h, got_y = h.host()[0], y.host()[0]
    close(got_h[ok], want["h"][0][ok], (1.01 * want["h"][1] + U["f32"] * want["h"][0].abs() * 1.01)[ok] + TINY, "h")
    close(got_y[ok], want["y"][0][ok], (1.01 * want["y"][1] + U["bf16"] * (want["y"][0].abs() + want["y"][1]))[ok] + TINY, "y")
    assert bool(got_y[1].isnan().all()) and bool(got_y[3].isnan().any())


def test_no_rows():
    c = Case(0, 64, k=2)
    run_forward(c)
    h, y, _, _ = run_forward(Case(0, 64, k=2, pre=""))
    assert all(t.numel() == 0 for t in h.host())


# ---- the gradient --------------------------------------------------------------------------------
def check_grad(c, dh=True, wanted=("dgate", "dgamma1", "dbeta1", "dgamma2", "dbeta2"), seed=100):
    full = ref.residual_norm(c.x, c.r, c.post, c.gate, c.alpha, c.pre)
    f32 = lambda t: t.float().double()  # noqa: E731
    h = rounded(full["h"][0], c.kr)
    stats = [f32(full[name][0]) if name in full else None for name in ("mean1", "rstd1", "mean2", "rstd2")]
    dev_stats = [None if t is None else c.stat(t) for t in stats]
    gh = rounded(normal(c.rows, c.cols, seed=seed), c.kr) if dh else None
    gy = rounded(normal(c.rows, c.cols, seed=seed + 1), c.ky) if c.pre else None
    outs = {"dx": c.out(c.kx), "dr": c.out(c.kr)}
    have = ["dgate"] + (["dgamma1"] + (["dbeta1"] if c.posts == "layer" else []) if c.post else []) + (["dgamma2"] + (["dbeta2"] if c.pres == "layer" else []) if c.pre else [])
    outs.update({name: column(c.cols, "f32", "B", c.k) for name in have if name in wanted})
    n1 = c.norm(1, dev_stats[:2], [outs.get("dgamma1"), outs.get("dbeta1")])
    n2 = c.norm(2, dev_stats[2:], [outs.get("dgamma2"), outs.get("dbeta2")])
    H = c.dev(h, c.kr) if c.pre else None
    DH, DY = c.dev(gh, c.kr, 0) if dh else None, c.dev(gy, c.ky) if c.pre else None
    d = lambda t: None if t is None else t.desc  # noqa: E731
    work = room(sbp.sbp_residual_norm_grad_workspace(c.rows, c.cols, SIG[c.sig], c.k)) if len(outs) > 2 else None

    def call():
        sbp.sbp_residual_norm_grad(c.X.desc, SIG[c.sig], n1, c.weight(c.gate), c.alpha, d(H), n2, d(DH), d(DY), outs["dx"].desc, outs["dr"].desc, d(outs.get("dgate")), work, c.k)
    call()
    got = {name: t.host() for name, t in outs.items()}
    pick = lambda t, a, b: None if t is None else t[a:b]  # noqa: E731
    for i in range(c.k):
        a, b = split(c.rows, c.k)[i] if c.sig == "S0" else (0, c.rows)
        want = ref.residual_norm_grad(c.x[a:b], c.post, c.gate, c.alpha, h[a:b], c.pre, pick(gh, a, b), pick(gy, a, b), [pick(t, a, b) for t in stats])
        for name in outs:
            v, e = want[name]
            u = {"dx": U[c.kx], "dr": U[c.kr]}.get(name, 0.0)
            close(got[name][i].reshape(v.shape), v, 1.01 * e + u * (v.abs() + e) + TINY, name)
    call()                                                # the same bits every time
    for name, t in outs.items():
        assert all(torch.equal(p, q) for p, q in zip(t.host(), got[name])), name


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("post,pre", FORMS[:5])
def test_gradient_sizes(rows, cols, post, pre):
    i = SIZES.index((rows, cols))
    x, r, y, w = ("f32", "bf16")[i % 2], ("bf16", "f32")[i // 2 % 2], ("f32", "bf16")[i // 4 % 2], ("f32", "bf16")[i // 3 % 2]
    check_grad(Case(rows, cols, x=x, r=r, y=y, w=w, post=post, pre=pre, gate=i % 3 != 0, pitch=i % 4, seed=i), dh=i % 2 == 0 or not pre)


@pytest.mark.parametrize("x,r,y", list(itertools.product(("f32", "bf16"), repeat=3)))
def test_gradient_types(x, r, y):
    for cols, w in ((300, "f32"), (1000, "bf16"), (1500, "f32"), (3001, "bf16"), (5000, "f32"), (9001, "bf16")):
        check_grad(Case(7, cols, x=x, r=r, y=y, w=w, pitch=3))


@pytest.mark.parametrize("k,sig,rows", [(2, "B", 3), (3, "S0", 100), (8, "S0", 5), (9, "S0", 40), (32, "S0", 70)])
@pytest.mark.parametrize("post,pre", FORMS)
def test_gradient_on_devices(k, sig, rows, post, pre):
    check_grad(Case(rows, 200, k=k, sig=sig, x="bf16", r="f32", y="bf16", post=post, pre=pre, pitch=2), dh=k != 3 or not pre)


def test_gradient_many_rows():
    check_grad(Case(5000, 130, k=2, x="bf16", r="bf16", y="bf16"))
    check_grad(Case(2000, 600, x="bf16", r="f32", y="f32", post="rms", pre="rms"))
    check_grad(Case(1300, 2600, x="f32", r="f32", y="bf16", bare=True))
    check_grad(Case(700, 9000, x="bf16", r="bf16", y="bf16"))


@pytest.mark.parametrize("wanted", [(), ("dgate",), ("dgamma1", "dbeta2"), ("dbeta1",), ("dgamma2",)])
def test_gradient_of_some_weights(wanted):
    check_grad(Case(70, 300, k=2), wanted=wanted)
    check_grad(Case(70, 300, k=2, post=""), wanted=wanted)


def test_gradient_no_rows():
    check_grad(Case(0, 100, k=2))                         # sums of nothing are zero


def test_gradient_replayed_graph_beside_eager_calls():
    c = Case(300, 1000, k=2, x="bf16", r="bf16", y="bf16")
    full = ref.residual_norm(c.x, c.r, c.post, c.gate, c.alpha, c.pre)
    stats = [c.stat(full[name][0].float().double()) for name in ("mean1", "rstd1", "mean2", "rstd2")]
    dgate, dg1, db1, dg2, db2 = (column(c.cols, "f32", "B", 2) for _ in range(5))
    n1, n2 = c.norm(1, stats[:2], [dg1, db1]), c.norm(2, stats[2:], [dg2, db2])
    H, DY, DX, DR = c.dev(full["h"][0], "bf16"), c.dev(normal(300, 1000, seed=3), "bf16"), c.out("bf16"), c.out("bf16")
    gate, work = c.weight(c.gate), [room(sbp.sbp_residual_norm_grad_workspace(300, 1000, sbp.S(0), 2)) for _ in range(2)]
    outs = [DX, DR, dgate, dg1, db1, dg2, db2]

    def step(w):
        sbp.sbp_residual_norm_grad(c.X.desc, sbp.S(0), n1, gate, c.alpha, H.desc, n2, None, DY.desc, DX.desc, DR.desc, dgate.desc, w, 2)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        step(work[0])
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            step(work[0])
    for turn in range(3):
        for b in DY.bufs:
            b.t.mul_(-0.5)
        for o in outs:
            for b in o.bufs:
                b.t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        replayed = [[t.clone() for t in o.host()] for o in outs]
        step(work[1])
        torch.cuda.synchronize()
        for o, old in zip(outs, replayed):
            assert all(torch.equal(a, b) and float(a.abs().max()) > 0 for a, b in zip(o.host(), old))


def test_offsets_past_32_bits():
    """rows whose elements lie more than 2^31 elements behind the first"""
    rows, cols = 140001, 16384
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    r, h, y = x, torch.empty_like(x), torch.empty_like(x)
    x[-1] = torch.arange(cols, device="cuda") % 7 - 3
    d = lambda t: sbp.SbpTensor([t], rows, cols, sbp.BF16)  # noqa: E731
    rms = sbp.SbpNorm(sbp.NORM_RMS, 1e-5)
    sbp.sbp_residual_norm(d(x), sbp.B, None, None, d(r), 1.0, d(h), rms, d(y), None, 1)
    assert torch.equal(h[-1], 2 * x[-1])
    v = 2 * x[-1].double()
    close(y[-1].double().cpu(), (v / (v.square().mean() + 1e-5).sqrt()).cpu(), 1.01 * U["bf16"] * 3 * torch.ones(cols, dtype=torch.float64))
    assert not bool(h[:-1].any()) and not bool(y[:-1].any())
