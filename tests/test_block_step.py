"""A training step of an MLP block by the operators together: forward, backward, the weights' gradients summed over the devices and clipped, in two layouts.

rows:    h = r + gate1 x;  n = norm1(h);  h2 = gelu(n W1 + b1) W2 + b2 + h.  Activations S(0), weights B, weights' gradients P(sum).
columns: the same n, gathered;  z = gelu(n W1 + b1) W2, W1 S(1), W2 S(0), z P(sum), scattered to S(0);  h2 = 0.9 h + gate2 rms(z).

On the GPU every call's results are compared with the formulas in 64 bits of what the calls before it left in memory, so that a bound holds one call's roundings
alone; that the formulas, chained like this, are the gradient is shown on the CPU against automatic differentiation.  Sums of n products in
fp32 in any order, the devices' among them, are within 2 (n + 64) E of the sum of their magnitudes."""
import math

import pytest
import torch

import paper_2110_15032_amd as sbp
import train_reference as ref
from train_harness import CODE, SIG, Dev, U, close, column, normal, room, rounded, same

E = 2.0 ** -24
TINY = 1e-37
EPS = 2.0 ** -17
ALPHA2 = float(torch.tensor(0.9).float())


def weights(d, n, layout, kind):
    w = {"gate1": 0.5 + 0.2 * normal(d, seed=1), "gamma1": 1.0 + 0.2 * normal(d, seed=2), "beta1": 0.2 * normal(d, seed=3), "W1": normal(d, n, seed=4, scale=d ** -0.5),
         "b1": 0.3 * normal(n, seed=5), "W2": normal(n, d, seed=6, scale=n ** -0.5)}
    if layout == "rows":
        w["b2"] = 0.3 * normal(d, seed=7)
    else:
        w["gate2"], w["gamma2"] = 0.7 + 0.2 * normal(d, seed=8), 1.0 + 0.2 * normal(d, seed=9)
    return {name: rounded(v, kind) for name, v in w.items()}


@pytest.mark.parametrize("layout", ["rows", "columns"])
def test_the_chain_is_the_gradient(layout):
    m, d, n = 7, 12, 20
    w = weights(d, n, layout, "f32")
    leaves = {name: v.clone().requires_grad_() for name, v in w.items()}
    x, r, dh2 = (normal(m, d, seed=s) for s in (20, 21, 22))
    x_, r_ = x.clone().requires_grad_(), r.clone().requires_grad_()
    L = leaves
    h = r_ + L["gate1"] * x_
    v = h - h.mean(1, keepdim=True)
    y = v * (v.square().mean(1, keepdim=True) + EPS).rsqrt() * L["gamma1"] + L["beta1"]
    u = torch.nn.functional.gelu(y @ L["W1"] + L["b1"])
    z = u @ L["W2"]
    h2 = z + L["b2"] + h if layout == "rows" else ALPHA2 * h + L["gate2"] * (z * (z.square().mean(1, keepdim=True) + EPS).rsqrt() * L["gamma2"])
    h2.backward(dh2)

    got = {}
    norm1 = ref.Norm(ref.LAYER, EPS, w["gamma1"], w["beta1"])
    f1 = ref.residual_norm(x, r, None, w["gate1"], 1.0, norm1)
    y, a = f1["y"][0], f1["y"][0] @ w["W1"] + w["b1"]
    u = ref.gelu(a)
    if layout == "rows":
        dz = dh = dh2
        got["b2"] = dz.sum(0)
    else:
        norm2 = ref.Norm(ref.RMS, EPS, w["gamma2"])
        z = u @ w["W2"]
        f2 = ref.residual_norm(z, f1["h"][0], norm2, w["gate2"], ALPHA2, None)
        b2 = ref.residual_norm_grad(z, norm2, w["gate2"], ALPHA2, None, None, dh2, None, (None, f2["rstd1"][0], None, None))
        dz, dh, got["gate2"], got["gamma2"] = b2["dx"][0], b2["dr"][0], b2["dgate"][0], b2["dgamma1"][0]
    da = dz @ w["W2"].T * ref.gelu_slope(a)
    got["W2"], got["W1"], got["b1"] = u.T @ dz, y.T @ da, da.sum(0)
    b1 = ref.residual_norm_grad(x, None, w["gate1"], 1.0, f1["h"][0], norm1, dh, da @ w["W1"].T, (None, None, f1["mean2"][0], f1["rstd2"][0]))
    got["gate1"], got["gamma1"], got["beta1"] = b1["dgate"][0], b1["dgamma2"][0], b1["dbeta2"][0]
    assert got.keys() == leaves.keys()
    for name, g in got.items():
        assert torch.allclose(g, leaves[name].grad, rtol=1e-10, atol=1e-10), name
    assert torch.allclose(b1["dx"][0], x_.grad, rtol=1e-10, atol=1e-10) and torch.allclose(b1["dr"][0], r_.grad, rtol=1e-10, atol=1e-10)


class Step:
    """The buffers of a step on k devices, its calls, and what they have to give."""

    def __init__(self, layout, kind, k, m, d, n, pitch):
        self.__dict__.update(layout=layout, kind=kind, k=k, m=m, d=d, n=n, pitch=pitch)
        self.rows = layout == "rows"
        self.w = weights(d, n, layout, kind)
        s1, s2 = ("B", "B") if self.rows else ("S1", "S0")
        self.W = {}
        for name, v in self.w.items():
            sig = {"W1": s1, "W2": s2, "b1": "B" if self.rows else "S0"}.get(name, "B")
            self.W[name] = Dev(v.shape, kind, sig, k, pitch, data=v) if v.dim() == 2 else column(v.shape[0], kind, sig, k, v)
        act = lambda cols, sig="S0", t=kind, data=None: Dev((m, cols), t, sig, k, pitch, data=data)  # noqa: E731
        self.X, self.R, self.DH2 = (act(d, data=rounded(normal(m, d, seed=s), kind)) for s in (20, 21, 22))
        su = "S0" if self.rows else "S1"
        self.H, self.Y, self.H2 = act(d), act(d), act(d)
        self.A, self.U, self.DU, self.DA = (act(n, su) for _ in range(4))
        stat = lambda: column(m, "f32", "S0", k)  # noqa: E731
        self.mean1, self.rstd1 = stat(), stat()
        self.DX, self.DR = act(d), act(d)
        vec = lambda size, sig="B": column(size, "f32", sig, k)  # noqa: E731
        mat = lambda a, b, sig="B": Dev((a, b), "f32", sig, k, 0)  # noqa: E731
        self.G, self.sigs = {}, {}                                     # as the backward calls leave them: P(sum) but where the layout says else
        for name, v in self.w.items():
            sig = "P" if self.rows else {"W1": "S1", "W2": "S0", "b1": "S0"}.get(name, "P")
            self.sigs[name] = sig
            self.G[name] = (mat if v.dim() == 2 else vec)(*v.shape, "B" if sig == "P" else sig)
        self.S = {name: (mat if v.dim() == 2 else vec)(*v.shape) if self.sigs[name] == "P" else self.G[name] for name, v in self.w.items()}   # summed
        self.C = {name: (mat if v.dim() == 2 else vec)(*v.shape, "B" if self.sigs[name] == "P" else self.sigs[name]) for name, v in self.w.items()}   # clipped
        self.squares, self.norm = vec(1), vec(1)
        self.DN = act(d, t=kind if self.rows else "f32")
        if not self.rows:
            # boxing takes dense rows
            dense = lambda sig, t: Dev((m, d), t, sig, k, 0)  # noqa: E731
            self.Y, self.YB = dense("S0", kind), dense("B", kind)
            self.ZP, self.Z, self.rstd2 = dense("B", "f32"), dense("S0", "f32"), stat()
            self.DZ, self.DZB, self.DH = dense("S0", "f32"), dense("B", kind), act(d)
            self.DNP, self.DN = dense("B", "f32"), dense("S0", "f32")
        lst = [self.S[name] for name in self.w]
        how = [SIG["B" if s == "P" else s] for s in self.sigs.values()]
        self.list, self.out = sbp.SbpList([t.desc for t in lst], how), sbp.SbpList([self.C[name].desc for name in self.w], how)
        self.rooms()

    def rooms(self):
        sn = sbp.S(0) if self.rows else sbp.S(1)
        self.work = {"norm": room(sbp.sbp_residual_norm_grad_workspace(self.m, self.d, sbp.S(0), self.k)), "linear": room(sbp.sbp_linear_grad_workspace(self.m, self.n, sn, self.k)),
                     "bias": room(sbp.sbp_linear_grad_workspace(self.m, self.d, sbp.S(0), self.k)), "squares": room(sbp.sbp_square_sum_workspace(self.list, self.k))}

    def turned(self, t):
        return sbp.SbpTensor(t.bufs, t.shape[1], t.shape[0], CODE[t.kind], 1, t.pitch)

    def run(self):
        k, W, G, s0, s1, b, p = self.k, self.W, self.G, sbp.S(0), sbp.S(1), sbp.B, sbp.P_SUM
        norm1 = sbp.SbpNorm(sbp.NORM_LAYER, EPS, W["gamma1"].desc, W["beta1"].desc, self.mean1.desc, self.rstd1.desc, G["gamma1"].desc, G["beta1"].desc)
        sbp.sbp_residual_norm(self.X.desc, s0, None, W["gate1"].desc, self.R.desc, 1.0, self.H.desc, norm1, self.Y.desc, None, k)
        if self.rows:
            sbp.sbp_linear(self.Y.desc, s0, W["W1"].desc, b, W["b1"].desc, None, self.A.desc, self.U.desc, s0, k, epilogue=sbp.EPI_GELU)
            sbp.sbp_linear(self.U.desc, s0, W["W2"].desc, b, W["b2"].desc, self.H.desc, None, self.H2.desc, s0, k)
            sbp.sbp_linear_grad(self.DH2.desc, s0, None, None, None, G["b2"].desc, self.work["bias"], k)
            sbp.sbp_matmul(self.turned(self.U), s1, self.DH2.desc, s0, G["W2"].desc, p, k)
            sbp.sbp_matmul(self.DH2.desc, s0, self.turned(W["W2"]), b, self.DU.desc, s0, k)
            sbp.sbp_linear_grad(self.DU.desc, s0, self.A.desc, None, self.DA.desc, G["b1"].desc, self.work["linear"], k, epilogue=sbp.EPI_GELU)
            sbp.sbp_matmul(self.turned(self.Y), s1, self.DA.desc, s0, G["W1"].desc, p, k)
            sbp.sbp_matmul(self.DA.desc, s0, self.turned(W["W1"]), b, self.DN.desc, s0, k)
        else:
            norm2 = sbp.SbpNorm(sbp.NORM_RMS, EPS, W["gamma2"].desc, None, None, self.rstd2.desc, G["gamma2"].desc)
            sbp.sbp_boxing(self.Y.desc, s0, self.YB.desc, b, k)
            sbp.sbp_linear(self.YB.desc, b, W["W1"].desc, s1, W["b1"].desc, None, self.A.desc, self.U.desc, s1, k, epilogue=sbp.EPI_GELU)
            sbp.sbp_matmul(self.U.desc, s1, W["W2"].desc, s0, self.ZP.desc, p, k)
            sbp.sbp_boxing(self.ZP.desc, p, self.Z.desc, s0, k)
            sbp.sbp_residual_norm(self.Z.desc, s0, norm2, W["gate2"].desc, self.H.desc, ALPHA2, self.H2.desc, None, None, None, k)
            sbp.sbp_residual_norm_grad(self.Z.desc, s0, norm2, W["gate2"].desc, ALPHA2, None, None, self.DH2.desc, None, self.DZ.desc, self.DH.desc, G["gate2"].desc, self.work["norm"], k)
            (sbp.sbp_boxing if self.kind == "f32" else sbp.sbp_boxing_cast)(self.DZ.desc, s0, self.DZB.desc, b, k)
            sbp.sbp_linear(self.turned(self.U), s0, self.DZB.desc, b, None, None, None, G["W2"].desc, s0, k)   # fp32 of bf16, as the P(sum) gradients are
            sbp.sbp_matmul(self.DZB.desc, b, self.turned(W["W2"]), s1, self.DU.desc, s1, k)
            sbp.sbp_linear_grad(self.DU.desc, s1, self.A.desc, None, self.DA.desc, G["b1"].desc, self.work["linear"], k, epilogue=sbp.EPI_GELU)
            sbp.sbp_linear(self.turned(self.YB), b, self.DA.desc, s1, None, None, None, G["W1"].desc, s1, k)
            sbp.sbp_matmul(self.DA.desc, s1, self.turned(W["W1"]), s0, self.DNP.desc, p, k)
            sbp.sbp_boxing(self.DNP.desc, p, self.DN.desc, s0, k)
        dh = self.DH2 if self.rows else self.DH
        sbp.sbp_residual_norm_grad(self.X.desc, s0, None, W["gate1"].desc, 1.0, self.H.desc, norm1, dh.desc, self.DN.desc, self.DX.desc, self.DR.desc, G["gate1"].desc, self.work["norm"], k)
        for name, sig in self.sigs.items():
            if sig == "P":
                sbp.sbp_boxing(G[name].desc, p, self.S[name].desc, b, k)
        sbp.sbp_square_sum(self.list, self.squares.desc, self.work["squares"], k)
        sbp.sbp_clip(self.list, self.squares.desc, p, 1.5, self.out, self.norm.desc, k)

    def results(self):
        devs = [self.H, self.Y, self.H2, self.A, self.U, self.DA, self.DX, self.DR, self.norm, *self.S.values(), *self.C.values()]
        return [t for dev in devs for t in dev.host()]

    def check(self):
        def whole(dev):
            parts = dev.host()
            if dev.sig == "B":
                assert all(same(t, parts[0]) for t in parts)
                return parts[0]
            return torch.cat(parts, 0 if dev.sig == "S0" else 1)

        def like(dev, value, bound, what):
            close(whole(dev), value, 1.01 * bound + U[dev.kind] * (value.abs() + bound) + TINY, what)

        def product(x, y):
            return x @ y, 2 * (x.shape[1] + 64) * E * (x.abs() @ y.abs())

        w, rows = self.w, self.rows
        x, r, dh2 = whole(self.X), whole(self.R), whole(self.DH2)
        norm1 = ref.Norm(ref.LAYER, EPS, w["gamma1"], w["beta1"])
        f1 = ref.residual_norm(x, r, None, w["gate1"], 1.0, norm1)
        like(self.H, *f1["h"], "h")
        like(self.Y, *f1["y"], "n")
        stats = whole(self.mean1), whole(self.rstd1)
        for got, (v, b), what in zip(stats, (f1["mean2"], f1["rstd2"]), ("mean", "rstd")):
            close(got, v, 1.01 * b + 2 * E * v.abs() + TINY, what)
        h, y = whole(self.H), whole(self.Y)
        v, b = product(y, w["W1"])
        a, da = v + w["b1"], b + 2 * E * (v.abs() + w["b1"].abs() + b)
        like(self.A, a, da, "pre")
        gelu = ref.gelu(a)
        like(self.U, gelu, 1.13 * da + (2.2e-5 if self.kind == "bf16" else (8 + 2 * a ** 2) * E) * (gelu.abs() + 1.13 * da), "gelu")
        pre, u = whole(self.A), whole(self.U)
        z, bz = product(u, w["W2"])
        if rows:
            h2 = z + w["b2"] + h
            like(self.H2, h2, bz + 4 * E * (z.abs() + w["b2"].abs() + h.abs()), "h2")
            dz, dh = dh2, dh2
            like(self.S["b2"], dz.sum(0)[:, None], (self.m + 16) * E * dz.abs().sum(0)[:, None], "b2")
        else:
            assert same(whole(self.YB), y)
            like(self.Z, z, bz, "z")
            z = whole(self.Z)
            norm2 = ref.Norm(ref.RMS, EPS, w["gamma2"])
            f2 = ref.residual_norm(z, h, norm2, w["gate2"], ALPHA2, None)
            like(self.H2, *f2["h"], "h2")
            b2 = ref.residual_norm_grad(z, norm2, w["gate2"], ALPHA2, None, None, dh2, None, (None, whole(self.rstd2), None, None))
            like(self.DZ, *b2["dx"], "dz")
            like(self.DH, *b2["dr"], "dh")
            for name, key in (("gate2", "dgate"), ("gamma2", "dgamma1")):
                like(self.S[name], b2[key][0][:, None], b2[key][1][:, None], name)
            assert same(whole(self.DZB), rounded(whole(self.DZ), self.kind))
            dz, dh = whole(self.DZB), whole(self.DH)
        like(self.S["W2"], *product(u.T, dz), "W2")
        like(self.DU, *product(dz, w["W2"].T), "du")
        du = whole(self.DU)
        v = du * ref.gelu_slope(pre)
        off = du.abs() * (5e-7 if self.kind == "bf16" else 3e-7) + 2 * E * v.abs()
        like(self.DA, v, off, "da")
        like(self.S["b1"], v.sum(0)[:, None], (off.sum(0) + (self.m + 16) * E * v.abs().sum(0))[:, None], "b1")
        da = whole(self.DA)
        like(self.S["W1"], *product(y.T, da), "W1")
        like(self.DN, *product(da, w["W1"].T), "dn")
        b1 = ref.residual_norm_grad(x, None, w["gate1"], 1.0, h, norm1, dh, whole(self.DN), (None, None, *stats))
        like(self.DX, *b1["dx"], "dx")
        like(self.DR, *b1["dr"], "dr")
        for name, key in (("gate1", "dgate"), ("gamma1", "dgamma2"), ("beta1", "dbeta2")):
            like(self.S[name], b1[key][0][:, None], b1[key][1][:, None], name)
        grads = {name: whole(t) for name, t in self.S.items()}
        norm = math.sqrt(sum(float((g ** 2).sum()) for g in grads.values()))
        got = whole(self.norm)
        close(got, torch.full_like(got, norm), torch.full_like(got, 1.01 * ((self.k + 1) / 2 + 1) * E * norm), "norm")
        factor = min(1.0, 1.5 / norm)
        for name, t in self.C.items():
            v = grads[name] * factor
            like(t, v, ((self.k + 1) / 2 + 2) * E * v.abs(), "clipped " + name)
        assert factor < 1.0


CASES = [("rows", "f32", 1, 9, 24, 40, 0), ("rows", "bf16", 2, 130, 96, 256, 8), ("rows", "f32", 3, 77, 100, 301, 1), ("columns", "bf16", 4, 130, 256, 512, 8), ("columns", "f32", 3, 50, 101, 130, 1),
         ("columns", "bf16", 8, 5, 64, 128, 0)]


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_step(case):
    step = Step(*case)
    step.run()
    step.check()


@pytest.mark.gpu
@pytest.mark.parametrize("case", [CASES[1], CASES[3]], ids=lambda c: "-".join(map(str, c)))
def test_step_in_a_graph(case):
    step = Step(*case)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step.run()
        stream.synchronize()
        kept = step.work
        with torch.cuda.graph(graph, stream=stream):
            step.run()
    step.rooms()                          # the eager calls have workspaces of their own
    for turn in range(3):
        for dev in (step.X, step.DH2):
            for b in dev.bufs:
                b.t.mul_(-0.75)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        replayed = step.results()
        for dev in (step.H, step.Y, step.A, step.U, step.DX, step.norm, *step.C.values()):
            for b in dev.bufs:
                b.t.zero_()
        step.run()
        torch.cuda.synchronize()
        assert all(same(a, b) for a, b in zip(step.results(), replayed)), turn
    step.check()
    assert kept
