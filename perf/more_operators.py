"""Performance cases of what a training step of an MLP block has around its products: the product with bias, activation and
residual in its epilogue, the norms behind and in front of a block with its gate and residual scale, their gradients, and the
norm of all gradients with their clipping.

`op` names the operator, `k` the number of logical devices (shard buffers in one GPU's memory), `sig` how the activations (for
`clip`: the gradients) lie on them: "S0" rows split, "S1" columns split, "B" one copy.

  linear       y = act(x w + bias) + residual; `pre`: x w + bias is kept for the backward pass
  linear_grad  da = dy * gelu'(pre), and the sum of da over the rows (without `gelu`: of dy), the bias' gradient
  norms        h = alpha r + gate * norm1(x), y = norm2(h); either norm ("layer", "rms") may be missing (""), and y is then
  norms_grad   its gradients: dx, dr, and those of gate and of both norms' weights, one partial sum for every device
  clip         the norm of a list of tensors, and all of them times min(1, max_norm / norm)

Rows lie `pad` elements apart rounded up (0: back to back).
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
SIZE = {"f32": 4, "bf16": 2, "e4m3": 1}
#: 8 bits: one power of two for 128 consecutive values; the largest value of e4m3 is 0.875 * 2^9
BLOCK, TOP = 128, 9
EPS = 1e-5


def listed():
    return [
        # decoding: one token through the column-parallel first product of an MLP block, the weight is the traffic
        dict(name="linear one token", op="linear", k=8, sig="S1", M=1, K=4096, N=16384, x="bf16", y="bf16", weights="bf16", w_trans=True, gelu=True, pre=False, residual="",
             pad=16),
        # training in fp32 on a last, uneven batch of a layer whose sizes divide nothing
        dict(name="linear odd", op="linear", k=3, sig="S0", M=777, K=1000, N=1501, x="f32", y="f32", weights="f32", w_trans=False, gelu=False, pre=False, residual="f32", pad=0),
        # the first product of the MLP block at its full size, its pre-activation kept
        dict(name="linear up", op="linear", k=8, sig="S1", M=8192, K=4096, N=16384, x="bf16", y="bf16", weights="f32", w_trans=False, gelu=True, pre=True, residual="", pad=16),
        # the second product, data-parallel, onto the residual stream
        dict(name="linear down", op="linear", k=8, sig="S0", M=8192, K=16384, N=4096, x="bf16", y="bf16", weights="f32", w_trans=True, gelu=False, pre=False, residual="bf16", pad=16),
        # backward of the activation and the bias, a small fp32 layer on an uneven batch
        dict(name="linear gradient odd", op="linear_grad", k=3, sig="S0", rows=1767, cols=1001, y="f32", pre="f32", gelu=True, pad=0),
        # backward of the MLP block's activation and first bias
        dict(name="linear gradient", op="linear_grad", k=8, sig="S1", rows=8192, cols=16384, y="bf16", pre="bf16", gelu=True, pad=16),
        # one token between two blocks: latency
        dict(name="norms one token", op="norms", k=1, sig="B", rows=1, cols=4096, x="bf16", r="bf16", y="bf16", weights="bf16", post="", pre="layer", gate=True, alpha=1.0,
             stats=False, pad=0),
        # between two blocks in training, an fp32 residual stream
        dict(name="norms", op="norms", k=8, sig="S0", rows=8192, cols=4096, x="bf16", r="f32", y="bf16", weights="f32", post="rms", pre="rms", gate=True, alpha=0.9, stats=True,
             pad=16),
        # training in fp32 on an uneven batch of a width that divides nothing
        dict(name="norms gradient odd", op="norms_grad", k=3, sig="S0", rows=1767, cols=1001, x="f32", r="f32", y="f32", weights="f32", post="layer", pre="layer", gate=True, alpha=1.0,
             dh=True, pad=0),
        # data-parallel training in bf16
        dict(name="norms gradient", op="norms_grad", k=8, sig="S0", rows=16384, cols=4096, x="bf16", r="bf16", y="bf16", weights="bf16", post="layer", pre="layer", gate=True, alpha=1.0,
             dh=True, pad=16),
        # the gradients of a small model, 72 tensors on two devices: latency
        dict(name="clip small", op="clip", k=2, sig="S1", width=64, inner=256, layers=12, x="f32", y="f32", max_norm=1.0, pad=0),
        # sharded optimizer state: bf16 gradients of 2^28 parameters into fp32
        dict(name="clip large", op="clip", k=8, sig="S0", width=4096, inner=16384, layers=2, x="bf16", y="f32", max_norm=1.0, pad=16),
    ]


def _size(rng, lo, hi, step=1):
    """Spread over the logarithm of lo .. hi, a multiple of step."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(step, n // step * step)


def draw(rng):
    op = rng.choice(["linear", "linear", "linear_grad", "norms", "norms_grad", "clip"])
    k = rng.choice([1, 2, 3, 4, 8])
    pad = rng.choice([0, 16, 16, 64])
    wide = ["f32", "bf16", "bf16"]
    if op == "linear":
        sig = rng.choice(["S0", "S1"])
        step = rng.choice([1, 1, 8, 64])
        x = rng.choice(["bf16", "bf16", "bf16", "f32"])
        most = 8192 * 4096 * 16384 // (16 if x == "f32" else 1)
        while True:
            m, kk, n = _size(rng, 1, 8192), _size(rng, 64, 16384, step), _size(rng, 64, 16384, step)
            if m * kk * n <= most:
                break
        n = -(-n // k) * k if sig == "S1" else n
        return dict(op=op, k=k, sig=sig, M=m, K=kk, N=n, x=x, y=rng.choice([x, x, "f32"]), weights=rng.choice(["f32", "bf16"]), w_trans=rng.random() < 0.5, gelu=rng.random() < 0.5,
                    pre=rng.random() < 0.4, residual=rng.choice(["", "f32", "bf16"]), pad=pad)
    if op == "clip":
        while True:
            width, inner, layers = _size(rng, 32, 4096), _size(rng, 64, 16384), _size(rng, 1, 24)
            if width * inner * layers <= 4096 * 16384 * 2:
                break
        sig = rng.choice(["S0", "S1", "B"])
        k = min(k, 3) if sig == "B" else k
        return dict(op=op, k=k, sig=sig, width=width, inner=inner, layers=layers, x=rng.choice(["f32", "bf16"]), y=rng.choice(["f32", "bf16"]), max_norm=rng.choice([0.1, 1.0, 1.0]),
                    pad=pad)
    while True:
        rows, cols = _size(rng, 1, 32768), _size(rng, 64, 16384, rng.choice([1, 8, 64]))
        if rows * cols <= 8192 * 8192:
            break
    if op == "linear_grad":
        sig = rng.choice(["S0", "S1"])
        cols = -(-cols // k) * k if sig == "S1" else cols
        return dict(op=op, k=k, sig=sig, rows=rows, cols=cols, y=rng.choice(wide), pre=rng.choice(wide), gelu=rng.random() < 0.7, pad=pad)
    post, pre = rng.choice([("", "layer"), ("", "rms"), ("layer", "layer"), ("rms", "rms"), ("rms", ""), ("layer", "rms")])
    c = dict(op=op, k=k, sig="S0", rows=rows, cols=cols, x=rng.choice(wide), r=rng.choice(wide), weights=rng.choice(["f32", "bf16"]), post=post, pre=pre, gate=rng.random() < 0.6,
             alpha=rng.choice([1.0, 1.0, 0.8]), pad=pad)
    if op == "norms":
        return dict(c, y=rng.choice(["bf16", "f32", "e4m3"]), stats=rng.random() < 0.7)
    return dict(c, y=rng.choice(wide), dh=pre == "" or rng.random() < 0.8)


# ---- shapes and buffers -------------------------------------------------------------------------
def _share(n, k):
    """Sizes of the balanced split: the first n mod k devices hold one more."""
    return [n // k + (i < n % k) for i in range(k)]


def _up(n, step):
    return -(-n // step) * step if step else n


def _rows(shape, dtype, pad):
    """A buffer whose rows lie a multiple of `pad` elements apart."""
    return torch.zeros(*shape[:-1], _up(shape[-1], pad), dtype=dtype, device="cuda")[..., : shape[-1]]


def _split_rows(shape, dtype, k, pad):
    """k buffers for the shares of the rows, each with a start of its own."""
    return [_rows((m, shape[-1]), dtype, pad) for m in _share(shape[0], k)]


def _on_devices(shape, kind, c):
    """The local tensors of an activation: k row shares, k column shares (of equal width), or one copy."""
    if c["sig"] == "S0":
        return _split_rows(shape, TYPES[kind], c["k"], c["pad"])
    if c["sig"] == "S1":
        return [_rows((shape[0], shape[1] // c["k"]), TYPES[kind], c["pad"]) for _ in range(c["k"])]
    return [_rows(shape, TYPES[kind], c["pad"])]


def _parts(whole, c):
    if c["sig"] == "S0":
        return whole.split(_share(whole.shape[0], c["k"]))
    return whole.chunk(c["k"], 1) if c["sig"] == "S1" else [whole]


def _layout(c):
    """Shapes and splits of the gradients that `clip` works on: every layer's two weights, their biases, and a norm's weights.
    Split: the axis, or None where every device has a copy."""
    w, n = c["width"], c["inner"]
    if c["sig"] == "S1":   # column-parallel, then row-parallel, the rest on every device
        layer = [((w, n), 1), ((n, 1), 0), ((n, w), 0), ((w, 1), None), ((w, 1), None), ((w, 1), None)]
    else:
        axis = 0 if c["sig"] == "S0" else None
        layer = [((w, n), axis), ((n, 1), axis), ((n, w), axis), ((w, 1), axis), ((w, 1), axis), ((w, 1), axis)]
    return layer * c["layers"]


def _local_shapes(shape, axis, k):
    if axis is None:
        return [shape] * k
    return [(m, shape[1]) if axis == 0 else (shape[0], m) for m in _share(shape[axis], k)]


def _buckets(c, dtype):
    """One buffer for all gradients of every device, and every tensor's parts in them, which start 8 elements apart or a multiple of
    it.  What lies between them stays zero."""
    parts, size = [], [0] * c["k"]
    for shape, axis in _layout(c):
        shapes = _local_shapes(shape, axis, c["k"])
        pitch = _up(max(n for _, n in shapes), c["pad"]) if shape[1] > 1 else 1   # vectors lie back to back
        parts.append([(size[i], m, n, pitch) for i, (m, n) in enumerate(shapes)])
        size = [_up(size[i] + m * pitch, 8) for i, (m, _) in enumerate(shapes)]
    buckets = [torch.zeros(n, dtype=dtype, device="cuda") for n in size]
    return buckets, [[b[at : at + m * pitch].view(m, pitch)[:, :n] for b, (at, m, n, pitch) in zip(buckets, part)] for part in parts]


# ---- the operators in their plain form ----------------------------------------------------------
def _narrow(x):
    """x in fp32 to e4m3 values and scales, blocks along the last axis."""
    n = x.shape[-1]
    b = torch.nn.functional.pad(x, (0, -n % BLOCK)).unflatten(-1, (-1, BLOCK))
    m, e = torch.frexp(b.abs().amax(-1))
    e = torch.where(m == 0, -127, e - TOP + (m > 0.875).int()).clamp(min=-127)
    values = torch.ldexp(b, -e.unsqueeze(-1)).float().to(TYPES["e4m3"]).flatten(-2)[..., :n]
    return values, (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _gelu(x):
    return 0.5 * x * (1.0 + torch.erf(x * math.sqrt(0.5)))


def _gelu_slope(x):
    return 0.5 * (1.0 + torch.erf(x * math.sqrt(0.5))) + x * torch.exp(-0.5 * x * x) * (1.0 / math.sqrt(2.0 * math.pi))


def _standard(x, kind):
    """Distances to the mean (RMS: to 0) over their root mean square, the mean and 1 / that root."""
    mean = x.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(x[:, :1])
    rstd = torch.rsqrt((x - mean).square().mean(-1, keepdim=True) + EPS)
    return (x - mean) * rstd, mean, rstd


def _standard_grad(xhat, rstd, g, kind):
    d = g - xhat * (g * xhat).mean(-1, keepdim=True)
    return rstd * (d - g.mean(-1, keepdim=True) if kind == "layer" else d)


def _weight(s, name, otherwise):
    return s[name].float() if name in s else torch.full((s["case"]["cols"],), otherwise, device="cuda")


def _sum_rows(t):
    return t.sum(0, dtype=torch.float64).float()


def _plain(s):
    c = s["case"]
    op, k = c["op"], c["k"]
    if op == "clip":
        total = torch.zeros((), dtype=torch.float64, device="cuda")
        for shards, (_, axis) in zip(s["grads"], _layout(c)):
            for t in shards if axis is not None else shards[:1]:   # a copy counts once
                total = total + t.double().square().sum()
        norm = total.sqrt()
        factor = torch.where(norm > c["max_norm"], c["max_norm"] / norm, torch.ones_like(norm)).float()
        return [(t.float() * factor).to(TYPES[c["y"]]) for t in s["buckets"]], [norm.float()] * k
    if op == "linear":
        if c["sig"] == "S0":
            x, w, bias = s["x"], [s["w"][0]] * k, [s["bias"][0]] * k
        else:
            x, w, bias = [s["x"][0]] * len(s["w"]), s["w"], s["bias"]
        pre, out = [], []
        for i in range(len(w)):
            a = torch.matmul(x[i].float(), w[i].float().T if c["w_trans"] else w[i].float()) + bias[i].float()
            y = _gelu(a) if c["gelu"] else a
            if c["residual"]:
                y = y + s["residual"][i].float()
            pre.append(a.to(TYPES[c["x"]]))
            out.append(y.to(TYPES[c["y"]]))
        return [out, pre] if c["pre"] else [out]
    if op == "linear_grad":
        out, sums = [], []
        for i in range(len(s["dy"])):
            da = s["dy"][i].float()
            if c["gelu"]:
                da = da * _gelu_slope(s["pre"][i].float())
            out.append(da.to(TYPES[c["y"]]))
            sums.append(_sum_rows(da))
        return [out, sums] if c["gelu"] else [sums]
    one, zero = (lambda name: _weight(s, name, 1.0)), (lambda name: _weight(s, name, 0.0))
    gate = one("gate")
    if op == "norms":
        hs, ys, scales, stats = [], [], [], []
        for x, r in zip(s["x"], s["r"]):
            t = x.float()
            if c["post"]:
                xhat, mean, rstd = _standard(t, c["post"])
                t = xhat * one("gamma1") + zero("beta1")
                stats += [mean, rstd] if c["post"] == "layer" else [rstd]
            h = c["alpha"] * r.float() + gate * t
            hs.append(h.to(TYPES[c["r"]]))
            if c["pre"]:
                xhat, mean, rstd = _standard(h, c["pre"])
                y = xhat * one("gamma2") + zero("beta2")
                stats += [mean, rstd] if c["pre"] == "layer" else [rstd]
                if c["y"] == "e4m3":
                    y, e = _narrow(y)
                    scales.append(e)
                ys.append(y.to(TYPES[c["y"]]))
        return [hs] + ([ys] if c["pre"] else []) + ([scales] if scales else []) + ([[t.flatten() for t in stats]] if c["stats"] else [])
    outs = {name: [] for name in _gradients(c)}
    for i, x in enumerate(s["x"]):
        dh = s["dh"][i].float() if c["dh"] else torch.zeros(x.shape, device="cuda")
        if c["pre"]:
            rstd, dy = s["rstd2"][i][:, None], s["dy"][i].float()
            h = s["h"][i].float()
            hhat = (h - s["mean2"][i][:, None] if c["pre"] == "layer" else h) * rstd
            dh = dh + _standard_grad(hhat, rstd, dy * one("gamma2"), c["pre"])
            outs["dgamma2"].append(_sum_rows(dy * hhat))
            if c["pre"] == "layer":
                outs["dbeta2"].append(_sum_rows(dy))
        outs["dr"].append((c["alpha"] * dh).to(TYPES[c["r"]]))
        dt, t = gate * dh, x.float()
        if c["post"]:
            rstd = s["rstd1"][i][:, None]
            xhat = (t - s["mean1"][i][:, None] if c["post"] == "layer" else t) * rstd
            t = xhat * one("gamma1") + zero("beta1")
            outs["dgamma1"].append(_sum_rows(dt * xhat))
            if c["post"] == "layer":
                outs["dbeta1"].append(_sum_rows(dt))
            dx = _standard_grad(xhat, rstd, dt * one("gamma1"), c["post"])
        else:
            dx = dt
        if c["gate"]:
            outs["dgate"].append(_sum_rows(dh * t))
        outs["dx"].append(dx.to(TYPES[c["x"]]))
    return outs


def _gradients(c):
    """The gradients that a case has."""
    return (["dx", "dr"] + (["dgate"] if c["gate"] else []) + (["dgamma1"] if c["post"] else []) + (["dbeta1"] if c["post"] == "layer" else []) + (["dgamma2"] if c["pre"] else [])
            + (["dbeta2"] if c["pre"] == "layer" else []))


# ---- the framework's own -------------------------------------------------------------------------
def _handles(s):
    """The descriptors and the calls that a program keeps with its buffers."""
    import paper_2110_15032_amd as sbp

    c = s["case"]
    k, op = c["k"], c["op"]
    code = {torch.float32: sbp.F32, torch.bfloat16: sbp.BF16, torch.float8_e4m3fn: sbp.F8E4M3}
    act = {"S0": sbp.S(0), "S1": sbp.S(1), "B": sbp.B}[c["sig"]]
    out = s["out"]

    def room(n):
        return torch.empty(n, dtype=torch.uint8, device="cuda") if n else None

    def tensor(shards, rows, cols, trans=0):
        shards = list(shards) if len(shards) == k else [shards[0]] * k
        return sbp.SbpTensor(shards, rows, cols, code[shards[0].dtype], trans, shards[0].stride(0))

    def vector(shards, n):
        """[n, 1]; one copy may stand for k."""
        shards = list(shards) if len(shards) == k else [shards[0]] * k
        return sbp.SbpTensor(shards, n, 1, code[shards[0].dtype])

    if op == "clip":
        layout = _layout(c)
        sigs = [sbp.B if axis is None else sbp.S(axis) for _, axis in layout]

        def listing(grads):
            return sbp.SbpList([sbp.SbpTensor(t, *shape, code[t[0].dtype], 0, t[0].stride(0)) for t, (shape, _) in zip(grads, layout)], sigs)

        grads, clipped = listing(s["grads"]), listing(s["clipped"])
        part = torch.empty(k, 4, device="cuda")
        squares, norm = sbp.SbpTensor(list(part), 1, 1, sbp.F32), sbp.SbpTensor([t.view(1) for t in out[1]], 1, 1, sbp.F32)
        return [(sbp.sbp_square_sum, (grads, squares, room(sbp.sbp_square_sum_workspace(grads, k)), k)), (sbp.sbp_clip, (grads, squares, sbp.P_SUM, c["max_norm"], clipped, norm, k))]
    if op == "linear":
        m, kk, n = c["M"], c["K"], c["N"]
        sx, sw = (sbp.S(0), sbp.B) if c["sig"] == "S0" else (sbp.B, sbp.S(1))
        return [(sbp.sbp_linear, (tensor(s["x"], m, kk), sx, tensor(s["w"], kk, n, int(c["w_trans"])), sw, vector(s["bias"], n),
                                  tensor(s["residual"], m, n) if c["residual"] else None, tensor(out[1], m, n) if c["pre"] else None, tensor(out[0], m, n), sbp.AUTO, k, None,
                                  sbp.EPI_GELU if c["gelu"] else sbp.EPI_NONE))]
    r, n = c["rows"], c["cols"]
    if op == "linear_grad":
        pre, da = (tensor(s["pre"], r, n), tensor(out[0], r, n)) if c["gelu"] else (None, None)
        return [(sbp.sbp_linear_grad, (tensor(s["dy"], r, n), act, pre, None, da, vector(out[-1], n), room(sbp.sbp_linear_grad_workspace(r, n, act, k)), k, None,
                                       sbp.EPI_GELU if c["gelu"] else sbp.EPI_NONE))]
    kinds = {"layer": sbp.NORM_LAYER, "rms": sbp.NORM_RMS}

    def weight(name):
        return vector([s[name]], n) if name in s else None

    def stat(t):
        return None if t is None else sbp.SbpTensor(t, r, 1, sbp.F32)

    if op == "norms":
        def norm(kind, which):
            if not kind:
                return None
            st = s["stats"][which] if c["stats"] else (None, None)
            return sbp.SbpNorm(kinds[kind], EPS, weight("gamma" + which), weight("beta" + which), stat(st[0]), stat(st[1]))

        y = tensor(out[1], r, n) if c["pre"] else None
        scales = sbp.SbpScales(out[2], out[2][0].stride(0)) if c["pre"] and c["y"] == "e4m3" else None
        return [(sbp.sbp_residual_norm, (tensor(s["x"], r, n), act, norm(c["post"], "1"), weight("gate"), tensor(s["r"], r, n), c["alpha"], tensor(out[0], r, n), norm(c["pre"], "2"),
                                         y, scales, k))]

    def norm(kind, which):
        if not kind:
            return None
        grads = [vector(out[name + which], n) if name + which in out else None for name in ("dgamma", "dbeta")]
        return sbp.SbpNorm(kinds[kind], EPS, weight("gamma" + which), weight("beta" + which), stat(s["mean" + which] if kind == "layer" else None), stat(s["rstd" + which]), *grads)

    return [(sbp.sbp_residual_norm_grad, (tensor(s["x"], r, n), act, norm(c["post"], "1"), weight("gate"), c["alpha"], tensor(s["h"], r, n) if c["pre"] else None, norm(c["pre"], "2"),
                                          tensor(s["dh"], r, n) if c["dh"] else None, tensor(s["dy"], r, n) if c["pre"] else None, tensor(out["dx"], r, n), tensor(out["dr"], r, n),
                                          vector(out["dgate"], n) if c["gate"] else None, room(sbp.sbp_residual_norm_grad_workspace(r, n, act, k)), k))]


# ---- what the tools call -------------------------------------------------------------------------
def prepare(case, seed):
    c, s = case, {"case": case}
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, k = c["op"], c["k"]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def fill(shards, parts):
        for t, v in zip(shards, parts):
            t.copy_(v)
        return shards

    def put(x, kind):
        return fill(_on_devices(x.shape, kind, c), _parts(x, c))

    def activation(*shape):
        """Normal values with a few strong channels, as residual streams have them."""
        strong = 1.0 + 7.0 * (torch.rand(shape[-1], generator=gen, device="cuda") < 0.02)
        return normal(*shape) * strong

    def vectors(n):
        """A vector for every device, 16 bytes apart or a multiple of it."""
        return list(_rows((k, n), torch.float32, 4))

    if op == "clip":
        layout = _layout(c)
        s["buckets"], s["grads"] = _buckets(c, TYPES[c["x"]])
        clipped, s["clipped"] = _buckets(c, TYPES[c["y"]])
        for shards, (shape, axis) in zip(s["grads"], layout):
            size = 10.0 ** torch.empty((), device="cuda").uniform_(-4.0, -1.0, generator=gen).item()   # layers' gradients differ in size
            whole = size * normal(*shape)
            fill(shards, [whole] * k if axis is None else whole.split(_share(shape[axis], k), axis))
        s["out"] = [clipped, [torch.zeros(4, device="cuda")[:1].view(()) for _ in range(k)]]
    elif op == "linear":
        m, kk, n = c["M"], c["K"], c["N"]
        x = activation(m, kk)
        s["x"] = fill(_split_rows((m, kk), TYPES[c["x"]], k, c["pad"]), x.split(_share(m, k))) if c["sig"] == "S0" else fill([_rows((m, kk), TYPES[c["x"]], c["pad"])], [x])
        devices = k if c["sig"] == "S1" else 1
        shape = (n // devices, kk) if c["w_trans"] else (kk, n // devices)
        s["w"] = [_rows(shape, TYPES[c["x"]], c["pad"]) for _ in range(devices)]
        fill(s["w"], [0.02 * normal(*shape) for _ in range(devices)])
        s["bias"] = [(0.1 * normal(n // devices)).to(TYPES[c["weights"]]) for _ in range(devices)]
        if c["residual"]:
            s["residual"] = put(activation(m, n), c["residual"])
        s["out"] = [_on_devices((m, n), c["y"], c)] + ([_on_devices((m, n), c["x"], c)] if c["pre"] else [])
    elif op == "linear_grad":
        shape = (c["rows"], c["cols"])
        s["dy"] = put(normal(*shape), c["y"])
        if c["gelu"]:
            s["pre"] = put(1.5 * activation(*shape), c["pre"])
        sums = vectors(shape[1] // (k if c["sig"] == "S1" else 1))
        s["out"] = [_on_devices(shape, c["y"], c), sums] if c["gelu"] else [sums]
    else:
        r, n = c["rows"], c["cols"]
        kind = TYPES[c["weights"]]
        if c["gate"]:
            s["gate"] = (0.5 + 0.2 * normal(n)).to(kind)
        for which, norm in (("1", c["post"]), ("2", c["pre"])):
            if norm:
                s["gamma" + which] = (1.0 + 0.1 * normal(n)).to(kind)
            if norm == "layer":
                s["beta" + which] = (0.1 * normal(n)).to(kind)
        s["x"] = put(activation(r, n) + 0.1 * normal(n), c["x"])
        stream = put(activation(r, n), c["r"])
        share = _share(r, k) if c["sig"] == "S0" else [r]

        def per_row():
            return [_rows((1, m), torch.float32, 4)[0] for m in share]

        if op == "norms":
            s["r"] = stream
            s["out"] = [_on_devices((r, n), c["r"], c)]
            if c["pre"]:
                s["out"].append(_on_devices((r, n), c["y"], c))
                if c["y"] == "e4m3":
                    s["out"].append([_rows((m, -(-n // BLOCK)), torch.uint8, 16).view(torch.float8_e8m0fnu) for m in share])
            if c["stats"]:
                s["stats"] = {w: (per_row() if norm == "layer" else None, per_row()) for w, norm in (("1", c["post"]), ("2", c["pre"])) if norm}
                pairs = [s["stats"][w] for w in ("1", "2") if w in s["stats"]]
                s["out"].append([t for i in range(len(share)) for pair in pairs for half in pair if half is not None for t in [half[i]]])
        else:
            # statistics and residual stream as the forward pass leaves them
            names = {w: (per_row(), per_row()) for w in ("1", "2")}
            s["h"] = []
            for i, (x, rr) in enumerate(zip(s["x"], stream)):
                t = x.double()
                if c["post"]:
                    xhat, mean, rstd = _standard(t, c["post"])
                    names["1"][0][i].copy_(mean[:, 0])
                    names["1"][1][i].copy_(rstd[:, 0])
                    t = xhat * s["gamma1"].double() + (s["beta1"].double() if "beta1" in s else 0.0)
                h = c["alpha"] * rr.double() + (s["gate"].double() if c["gate"] else 1.0) * t
                if c["pre"]:
                    _, mean, rstd = _standard(h, c["pre"])
                    names["2"][0][i].copy_(mean[:, 0])
                    names["2"][1][i].copy_(rstd[:, 0])
                rr.copy_(h)
                s["h"].append(rr)
            for w in ("1", "2"):
                s["mean" + w], s["rstd" + w] = names[w]
            if c["pre"]:
                s["dy"] = put(normal(r, n), c["y"])
            if c["dh"]:
                s["dh"] = put(normal(r, n), c["r"])
            s["out"] = {name: _on_devices((r, n), c["x" if name == "dx" else "r"], c) if name in ("dx", "dr") else vectors(n) for name in _gradients(c)}
    if own:
        s["calls"] = _handles(s)
    return s


def run(s):
    if own:
        for call, args in s["calls"]:
            call(*args)
        return s["out"]
    return _plain(s)


def work(case):
    c = case
    if c["op"] == "linear":
        m, kk, n = c["M"], c["K"], c["N"]
        out = SIZE[c["y"]] + (SIZE[c["x"]] if c["pre"] else 0) + (SIZE[c["residual"]] if c["residual"] else 0)
        return {"bytes": (m + n) * kk * SIZE[c["x"]] + n * SIZE[c["weights"]] + m * n * out, "flops": 2.0 * m * kk * n}
    if c["op"] == "clip":
        values = sum(a * b for shape, axis in _layout(c) for a, b in _local_shapes(shape, axis, 1 if axis is None else c["k"]))
        copies = sum(a * b for shape, axis in _layout(c) for a, b in _local_shapes(shape, axis, c["k"]))
        return {"bytes": copies * (SIZE[c["x"]] + SIZE[c["y"]]), "flops": 2.0 * values + copies}
    v, n, k = c["rows"] * c["cols"], c["cols"], c["k"]
    if c["op"] == "linear_grad":
        read, wrote = SIZE[c["y"]] + (SIZE[c["pre"]] if c["gelu"] else 0), SIZE[c["y"]] if c["gelu"] else 0
        return {"bytes": v * (read + wrote) + 4 * n * (1 if c["sig"] == "S1" else k), "flops": (21.0 if c["gelu"] else 1.0) * v}
    weights = (1 if c["gate"] else 0) + {"": 0, "rms": 1, "layer": 2}[c["post"]] + {"": 0, "rms": 1, "layer": 2}[c["pre"]]
    stats = {"": 0, "rms": 1, "layer": 2}[c["post"]] + {"": 0, "rms": 1, "layer": 2}[c["pre"]]
    if c["op"] == "norms":
        each = SIZE[c["x"]] + 2 * SIZE[c["r"]] + (SIZE[c["y"]] + (1 / BLOCK if c["y"] == "e4m3" else 0) if c["pre"] else 0)
        return {"bytes": v * each + n * weights * SIZE[c["weights"]] + (4 * c["rows"] * stats if c["stats"] else 0), "flops": 20.0 * v}
    each = 2 * SIZE[c["x"]] + SIZE[c["r"]] * (1 + (1 if c["pre"] else 0) + (1 if c["dh"] else 0)) + (SIZE[c["y"]] if c["pre"] else 0)
    return {"bytes": v * each + n * weights * (SIZE[c["weights"]] + 4 * k) + 4 * c["rows"] * stats, "flops": 35.0 * v}


# ---- the definitions in 64 bits ------------------------------------------------------------------
def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    c = case
    op, k = c["op"], c["k"]
    cdf = lambda t: 0.5 * torch.erfc(-t / math.sqrt(2.0))  # noqa: E731
    if op == "clip":
        squares = [torch.dot(t.double().flatten(), t.double().flatten()) for shards, (_, axis) in zip(s["grads"], _layout(c)) for t in (shards[:1] if axis is None else shards)]
        norm = math.sqrt(math.fsum(t.item() for t in squares))
        factor = c["max_norm"] / max(norm, c["max_norm"])
        return [t.double() * factor for t in s["buckets"]], [torch.tensor(norm, dtype=torch.float64, device="cuda")] * k
    if op == "linear":
        out, pre = [], []
        for i in range(k):
            x, w, b = s["x"][i % len(s["x"])].double(), s["w"][i % len(s["w"])].double(), s["bias"][i % len(s["bias"])].double()
            a = torch.addmm(b.expand(x.shape[0], -1), x, (w.T if c["w_trans"] else w).contiguous())
            pre.append(a)
            y = a * cdf(a) if c["gelu"] else a
            out.append(y + s["residual"][i].double() if c["residual"] else y)
        return [out, pre] if c["pre"] else [out]
    if op == "linear_grad":
        out = [t.double() for t in s["dy"]]
        if c["gelu"]:
            slope = lambda a: cdf(a) + a * torch.exp(-a * a / 2.0) / math.sqrt(2.0 * math.pi)  # noqa: E731
            out = [d * slope(a.double()) for d, a in zip(out, s["pre"])]
        sums = [t.sum(0) for t in out]
        return [out, sums] if c["gelu"] else [sums]
    n = c["cols"]
    weight = {name: s[name].double() if name in s else None for name in ("gate", "gamma1", "beta1", "gamma2", "beta2")}

    def affine(t, which):
        t = t * weight["gamma" + which]
        return t if weight["beta" + which] is None else t + weight["beta" + which]

    def statistics(t, kind):
        mean = t.sum(-1) / n if kind == "layer" else None
        d = t - mean[:, None] if kind == "layer" else t
        return d, mean, 1.0 / torch.sqrt((d * d).sum(-1) / n + EPS)

    gated = lambda t: t if weight["gate"] is None else t * weight["gate"]  # noqa: E731
    if op == "norms":
        hs, ys, scales, stats = [], [], [], []
        for x, r in zip(s["x"], s["r"]):
            t = x.double()
            for_row = []
            if c["post"]:
                d, mean, rstd = statistics(t, c["post"])
                t = affine(d * rstd[:, None], "1")
                for_row += [mean, rstd]
            h = gated(t) + c["alpha"] * r.double()
            hs.append(h)
            if c["pre"]:
                d, mean, rstd = statistics(h, c["pre"])
                y = affine(d * rstd[:, None], "2")
                for_row += [mean, rstd]
                if c["y"] == "e4m3":
                    most = torch.stack([b.abs().amax(-1) for b in y.split(BLOCK, -1)], -1)
                    scale = torch.exp2(torch.ceil(torch.log2(most / (0.875 * 2.0 ** TOP))).clamp(min=-127.0))
                    scales.append(scale)
                    y = y / scale[:, torch.arange(n, device="cuda") // BLOCK]
                ys.append(y)
            stats += [t for t in for_row if t is not None]
        return [hs] + ([ys] if c["pre"] else []) + ([scales] if scales else []) + ([stats] if c["stats"] else [])
    outs = {name: [] for name in _gradients(c)}
    for i, x in enumerate(s["x"]):
        total = s["dh"][i].double() if c["dh"] else 0.0
        if c["pre"]:
            dy, h, rstd = s["dy"][i].double(), s["h"][i].double(), s["rstd2"][i].double()[:, None]
            hhat = (h - s["mean2"][i].double()[:, None]) * rstd if c["pre"] == "layer" else h * rstd
            g = dy * weight["gamma2"]
            along = n * g - hhat * (g * hhat).sum(-1, keepdim=True) - (g.sum(-1, keepdim=True) if c["pre"] == "layer" else 0.0)
            total = total + rstd / n * along
            outs["dgamma2"].append((dy * hhat).sum(0))
            if c["pre"] == "layer":
                outs["dbeta2"].append(dy.sum(0))
        outs["dr"].append(c["alpha"] * total)
        t = x.double()
        dt = gated(total)
        if c["post"]:
            rstd = s["rstd1"][i].double()[:, None]
            xhat = (t - s["mean1"][i].double()[:, None]) * rstd if c["post"] == "layer" else t * rstd
            t = affine(xhat, "1")
            outs["dgamma1"].append((dt * xhat).sum(0))
            if c["post"] == "layer":
                outs["dbeta1"].append(dt.sum(0))
            g = dt * weight["gamma1"]
            dx = rstd / n * (n * g - xhat * (g * xhat).sum(-1, keepdim=True) - (g.sum(-1, keepdim=True) if c["post"] == "layer" else 0.0))
        else:
            dx = dt
        if c["gate"]:
            outs["dgate"].append((total * t).sum(0))
        outs["dx"].append(dx)
    return outs
