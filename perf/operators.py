"""Performance cases of the 8-bit training and serving operators of an MLP block: layer normalisation with its gradient,
activations kept in 8 bits and used from there in the backward pass, and the product of two 8-bit tensors.

An 8-bit tensor is float8 (e4m3 or e5m2) values, and one power of two for every 128 consecutive values of a stored row:
scale = 2^e, e the smallest integer >= -127 with max|block| / 2^e within the type (448 and 57344), values = round(x / scale).
Scales are held in one byte each (e + 127, torch.float8_e8m0fnu).  Outputs in 8 bits are returned as the two tensors in
their own floating types: numbers, not codes.

`op` names the operator, `k` the number of logical devices (shard buffers in one GPU's memory), `sig` the signature of the
activations: "S0" rows split, "S1" columns split, "P" reduction split (products only; the result is P(sum)), "B" one copy.

  norm        y = (x - mean) / sqrt(var + eps) * gamma + beta over every row, with mean and 1/sqrt(var + eps) for training
  norm_grad   dx, and the sums over the rows of dy * xhat (gamma) and dy (beta), one partial for every device
  save        an activation (or, `gelu`, GeLU of it) into 8 bits; `trans`: stored transposed, blocks along the rows
  restore     from 8 bits back to bf16 or fp32 (`gelu`: GeLU of it, recomputed instead of kept)
  gelu_grad   da = dh * gelu'(a) with the pre-activation a from 8 bits or whole
  matmul      y = x w of 8-bit operands, both stored with the reduction index contiguous

Rows lie `pad` elements apart rounded up (0: back to back).
"""
import math

import torch

own = False

BLOCK = 128
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
SIZE = {"f32": 4, "bf16": 2, "e4m3": 1, "e5m2": 1}
#: the largest value of a type is 0.875 * 2^TOP
TOP = {"e4m3": 9, "e5m2": 16}
EPS = 1e-5


def listed():
    return [
        # one token through the norm in front of a block: latency
        dict(name="norm one token", op="norm", k=1, sig="B", rows=1, cols=4096, x="bf16", y="bf16", weights="bf16", stats=False, pad=0),
        # the norm in front of the MLP block at its full size, straight into the 8-bit operand of the first product
        dict(name="norm to 8 bits", op="norm", k=8, sig="S0", rows=8192, cols=4096, x="bf16", y="e4m3", weights="f32", stats=True, pad=16),
        # training in fp32 on a last, uneven batch of a layer whose width divides nothing
        dict(name="norm gradient odd", op="norm_grad", k=3, sig="S0", rows=1767, cols=1001, x="f32", y="f32", weights="f32", pad=16),
        # data-parallel training: the norm's input was kept in 8 bits
        dict(name="norm gradient", op="norm_grad", k=8, sig="S0", rows=16384, cols=4096, x="e4m3", y="bf16", weights="bf16", pad=16),
        # the MLP block's pre-activation, column-parallel, kept for the backward pass
        dict(name="save", op="save", k=8, sig="S1", rows=8192, cols=16384, x="bf16", y="e4m3", gelu=False, trans=False, pad=16),
        # the operand of a weight gradient: GeLU of the pre-activation, blocks along the tokens
        dict(name="save transposed gelu", op="save", k=8, sig="S0", rows=16384, cols=1024, x="bf16", y="e4m3", gelu=True, trans=True, pad=16),
        # GeLU recomputed from the kept pre-activation for a 16-bit weight gradient, an uneven batch
        dict(name="restore gelu", op="restore", k=3, sig="S0", rows=7777, cols=4081, x="e4m3", y="bf16", gelu=True, trans=False, pad=16),
        # backward of the activation, a small fp32 layer
        dict(name="gelu gradient odd", op="gelu_grad", k=1, sig="B", rows=333, cols=1001, x="f32", y="f32", pad=0),
        # backward of the MLP block's activation from the kept pre-activation
        dict(name="gelu gradient", op="gelu_grad", k=8, sig="S1", rows=8192, cols=16384, x="e4m3", y="bf16", pad=16),
        # decoding: one token through a column-parallel weight, the weight is the traffic
        dict(name="matmul one token", op="matmul", k=8, sig="S1", M=1, K=4096, N=16384, x="e4m3", w="e4m3", y="bf16", gelu=False, pad=16),
        # gradients (e5m2) times a weight, row-parallel on three devices, lengths that no block divides, fp32 partials
        dict(name="matmul ragged", op="matmul", k=3, sig="P", M=777, K=3 * 1000, N=1501, x="e5m2", w="e4m3", y="f32", gelu=False, pad=16),
        # the first product of the MLP block at its full size
        dict(name="matmul mlp", op="matmul", k=8, sig="S1", M=8192, K=4096, N=16384, x="e4m3", w="e4m3", y="bf16", gelu=False, pad=16),
    ]


def _size(rng, lo, hi, step=1):
    """Spread over the logarithm of lo .. hi, a multiple of step."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(step, n // step * step)


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "save", "restore", "gelu_grad", "matmul"])
    k = rng.choice([1, 2, 3, 4, 8])
    pad = rng.choice([16, 16, 64, 128])
    if op == "matmul":
        sig = rng.choice(["S0", "S1", "P"])
        step = rng.choice([1, 1, 8, 16, 128])
        while True:
            m, kk, n = _size(rng, 1, 8192), _size(rng, 128, 16384, step), _size(rng, 64, 16384, step)
            if m * kk * n <= 8192 * 4096 * 16384:
                break
        kk, n = (-(-kk // k) * k, n) if sig == "P" else (kk, -(-n // k) * k)
        y = "f32" if sig == "P" else rng.choice(["bf16", "bf16", "f32"])
        return dict(op=op, k=k, sig=sig, M=m, K=kk, N=n, x=rng.choice(["e4m3", "e4m3", "e5m2"]), w=rng.choice(["e4m3", "e4m3", "e5m2"]), y=y,
                    gelu=sig != "P" and rng.random() < 0.3, pad=pad)
    while True:
        rows, cols = _size(rng, 1, 32768), _size(rng, 64, 16384, rng.choice([1, 8, 64]))
        if rows * cols <= 8192 * 8192:
            break
    if op == "norm":
        return dict(op=op, k=k, sig="S0", rows=rows, cols=cols, x=rng.choice(["bf16", "bf16", "f32"]), y=rng.choice(["bf16", "e4m3", "f32"]),
                    weights=rng.choice(["f32", "bf16"]), stats=rng.random() < 0.7, pad=pad)
    if op == "norm_grad":
        return dict(op=op, k=k, sig="S0", rows=rows, cols=cols, x=rng.choice(["bf16", "f32", "e4m3"]), y=rng.choice(["bf16", "bf16", "f32"]),
                    weights=rng.choice(["f32", "bf16"]), pad=pad)
    sig = rng.choice(["S0", "S1"])
    if sig == "S1":
        cols = -(-cols // k) * k
    if op == "gelu_grad":
        return dict(op=op, k=k, sig=sig, rows=rows, cols=cols, x=rng.choice(["e4m3", "e4m3", "bf16", "f32"]), y=rng.choice(["bf16", "bf16", "f32"]), pad=pad)
    trans = rng.random() < 0.4
    if trans and sig == "S0":
        rows = -(-rows // k) * k
    gelu = rng.random() < 0.3
    if op == "save":
        return dict(op=op, k=k, sig=sig, rows=rows, cols=cols, x=rng.choice(["bf16", "bf16", "f32"]), y=rng.choice(["e4m3", "e4m3", "e5m2"]), gelu=gelu,
                    trans=trans, pad=pad)
    return dict(op=op, k=k, sig=sig, rows=rows, cols=cols, x=rng.choice(["e4m3", "e4m3", "e5m2"]), y=rng.choice(["bf16", "bf16", "f32"]), gelu=gelu,
                trans=trans, pad=pad)


# ---- shapes and buffers -------------------------------------------------------------------------
def _share(n, k):
    """Sizes of the balanced split: the first n mod k devices hold one more."""
    return [n // k + (i < n % k) for i in range(k)]


def _shape(c, trans=False):
    """Shape of all local tensors of an activation together: S(1) ones (and transposed S(0) ones) have a leading index for the device."""
    shape = (c["k"], c["rows"], c["cols"] // c["k"]) if c["sig"] == "S1" else (c["rows"], c["cols"])
    if trans and c["sig"] == "S0":
        shape = (c["k"], c["rows"] // c["k"], c["cols"])
    return (*shape[:-2], shape[-1], shape[-2]) if trans else shape


def _up(n, step):
    return -(-n // step) * step if step else n


def _rows(shape, dtype, pad):
    """A buffer whose rows lie a multiple of `pad` elements apart."""
    return torch.zeros(*shape[:-1], _up(shape[-1], pad), dtype=dtype, device="cuda")[..., : shape[-1]]


def _blocks(n):
    return -(-n // BLOCK)


def _in8(shape, kind, pad):
    """Buffers of an 8-bit tensor and its scales, whose rows always lie 16 bytes apart or a multiple of it."""
    values = _rows(shape, torch.uint8, pad).view(TYPES[kind])
    return values, _rows((*shape[:-1], _blocks(shape[-1])), torch.uint8, 16).view(torch.float8_e8m0fnu)


def _shards(t, c):
    """The k local tensors: views of the buffer that holds them all."""
    if t.dim() == 3:
        return list(t)
    return list(t.split(_share(t.shape[0], c["k"]))) if c["sig"] == "S0" else [t] * c["k"]


# ---- the operators in their plain form ----------------------------------------------------------
def _widen(values, scales):
    """8 bits to fp32 (exact)."""
    return values.float() * scales.float().repeat_interleave(BLOCK, -1)[..., : values.shape[-1]]


def _narrow(x, kind):
    """x in fp32 (or 64 bits) to 8-bit values and scales, blocks along the last axis."""
    n = x.shape[-1]
    b = torch.nn.functional.pad(x, (0, -n % BLOCK)).unflatten(-1, (-1, BLOCK))
    m, e = torch.frexp(b.abs().amax(-1))
    e = torch.where(m == 0, -127, e - TOP[kind] + (m > 0.875).int()).clamp(min=-127)
    values = torch.ldexp(b, -e.unsqueeze(-1)).float().to(TYPES[kind]).flatten(-2)[..., :n]
    return values, (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _gelu(x):
    return 0.5 * x * (1.0 + torch.erf(x * math.sqrt(0.5)))


def _gelu_slope(x):
    return 0.5 * (1.0 + torch.erf(x * math.sqrt(0.5))) + x * torch.exp(-0.5 * x * x) * (1.0 / math.sqrt(2.0 * math.pi))


def _read(s, name):
    """An input in fp32, from 8 bits where its scales are there."""
    return _widen(s[name], s[name + "_scales"]) if name + "_scales" in s else s[name].float()


def _plain(s):
    c = s["case"]
    op = c["op"]
    if op == "norm":
        x = s["x"].float()
        mean = x.mean(-1)
        d = x - mean.unsqueeze(-1)
        rstd = torch.rsqrt(d.square().mean(-1) + EPS)
        y = d * rstd.unsqueeze(-1) * s["gamma"].float() + s["beta"].float()
        out = list(_narrow(y, c["y"])) if c["y"] in TOP else [y.to(TYPES[c["y"]])]
        return out + ([t.split(_share(c["rows"], c["k"])) for t in (mean, rstd)] if c["stats"] else [])
    if op == "norm_grad":
        x, dy = _read(s, "x"), s["dy"].float()
        rstd = s["rstd"].unsqueeze(-1)
        xhat = (x - s["mean"].unsqueeze(-1)) * rstd
        g = dy * s["gamma"].float()
        dx = rstd * (g - g.mean(-1, keepdim=True) - xhat * (g * xhat).mean(-1, keepdim=True))
        share = _share(c["rows"], c["k"])
        return [dx.to(TYPES[c["y"]]), torch.stack([t.sum(0) for t in (dy * xhat).split(share)]), torch.stack([t.sum(0) for t in dy.split(share)])]
    if op == "save":
        x = s["x"].float()
        x = _gelu(x) if c["gelu"] else x
        if c["trans"]:
            x = (x.unflatten(0, (c["k"], -1)) if c["sig"] == "S0" else x).transpose(-1, -2)
        return list(_narrow(x, c["y"]))
    if op == "restore":
        x = _read(s, "x")
        x = (_gelu(x) if c["gelu"] else x).to(TYPES[c["y"]])
        if c["trans"]:
            x = x.transpose(-1, -2)
            x = x.flatten(0, 1) if c["sig"] == "S0" else x
        return [x]
    if op == "gelu_grad":
        return [(s["dh"].float() * _gelu_slope(_read(s, "x"))).to(TYPES[c["y"]])]
    x, w = _read(s, "x"), _read(s, "w")
    y = torch.matmul(x, w.transpose(-1, -2))
    y = (_gelu(y) if c["gelu"] else y).to(TYPES[c["y"]])
    return [y.unflatten(1, (c["k"], -1)).transpose(0, 1) if c["sig"] == "S1" else y]


# ---- the framework's own -------------------------------------------------------------------------
def _handles(s):
    """The descriptors and the call that a program keeps with its buffers."""
    import paper_2110_15032_amd as sbp

    c = s["case"]
    k, op = c["k"], c["op"]
    code = {torch.float32: sbp.F32, torch.bfloat16: sbp.BF16, torch.float8_e4m3fn: sbp.F8E4M3, torch.float8_e5m2: sbp.F8E5M2}
    sig = {"S0": sbp.S(0), "S1": sbp.S(1), "B": sbp.B}

    def tensor(shards, rows, cols, trans=0):
        return sbp.SbpTensor(shards, rows, cols, code[shards[0].dtype], trans, shards[0].stride(0) if shards[0].dim() == 2 else 0)

    def scales(name):
        t = _shards(s[name + "_scales"], c) if name + "_scales" in s else None
        return None if t is None else sbp.SbpScales(t, t[0].stride(0))

    def vector(name):
        """A weight that every device has: one copy stands for k."""
        return sbp.SbpTensor([s[name]] * k, s[name].numel(), 1, code[s[name].dtype])

    if op == "matmul":
        m, kk, n = c["M"], c["K"], c["N"]
        sx, sw, sy = {"S0": (sbp.S(0), sbp.B, sbp.S(0)), "S1": (sbp.B, sbp.S(1), sbp.S(1)), "P": (sbp.S(1), sbp.S(0), sbp.P_SUM)}[c["sig"]]

        def parts(t, split):
            return list(t) if t.dim() == 3 else list(t.split(_share(t.shape[0], k))) if split else [t] * k

        x, xs = (parts(s[n_], c["sig"] == "S0") for n_ in ("x", "x_scales"))
        w, ws = (parts(s[n_], c["sig"] == "S1") for n_ in ("w", "w_scales"))
        y = parts(s["out"][0], c["sig"] == "S0")
        a = (tensor(x, m, kk), sbp.SbpScales(xs, xs[0].stride(0)), sx, tensor(w, kk, n, 1), sbp.SbpScales(ws, ws[0].stride(0)), sw, tensor(y, m, n), sy, k, None,
             sbp.EPI_GELU if c["gelu"] else sbp.EPI_NONE)
        return sbp.sbp_matmul_f8, a
    r, n = c["rows"], c["cols"]
    act = sig[c["sig"]]
    epi = sbp.EPI_GELU if c.get("gelu") else sbp.EPI_NONE
    x = tensor(_shards(s["x"], c), r, n, int(op == "restore" and c["trans"]))
    out = s["out"]
    if op == "norm":
        y = tensor(_shards(out[0], c), r, n)
        ys = sbp.SbpScales(_shards(out[1], c), out[1].stride(0)) if c["y"] in TOP else None
        st = [sbp.SbpTensor(t, r, 1, sbp.F32) for t in s["stats"]] if c["stats"] else [None, None]
        return sbp.sbp_layernorm, (x, act, vector("gamma"), vector("beta"), EPS, y, ys, *st, k)
    if op == "norm_grad":
        st = [sbp.SbpTensor(t, r, 1, sbp.F32) for t in s["stats"]]
        dg, db = (sbp.SbpTensor(list(t), n, 1, sbp.F32) for t in out[1:])
        room = torch.empty(sbp.sbp_layernorm_grad_workspace(r, n, act, k), dtype=torch.uint8, device="cuda")
        return sbp.sbp_layernorm_grad, (x, scales("x"), act, vector("gamma"), *st, tensor(_shards(s["dy"], c), r, n), tensor(_shards(out[0], c), r, n), dg, db, room, k)
    if op == "save":
        q, qs = (_shards(t, c) for t in out)
        return sbp.sbp_quantize, (x, act, tensor(q, r, n, int(c["trans"])), sbp.SbpScales(qs, qs[0].stride(0)), k, None, epi)
    if op == "restore":
        return sbp.sbp_dequantize, (x, scales("x"), act, tensor(_shards(out[0], c), r, n), k, None, epi)
    return sbp.sbp_gelu_grad, (x, scales("x"), act, tensor(_shards(s["dh"], c), r, n), tensor(_shards(out[0], c), r, n), k)


# ---- what the tools call -------------------------------------------------------------------------
def prepare(case, seed):
    c, s = case, {"case": case}
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def put(x, kind):
        t = _rows(x.shape, TYPES[kind], c["pad"])
        t.copy_(x)
        return t

    def put8(name, x, kind):
        s[name], s[name + "_scales"] = _in8(x.shape, kind, c["pad"])
        values, scales = _narrow(x, kind)
        s[name].view(torch.uint8).copy_(values.view(torch.uint8))
        s[name + "_scales"].view(torch.uint8).copy_(scales.view(torch.uint8))

    def activation(*shape):
        """Normal values with a few strong channels, as residual streams have them."""
        strong = 1.0 + 7.0 * (torch.rand(shape[-1], generator=gen, device="cuda") < 0.02)
        return normal(*shape) * strong

    def per_row():
        """Every device's own vectors of means and of 1 / deviation, 16 bytes apart or a multiple of it."""
        room = [torch.zeros(c["k"], _up(-(-c["rows"] // c["k"]), 4), device="cuda") for _ in range(2)]
        return [[t[i, :m] for i, m in enumerate(_share(c["rows"], c["k"]))] for t in room]

    op, k = c["op"], c["k"]
    if op == "matmul":
        m, kk, n = c["M"], c["K"], c["N"]
        split = c["sig"] == "P"
        put8("x", activation(k, m, kk // k) if split else activation(m, kk), c["x"])
        put8("w", 0.02 * (normal(k, n, kk // k) if split else normal(n, kk)), c["w"])
        s["out"] = [_rows((k, m, n // k) if c["sig"] == "S1" else (k, m, n) if split else (m, n), TYPES[c["y"]], c["pad"])]
    elif op in ("norm", "norm_grad"):
        r, n = c["rows"], c["cols"]
        x = activation(r, n) + 0.1 * normal(n)
        s["gamma"] = (1.0 + 0.1 * normal(n)).to(TYPES[c["weights"]])
        if op == "norm":
            s["x"] = put(x, c["x"])
            s["beta"] = (0.1 * normal(n)).to(TYPES[c["weights"]])
            s["out"] = list(_in8((r, n), c["y"], c["pad"])) if c["y"] in TOP else [_rows((r, n), TYPES[c["y"]], c["pad"])]
            if c["stats"]:
                s["stats"] = per_row()
        else:
            if c["x"] in TOP:
                put8("x", x, c["x"])
            else:
                s["x"] = put(x, c["x"])
            x = _read(s, "x").double()
            s["mean"], s["rstd"] = x.mean(-1).float(), torch.rsqrt(x.var(-1, correction=0) + EPS).float()
            s["stats"] = per_row()
            for part, whole in zip(s["stats"], (s["mean"], s["rstd"])):
                for p, v in zip(part, whole.split(_share(r, k))):
                    p.copy_(v)
            s["dy"] = put(normal(r, n), c["y"])
            s["out"] = [_rows((r, n), TYPES[c["y"]], c["pad"])] + [_rows((k, n), torch.float32, 4) for _ in range(2)]
    else:
        shape = _shape(c)
        if op == "save":
            s["x"] = put(1.5 * activation(*shape), c["x"])
            s["out"] = list(_in8(_shape(c, c["trans"]), c["y"], c["pad"]))
        elif op == "restore":
            put8("x", 1.5 * activation(*_shape(c, c["trans"])), c["x"])
            s["out"] = [_rows(shape, TYPES[c["y"]], c["pad"])]
        else:
            x = 1.5 * activation(*shape)
            if c["x"] in TOP:
                put8("x", x, c["x"])
            else:
                s["x"] = put(x, c["x"])
            s["dh"] = put(normal(*shape), c["y"])
            s["out"] = [_rows(shape, TYPES[c["y"]], c["pad"])]
    if own:
        s["call"] = _handles(s)
    return s


def run(s):
    if own:
        call, args = s["call"]
        call(*args)
        return s["out"] + s["stats"] if s["case"]["op"] == "norm" and s["case"]["stats"] else list(s["out"])
    return _plain(s)


def work(case):
    c = case
    if c["op"] == "matmul":
        m, kk, n, k = c["M"], c["K"], c["N"], c["k"]
        b = _blocks(kk // k) * k if c["sig"] == "P" else _blocks(kk)
        out = m * n * (k if c["sig"] == "P" else 1) * SIZE[c["y"]]
        return {"bytes": (m + n) * (kk + b) + out, "flops": 2.0 * m * kk * n}
    r, n = c["rows"], c["cols"]
    v = r * n
    in8 = v / BLOCK
    read = v * SIZE[c["x"]] + (in8 if c["x"] in TOP else 0)
    wrote = v * SIZE[c["y"]] + (in8 if c["y"] in TOP else 0)
    if c["op"] == "norm":
        return {"bytes": read + wrote + 2 * n * SIZE[c["weights"]] + (8 * r if c["stats"] else 0), "flops": 8.0 * v}
    if c["op"] == "norm_grad":
        return {"bytes": read + 2 * wrote + n * SIZE[c["weights"]] + 8 * r + 8 * n * c["k"], "flops": 14.0 * v}
    if c["op"] == "gelu_grad":
        return {"bytes": read + 2 * wrote, "flops": 20.0 * v}
    return {"bytes": read + wrote, "flops": (20.0 if c["gelu"] else 2.0) * v}


# ---- the definitions in 64 bits ------------------------------------------------------------------
def _value(s, name):
    """An input's values in 64 bits, block by block."""
    if name + "_scales" not in s:
        return s[name].double()
    v = s[name].double()
    place = torch.arange(v.shape[-1], device=v.device) // BLOCK
    power = s[name + "_scales"].view(torch.uint8).double() - 127.0
    return v * torch.exp2(power[..., place])


def _to8(x, kind):
    """Unrounded values and scales of a tensor in 8 bits, found by looking at each block's largest magnitude."""
    most = 0.875 * 2.0 ** TOP[kind]
    scale = torch.stack([t.abs().amax(-1) for t in x.split(BLOCK, -1)], -1)
    scale = torch.exp2(torch.ceil(torch.log2(scale / most)).clamp(min=-127.0))
    place = torch.arange(x.shape[-1], device=x.device) // BLOCK
    return [x / scale[..., place], scale]


def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    c = case
    op, k = c["op"], c["k"]
    normal_cdf = lambda t: 0.5 * torch.erfc(-t / math.sqrt(2.0))  # noqa: E731
    if op == "matmul":
        x, w = _value(s, "x"), _value(s, "w")
        if c["sig"] == "P":
            return [torch.stack([x[i] @ w[i].T.contiguous() for i in range(k)])]
        y = x @ w.T.contiguous()
        y = y * normal_cdf(y) if c["gelu"] else y
        return [torch.stack(y.chunk(k, 1)) if c["sig"] == "S1" else y]
    x = _value(s, "x")
    if op in ("norm", "norm_grad"):
        n = c["cols"]
        if op == "norm":
            mean = x.sum(-1) / n
            var = (x - mean[:, None]).square().sum(-1) / n
            rstd = 1.0 / torch.sqrt(var + EPS)
            y = (x - mean[:, None]) * rstd[:, None] * s["gamma"].double() + s["beta"].double()
            return (_to8(y, c["y"]) if c["y"] in TOP else [y]) + ([t.split(_share(c["rows"], k)) for t in (mean, rstd)] if c["stats"] else [])
        dy, mean, rstd = s["dy"].double(), s["mean"].double()[:, None], s["rstd"].double()[:, None]
        xhat, g = (x - mean) * rstd, dy * s["gamma"].double()
        dx = rstd / n * (n * g - g.sum(-1, keepdim=True) - xhat * (g * xhat).sum(-1, keepdim=True))
        edge = [0]
        for m in _share(c["rows"], k):
            edge.append(edge[-1] + m)
        cut = lambda t: torch.stack([t[a:b].sum(0) for a, b in zip(edge, edge[1:])])  # noqa: E731
        return [dx, cut(dy * xhat), cut(dy)]
    if op == "gelu_grad":
        return [s["dh"].double() * (normal_cdf(x) + x * torch.exp(-x * x / 2.0) / math.sqrt(2.0 * math.pi))]
    if c["gelu"]:
        x = x * normal_cdf(x)
    if c["trans"]:
        if op == "save" and c["sig"] == "S0":
            x = torch.stack(x.chunk(k, 0))
        x = x.transpose(-1, -2)
        if op == "restore" and c["sig"] == "S0":
            x = x.reshape(c["rows"], c["cols"])
    return _to8(x.contiguous(), c["y"]) if op == "save" else [x]
