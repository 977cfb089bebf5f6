"""The 64-bit forms that the operators around an MLP block's products are tested against, against differences and automatic differentiation."""
import pytest
import torch

import train_reference as ref

FORMS = [(None, ref.LAYER), (None, ref.RMS), (ref.LAYER, ref.LAYER), (ref.RMS, ref.RMS), (ref.RMS, None), (ref.LAYER, ref.RMS), (ref.LAYER, None)]


def rand(*shape, seed):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def forward(x, r, w, post, pre, alpha):
    """The definition, in plain operations."""
    def norm(v, kind, gamma, beta):
        if kind == ref.LAYER:
            v = v - v.mean(1, keepdim=True)
        v = v * (v.square().mean(1, keepdim=True) + 1e-3).rsqrt() * gamma
        return v + beta if kind == ref.LAYER else v
    t = x if post is None else norm(x, post, w["gamma1"], w["beta1"])
    h = alpha * r + w["gate"] * t
    return h, None if pre is None else norm(h, pre, w["gamma2"], w["beta2"])


@pytest.mark.parametrize("post,pre", FORMS)
@pytest.mark.parametrize("rows,n", [(5, 9), (1, 1), (3, 64)])
def test_norms_and_their_gradients(post, pre, rows, n):
    alpha = 0.7
    w = {name: rand(n, seed=i) + 1.0 for i, name in enumerate(("gate", "gamma1", "beta1", "gamma2", "beta2"))}
    x, r = rand(rows, n, seed=7), rand(rows, n, seed=8)
    dh, dy = rand(rows, n, seed=9), rand(rows, n, seed=10)
    p1 = None if post is None else ref.Norm(post, 1e-3, w["gamma1"], w["beta1"] if post == ref.LAYER else None)
    p2 = None if pre is None else ref.Norm(pre, 1e-3, w["gamma2"], w["beta2"] if pre == ref.LAYER else None)
    got = ref.residual_norm(x, r, p1, w["gate"], alpha, p2)
    h, y = forward(x, r, w, post, pre, alpha)
    assert torch.allclose(got["h"][0], h, rtol=1e-12, atol=1e-12) and (y is None or torch.allclose(got["y"][0], y, rtol=1e-10, atol=1e-12))
    stats = [got[name][0] if name in got else None for name in ("mean1", "rstd1", "mean2", "rstd2")]
    grads = ref.residual_norm_grad(x, p1, w["gate"], alpha, h, p2, dh, dy if pre is not None else None, stats)

    def loss(x, r, w):
        h, y = forward(x, r, w, post, pre, alpha)
        return (h * dh).sum() + (0.0 if y is None else (y * dy).sum())
    inputs = {"x": x, "r": r, **w}
    for name, value in inputs.items():
        key = "d" + name
        if key not in grads or (key == "dbeta1" and post == ref.RMS) or (key == "dbeta2" and pre == ref.RMS):
            continue
        leaf = value.clone().requires_grad_()
        rest = {k: (leaf if k == name else v) for k, v in inputs.items()}
        loss(rest["x"], rest["r"], {k: rest[k] for k in w}).backward()
        assert torch.allclose(grads[key][0], leaf.grad, rtol=1e-8, atol=1e-9), key
        for at in range(0, value.numel(), max(1, value.numel() // 5)):          # central differences
            step = 1e-5
            both = []
            for sign in (1, -1):
                moved = value.clone()
                moved.view(-1)[at] += sign * step
                rest = {k: (moved if k == name else v) for k, v in inputs.items()}
                both.append(float(loss(rest["x"], rest["r"], {k: rest[k] for k in w})))
            slope = (both[0] - both[1]) / (2 * step)
            assert abs(slope - float(grads[key][0].reshape(-1)[at])) <= 1e-5 * (1 + abs(slope)), key
