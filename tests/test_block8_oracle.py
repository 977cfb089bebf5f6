"""The 64-bit implementation of 8-bit tensors and layer normalisation against torch's casts, scipy-free formulas and differences (CPU)."""
import numpy as np
import pytest
import torch

from oracle import block8_oracle as o8

TORCH = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


@pytest.mark.parametrize("kind", ["e4m3", "e5m2"])
def test_decoding_is_torchs(kind):
    codes = torch.arange(256, dtype=torch.uint8)
    np.testing.assert_array_equal(o8.decode_table(kind), codes.view(TORCH[kind]).double().numpy())


@pytest.mark.parametrize("kind", ["e4m3", "e5m2"])
def test_encoding_is_torchs_nearest_even(kind):
    rng = np.random.default_rng(0)
    t = o8.decode_table(kind)[:128]
    t = t[np.isfinite(t)]
    x = np.concatenate([t, (t[1:] + t[:-1]) / 2, rng.uniform(-1, 1, 4000) * 2.0 ** rng.integers(-16, 8, 4000)]).astype(np.float32)
    x = np.concatenate([x, -x])
    want = torch.from_numpy(x).to(TORCH[kind]).view(torch.uint8).numpy()
    np.testing.assert_array_equal(o8.encode(x.astype(np.float64), kind), want)


@pytest.mark.parametrize("kind,top", [("e4m3", 448.0), ("e5m2", 57344.0)])
def test_scale_is_the_smallest_that_fits(kind, top):
    assert o8.largest(kind) == top
    for most in (1.0, 0.875, 0.8750001, 1.75, 1.7500001, 448.0, 448.1, 1e-30, 3e38, 2.0 ** -133, 0.0):
        x = np.zeros((1, 130))
        x[0, 5], x[0, 128] = most, -most
        s = o8.scale_bytes(x, kind)
        assert s.shape == (1, 2) and s[0, 0] == s[0, 1]
        e = int(s[0, 0]) - 127
        assert most / 2.0 ** e <= top and (e == -127 or most / 2.0 ** (e - 1) > top)


def test_specials_leave_their_block_alone():
    x = np.ones((1, 128))
    x[0, 3], x[0, 4] = np.inf, np.nan
    for kind in ("e4m3", "e5m2"):
        q, s = o8.quantize(x, kind)
        v = o8.dequantize(q, s, kind)
        assert (np.delete(v, [3, 4]) == 1.0).all() and np.isnan(v[0, 4])
        assert np.isnan(v[0, 3]) if kind == "e4m3" else np.isinf(v[0, 3])


def test_gradients_are_differences():
    rng = np.random.default_rng(1)
    x, dy = rng.normal(size=(5, 37)), rng.normal(size=(5, 37))
    gamma, beta, eps = rng.normal(size=37), rng.normal(size=37), 1e-5
    y, mean, rstd = o8.layernorm(x, gamma, beta, eps)
    np.testing.assert_allclose(y, torch.nn.functional.layer_norm(torch.from_numpy(x), (37,), torch.from_numpy(gamma), torch.from_numpy(beta), eps).numpy(), atol=1e-12)
    dx, dg, db = o8.layernorm_grad(x, gamma, mean, rstd, dy)
    h = 1e-6
    loss = lambda x_, g_, b_: (o8.layernorm(x_, g_, b_, eps)[0] * dy).sum()  # noqa: E731
    for _ in range(20):
        i, j = rng.integers(5), rng.integers(37)
        d = np.zeros_like(x)
        d[i, j] = h
        assert abs((loss(x + d, gamma, beta) - loss(x - d, gamma, beta)) / (2 * h) - dx[i, j]) < 1e-7
        d = np.zeros(37)
        d[j] = h
        assert abs((loss(x, gamma + d, beta) - loss(x, gamma - d, beta)) / (2 * h) - dg[j]) < 1e-7
        assert abs((loss(x, gamma, beta + d) - loss(x, gamma, beta - d)) / (2 * h) - db[j]) < 1e-7
    a = np.linspace(-9, 9, 400)
    np.testing.assert_allclose((o8.gelu(a + h) - o8.gelu(a - h)) / (2 * h), o8.gelu_slope(a), atol=1e-8)
