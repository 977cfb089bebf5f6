"""sbp_linear with operands of 4 GiB and more, whose bytes the matrix kernels cannot count in 32 bits, and with more rows than the second dimension of a grid holds.

Operands, bias and residual are small whole numbers, so that every sum is a whole number below 2^24 and fp32 results are exact in any order of adding."""
import pytest
import torch

import paper_2110_15032_amd as sbp
from train_harness import CODE, TYPE

pytestmark = pytest.mark.gpu


def whole(rows, cols, kind="bf16", most=2):
    return torch.randint(-most, most + 1, (rows, cols), dtype=torch.int8, device="cuda").to(TYPE[kind])


def stored(t, rows, cols, kind, trans=0):
    return sbp.SbpTensor(t if isinstance(t, list) else [t], rows, cols, CODE[kind], trans)


def product(x, w, x_trans, w_trans, rows, cols):
    """rows x cols places of x w in fp32, the places as index tensors"""
    a = (x[:, rows].T if x_trans else x[rows]).float()
    b = (w[cols].T if w_trans else w[:, cols]).float()
    return a @ b


@pytest.mark.parametrize("m,kk,n,x_trans,w_trans", [
    (1100000, 2048, 72, 0, 1),         # x of 4.5 GB along the reduction, and more rows than 65535 x 16
    (1100000, 2048, 72, 0, 0),
    (66, 8192, 262144 + 133, 0, 1),    # w of 4.3 GB along the reduction
    (66, 8192, 262144 + 133, 0, 0),    # ... along the columns
    (1100000, 2050, 9, 0, 1),          # rows at any alignment
    (1100008, 2048, 40, 1, 1),         # x of 4.5 GB along its rows
    (1050000, 2176, 520, 0, 1),        # the largest tiles
    (1050000, 2176, 520, 1, 0),
])
def test_operands_of_four_gigabytes(m, kk, n, x_trans, w_trans):
    x = whole(kk, m) if x_trans else whole(m, kk)
    w = whole(n, kk) if w_trans else whole(kk, n)
    bias, res = whole(n, 1, "f32", 9), whole(m, n, "bf16", 9)
    pre, y = (torch.full((m, n), float("nan"), dtype=torch.float32, device="cuda") for _ in range(2))
    sbp.sbp_linear(stored(x, m, kk, "bf16", x_trans), sbp.B, stored(w, kk, n, "bf16", w_trans), sbp.B, stored(bias, n, 1, "f32"), stored(res, m, n, "bf16"), stored(pre, m, n, "f32"),
                   stored(y, m, n, "f32"), sbp.AUTO, 1)
    assert torch.equal(y - res.float(), pre) and not bool(pre.isnan().any())
    step = 1 << 16
    for r in range(0, m, step):
        rows = torch.arange(r, min(r + step, m), device="cuda")
        for c in range(0, n, step):
            cols = torch.arange(c, min(c + step, n), device="cuda")
            assert torch.equal(pre[r:r + step, c:c + step], product(x, w, x_trans, w_trans, rows, cols) + bias[cols, 0]), (r, c)


def test_four_gigabytes_on_devices():
    """ranges that a device has fewer rows for than another, and GeLU with bf16 results"""
    m, kk, n, k = 2100003, 2048, 24, 2
    half = (m + 1) // 2
    x, w = whole(m, kk), whole(n, kk, most=1)
    pre, y = torch.empty(m, n, dtype=torch.bfloat16, device="cuda"), torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    cut = lambda t: [t[:half].clone(), t[half:].clone()] if t is not x else [x[:half], x[half:]]  # noqa: E731
    pres, ys = cut(pre), cut(y)
    sbp.sbp_linear(stored(cut(x), m, kk, "bf16"), sbp.S(0), stored([w, w], kk, n, "bf16", 1), sbp.B, None, None, stored(pres, m, n, "bf16"), stored(ys, m, n, "bf16"), sbp.AUTO, k, None, sbp.EPI_GELU)
    for part, p, v in zip(cut(x), pres, ys):
        for r in range(0, part.shape[0], 1 << 16):
            a = part[r:r + (1 << 16)].float() @ w.T.float()
            assert torch.equal(p[r:r + (1 << 16)], a.to(torch.bfloat16))
            want = torch.nn.functional.gelu(a.double())
            # 2.2e-5 of its value, one rounding to bf16, and what torch's erf leaves of the far tail (2^-53 of the argument)
            assert bool(((v[r:r + (1 << 16)].double() - want).abs() <= (2.2e-5 + 2.0 ** -8) * 1.01 * want.abs() + 1e-14).all())


def test_more_rows_than_a_grid_of_tiles_or_elements():
    """tall and narrow: tiles of 64 rows would be 2^32 threads and more, single elements more than 65535 workgroups along the rows"""
    m = 2 ** 30 + 70
    x = whole(m, 1)
    y = torch.full((m, 1), float("nan"), dtype=torch.bfloat16, device="cuda")
    w = torch.full((1, 1), 3.0, dtype=torch.bfloat16, device="cuda")
    sbp.sbp_linear(stored(x, m, 1, "bf16"), sbp.B, stored(w, 1, 1, "bf16"), sbp.B, None, None, None, stored(y, m, 1, "bf16"), sbp.AUTO, 1)
    assert torch.equal(y, 3 * x)


def test_rows_of_x_that_are_too_long_for_the_matrix_kernels():
    """x stored along its rows, each of more than 2^22 elements, 4 GiB in all"""
    m, kk, n = 2 ** 22 + 77, 513, 5
    x, w, res = whole(kk, m), whole(kk, n), whole(m, n, "f32", 9)
    y = torch.full((m, n), float("nan"), dtype=torch.float32, device="cuda")
    sbp.sbp_linear(stored(x, m, kk, "bf16", 1), sbp.B, stored(w, kk, n, "bf16"), sbp.B, None, stored(res, m, n, "f32"), None, stored(y, m, n, "f32"), sbp.AUTO, 1)
    for r in range(0, m, 1 << 18):
        assert torch.equal(y[r:r + (1 << 18)] - res[r:r + (1 << 18)], x[:, r:r + (1 << 18)].T.float() @ w.float())


@pytest.mark.parametrize("m,kk,n,x_trans,w_trans", [(530000, 2051, 72, 0, 1), (530000, 2048, 260, 1, 0), (70, 8192, 131072 + 133, 0, 1), (70, 8192, 131072 + 133, 0, 0), (3, 8192, 131072 + 133, 0, 1)])
def test_fp32_operands_of_four_gigabytes(m, kk, n, x_trans, w_trans):
    x, w = (whole(kk, m, "f32") if x_trans else whole(m, kk, "f32")), (whole(n, kk, "f32") if w_trans else whole(kk, n, "f32"))
    res = whole(m, n, "bf16", 9)
    y = torch.full((m, n), float("nan"), dtype=torch.float32, device="cuda")
    sbp.sbp_linear(stored(x, m, kk, "f32", x_trans), sbp.B, stored(w, kk, n, "f32", w_trans), sbp.B, None, stored(res, m, n, "bf16"), None, stored(y, m, n, "f32"), sbp.AUTO, 1)
    step = 1 << 16
    for r in range(0, m, step):
        rows = torch.arange(r, min(r + step, m), device="cuda")
        for c in range(0, n, step):
            cols = torch.arange(c, min(c + step, n), device="cuda")
            assert torch.equal(y[r:r + step, c:c + step] - res[r:r + step, c:c + step].float(), product(x, w, x_trans, w_trans, rows, cols)), (r, c)
