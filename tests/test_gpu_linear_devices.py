"""Layers and their gradient on more devices than there are columns: those without any have null buffers."""
import pytest

from test_gpu_linear import Layer, check_grad

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m", [1, 3, 9, 40, 300])
@pytest.mark.parametrize("n,k", [(3, 4), (1, 2), (5, 8), (9, 64)])
@pytest.mark.parametrize("x", ["bf16", "f32"])
def test_fewer_columns_than_devices(m, n, k, x):
    for w_trans, x_trans, kk in ((1, 0, 1500), (0, 0, 1500), (1, 0, 20), (0, 1, 77), (1, 1, 640)):
        Layer(m, kk, n, k, "S1", x=x, residual="f32", pre="bf16", gelu=kk == 1500, w_trans=w_trans, x_trans=x_trans, pitch=3 if kk == 77 else 0).check()


@pytest.mark.parametrize("rows", [1, 100, 3000])
@pytest.mark.parametrize("gelu", [False, True])
def test_gradient_of_fewer_columns_than_devices(rows, gelu):
    for n, k in ((3, 4), (9, 64)):
        check_grad(rows, n, k, "S1", gelu=gelu)
        check_grad(rows, n, k, "S1", y="f32", pre="e4m3", gelu=gelu, pitch=1)


@pytest.mark.parametrize("gelu", [False, True])
def test_gradient_of_fewer_rows_than_devices(gelu):
    for y in ("bf16", "f32"):
        check_grad(3, 300, 8, "S0", y=y, gelu=gelu)
