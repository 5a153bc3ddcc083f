"""Layer norm at the magnitudes that its statistics are good for: values up to 1e16.

Tolerances as for rows of ordinary size (test_gpu_layer_norm): 64 u of what is added up covers a row's sums; a constant row's first
mean is off by 64 u of its value at most, and what is left of that by 64 u of itself, which the reciprocal deviation of a
row without spread, 1 / sqrt(eps), then multiplies."""
import pytest
import torch

from tests.test_gpu_layer_norm import BF16, DEV, F32, U, check_backward, check_forward, vectors

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    from paper_1910_02120_b200 import api as a
    return a


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [2, 7, 16, 24, 33, 64, 129, 1000, 1001, 4096, 8192, 16384, 40000, 65536, 70003])
def test_the_largest_rows(api, cols, dtype):
    gen = torch.Generator(device=DEV).manual_seed(cols)
    w, b = vectors(1, cols, gen)
    sign = torch.randint(0, 2, (6, cols), generator=gen, device=DEV) * 2.0 - 1.0
    x = torch.empty(6, cols, device=DEV)
    x[0], x[1] = 1e16 * sign[0], 1e16 * torch.rand(cols, generator=gen, device=DEV)
    x[2], x[3] = 0.0, -1e16
    x[2, 0], x[3, -1] = 1e16, 1e16                          # one value far from all others
    x[4], x[5] = 1e16 * sign[4] * torch.rand(cols, generator=gen, device=DEV), 1e8 * sign[5]
    x = x.to(dtype)
    y, mean, rstd = check_forward(api, x, w, b, y_dtype=F32)
    dy = torch.randn(6, cols, generator=gen, device=DEV) * 1e-3
    check_backward(api, dy, x, w, mean, rstd)


@pytest.mark.parametrize("cols", [3, 16, 24, 1000, 1001, 16384, 65536])
def test_the_largest_constant_rows(api, cols):
    gen = torch.Generator(device=DEV).manual_seed(cols)
    w, b = vectors(1, cols, gen)
    x = torch.tensor([1e16, -1e16, 9.87654321e15, 1.2345678e10], device=DEV)[:, None].expand(4, cols).contiguous()
    y, mean, rstd = api.ist_layer_norm_forward(x, w, b)
    step = x.double().abs()[:, :1] * 64 * U
    assert ((y.double() - b.double()).abs() <= w.double().abs() * step * 64 * U / 1e-5 ** 0.5 + 2 * U * b.double().abs()).all()
    assert ((mean.double() - x[:, 0].double()).abs() <= 2 * U * x[:, 0].double().abs()).all()
