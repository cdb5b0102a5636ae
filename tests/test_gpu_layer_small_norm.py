"""The norm in 8 bits where rows, or blocks of 128 columns of them, are zero or nearly so and eps is small: 1 / sqrt(mean + eps) is then a
million and more.  Definitions and bars of test_gpu_layer.py."""
import pytest
import torch

from test_gpu_layer import BF, F32, HALF, U, check_e4m3, layer, near, rnd  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("eps", [1e-5, 1e-12, 1e-20, 0.0])
@pytest.mark.parametrize("D", [100, 256, 1000, 4100])
def test_norm_of_next_to_nothing(layer, D, eps, dt):  # noqa: F811
    x = rnd(1, 9, D) * torch.tensor([1.0, 1e-7, 1e-7, 1e-7, 1e-9, 1e-9, 1e-15, 1e10, 0.0]).view(9, 1)
    if D > 128:
        for row, size in ((1, 0.0), (2, 1e-36), (3, 1e-38), (4, 0.0), (5, 1e-30), (6, 1e-25), (7, 1e-25)):
            x[row, :128] = rnd(2, 128) * size
    if eps == 0:
        x = x[:8]      # (a row of zeros gives NaN)
    x = x.to(dt)
    w = rnd(3, D, std=0.1, mean=1).to(dt)
    y = x.double() / ((x.double() ** 2).mean(1, keepdim=True) + eps).sqrt() * w.double()
    _, Y, Q, scale = layer.norm_fwd(x.cuda(), w.cuda(), eps=eps, fp8=True)
    near(Y, y, y.abs() * (64 * U + HALF[dt]) + 2.0 ** -126)
    assert Q.float().isfinite().all()
    check_e4m3(Q, scale, y)
