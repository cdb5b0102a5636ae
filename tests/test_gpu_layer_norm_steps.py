"""The norm's 8-bit values where they lie at or near the middle of two steps of e4m3.  A value is 448 u / top, u = s w, top the largest of its
block: with one rounding at the end it is off by 1 u at most (u = 2^-24 here) where s w needs no rounding, in bf16 or without w, else by 3 u,
and so equals the rounding of the exact value wherever that is farther from a middle; where it is the middle itself, the even one is taken."""
import pytest
import torch

from test_gpu_layer import BF, E4, F32, U, layer, rnd  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


def middles():
    """The middles between neighbouring finite e4m3 numbers of one sign, in 64 bits."""
    v = torch.arange(127, dtype=torch.uint8).view(E4).double()
    return (v[1:] + v[:-1]) / 2


@pytest.mark.parametrize("dt,weights,units", [(BF, True, 1), (BF, False, 1), (F32, True, 3), (F32, False, 1)])
@pytest.mark.parametrize("M,D", [(20000, 1024), (9000, 256), (30, 8192), (4, 4096)])
def test_values_between_two_steps(layer, M, D, dt, weights, units):  # noqa: F811
    x, w = rnd(1, M, D, dt=dt).cuda(), rnd(2, D, std=0.1, mean=1, dt=dt).cuda() if weights else None
    Q = layer.norm_fwd(x, w, eps=1e-5, y=False, fp8=True)[2]
    u = (x.double() * w.double() if weights else x.double()).view(M, -1, 128)
    exact = (u * 448 / u.abs().amax(2, keepdim=True)).view(M, D)
    mid = middles().cuda()
    i = torch.searchsorted(mid, exact.abs()).clamp(1, len(mid) - 1)
    off = torch.minimum((exact.abs() - mid[i]).abs(), (exact.abs() - mid[i - 1]).abs())
    sure = off > units * U * exact.abs() * (1 + 2.0 ** -20)
    if units == 1:
        sure |= off == 0
    want = exact.float().to(E4).double()      # (a middle is a float; what that rounding could move onto one is not sure)
    wrong = (Q.double() != want) & sure
    assert sure.double().mean() > 0.99 and not wrong.any(), (int(wrong.sum()), wrong.numel())
