"""The gates themselves, in fp32, for gates of every size: one token from a state of one.  The exponential is the instruction's, off by one
unit of its result (2 u, u = 2^-24), put right for the rounding of g log2 e and rounded once more: 4 u; the logistic forms add a sum, a reciprocal
with one step of Newton and a product: 8 u."""
import pytest
import torch

from test_gpu_layer import U, gate_ref, layer, near  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gate,units", [("log", 4), ("logit", 8)])
@pytest.mark.parametrize("top", [1.0, 5.0, 20.0, 86.0])
def test_gates_in_fp32(layer, top, gate, units):  # noqa: F811
    B, D = 3, 4096
    g = (torch.rand(B, 1, D, generator=torch.Generator().manual_seed(1)) * 2 - 1) * top
    zero, one = torch.zeros(B, 1, D).cuda(), torch.ones(B, D).cuda()
    a, _, slope = gate_ref(g.double(), gate)
    Y, hL = layer.gated_fwd(zero, g.cuda(), one, gate=gate)
    near(Y, a, units * U * a)
    near(hL, a[:, 0], units * U * a[:, 0])
    dX, dG, dh0 = layer.gated_bwd(None, g.cuda(), zero, one.view(B, 1, D), one, gate=gate)
    assert (dX == 1).all()
    near(dG, slope, (units + 8 * (gate == "logit")) * U * slope + 2.0 ** -149)
    near(dh0, a[:, 0], units * U * a[:, 0])


def test_infinite_gates_in_fp32(layer):  # noqa: F811
    g = torch.tensor([float("-inf"), float("inf"), -1e30, 1e30, -200.0, float("nan")]).view(1, 1, 6).cuda()
    one = torch.ones(1, 6).cuda()
    a = layer.gated_fwd(torch.zeros_like(g), g, one)[1][0].cpu()
    assert a[[0, 2, 4]].eq(0).all() and a[[1, 3]].eq(float("inf")).all() and a[5].isnan()
    a = layer.gated_fwd(torch.zeros_like(g), g, one, gate="logit")[1][0].cpu()
    assert a[[0, 2, 4]].eq(0).all() and a[[1, 3]].eq(1).all() and a[5].isnan()
