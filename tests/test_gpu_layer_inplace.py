"""Outputs of include/pf_layer.h that may lie in the place of inputs: the same bits as into arrays of their own."""
import pytest
import torch

from test_gpu_layer import BF, EPS, F32, gates, layer, rnd  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

CODE = {F32: 0, BF: 1}


def gated_calls(layer, B, L, D, dt):
    """(forward, backward) as functions of the buffers in which a state comes in and goes out."""
    x, g, y, dy = rnd(1, B, L, D, dt=dt).cuda(), gates(2, B, L, D, "log", dt).cuda(), rnd(4, B, L, D, dt=dt).cuda(), rnd(5, B, L, D, dt=dt).cuda()
    need = layer.pf_gated_workspace_bytes(B, L, D, CODE[dt])
    work = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    h0 = rnd(7, B, D).cuda()

    def forward(h, hL):
        Y = torch.empty_like(x)
        assert layer.pf_gated_fwd(x, L * D, D, g, L * D, D, h, Y, hL, B, L, D, 1, 0, CODE[dt], work, need) == 0
        return Y, hL

    def backward(dhL, dh0):
        dX, dG = torch.empty_like(x), torch.empty_like(x)
        assert layer.pf_gated_bwd(x, L * D, D, g, L * D, D, h0, y, dy, L * D, D, dhL, dX, dG, dh0, B, L, D, 1, 1, CODE[dt], work, need) == 0
        return dX, dG, dh0
    return forward, backward


# a few tokens; a workgroup to a chain, one and several rounds, and with many chains; tiles, two of them to many, and where more in
# front are listened to
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("B,L,D", [(5, 9, 130), (3, 60, 70), (2, 256, 64), (1024, 600, 8), (2, 257, 260), (1, 300, 1024), (3, 700, 1000), (40, 2000, 64),
                                   (1, 20000, 64)])
def test_gated_state_in_place(layer, B, L, D, dt):  # noqa: F811
    for call in gated_calls(layer, B, L, D, dt):
        state = rnd(3, B, D).cuda()
        want = call(state, torch.empty_like(state))
        for _ in range(3):
            here = state.clone()
            for a, b in zip(call(here, here), want):
                assert torch.equal(a, b)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("M,D", [(1, 64), (33, 128), (70, 1000), (9, 4096), (600, 2048), (5, 8200)])
def test_norm_in_place(layer, M, D, dt):  # noqa: F811
    x, r, w = rnd(1, M, D, dt=dt).cuda(), rnd(2, M, D, dt=dt).cuda(), rnd(3, D, dt=dt).cuda()
    S, Y = torch.empty_like(x), torch.empty_like(x)

    def call(x, r, S):
        assert layer.pf_norm_fwd(x, D, r, D, w, S, Y, None, 0, None, M, D, EPS, CODE[dt]) == 0
        return Y.clone(), S.clone()
    want = call(x, r, S)
    here, there = x.clone(), r.clone()
    for got in (call(here, r, here), call(x, there, there)):
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("M,D", [(1, 64), (33, 128), (70, 1000), (9, 4096), (600, 2048), (5, 8200)])
def test_norm_backward_in_place(layer, M, D, dt):  # noqa: F811
    s, dy, ds, w = rnd(1, M, D, dt=dt).cuda(), rnd(2, M, D, dt=dt).cuda(), rnd(4, M, D, dt=dt).cuda(), rnd(3, D, dt=dt).cuda()
    need = layer.pf_norm_bwd_workspace_bytes(M, D)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")

    def call(dy, ds, dx):
        dw = torch.empty(D, device="cuda")
        assert layer.pf_norm_bwd(s, D, w, dy, D, ds, D, dx, dw, M, D, EPS, CODE[dt], work, need) == 0
        return dx.clone(), dw
    want = call(dy, ds, torch.empty_like(dy))
    here, there = dy.clone(), ds.clone()
    for got in (call(here, ds, here), call(dy, there, there)):
        assert all(torch.equal(a, b) for a, b in zip(got, want))
