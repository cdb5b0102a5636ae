"""Workspaces handed to the functions on tensors: right ones serve, such that the kernels could not use are refused."""
import pytest
import torch

from test_gpu_layer import BF, EPS, e4m3, gates, layer, rnd  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


def calls(layer):
    x, g = rnd(1, 2, 1000, 64, dt=BF).cuda(), gates(2, 2, 1000, 64, "log", BF).cuda()
    A, B = e4m3(1, 200, 4096)[0], e4m3(2, 128, 4096)[0]
    sa, sb = torch.ones(32, 200, device="cuda"), torch.ones(32, 128, device="cuda")
    return (lambda **k: layer.gated_fwd(x, g, **k), lambda **k: layer.gated_bwd(None, g, x, x, **k),
            lambda **k: layer.norm_bwd(x[0], x[1], eps=EPS, **k), lambda **k: (layer.matmul_fp8(A, sa, B, sb, b_rows=1, **k),))


def test_workspace_handed_in(layer):  # noqa: F811
    work = torch.empty(1 << 25, dtype=torch.uint8, device="cuda")
    for call in calls(layer):
        want = call()
        assert all(torch.equal(a, b) for a, b in zip(call(workspace=work), want))
        for wrong in (torch.empty(1 << 25, dtype=torch.uint8), work[:1].expand(1 << 25), work[::2]):
            with pytest.raises(ValueError, match="workspace"):
                call(workspace=wrong)
