"""Workspaces and streams handed to the functions on tensors: right ones serve, such that the kernels could not use are refused."""
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


def test_stream_by_keyword(layer):  # noqa: F811
    """A stream, or its handle, with all tensors given by keyword."""
    x, g = rnd(1, 2, 400, 64, dt=BF).cuda(), gates(2, 2, 400, 64, "log", BF).cuda()
    want, grads = layer.gated_fwd(x, g), layer.gated_bwd(None, g, x, x)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    for stream in (other, other.cuda_stream, 0):
        got = (*layer.gated_fwd(X=x, G=g, stream=stream), *layer.gated_bwd(X=None, G=g, Y=x, dY=x, stream=stream))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (*want, *grads)))


def test_stream_of_another_device(layer):  # noqa: F811
    class Elsewhere:
        device = torch.device("cuda", 99)
    x = torch.zeros(1, 4, 64, device="cuda")
    with pytest.raises(ValueError, match="stream must be one of cuda:0"):
        layer.gated_fwd(x, x, stream=Elsewhere())
