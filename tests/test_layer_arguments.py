"""What the functions on tensors (paper_2504_00492_amd.layer) check of workspaces and streams, without a GPU: memory that a kernel could not
reach, or that is shorter than it counts, is refused before the library's call."""
import pytest
import torch

from test_layer_host import layer  # noqa: F401  (fixture)


def test_workspace_elsewhere(layer):  # noqa: F811
    with pytest.raises(ValueError, match="workspace must be on cuda:0"):
        layer._workspace(64, torch.empty(64, dtype=torch.uint8), torch.device("cuda:0"))


def test_workspace_in_pieces(layer):  # noqa: F811
    """A view that counts more bytes than it has, and one whose bytes are apart."""
    for t in (torch.empty(1, dtype=torch.uint8).expand(64), torch.empty(128, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError, match="workspace must be contiguous"):
            layer._workspace(64, t, torch.device("cpu"))
    whole = torch.empty(64, dtype=torch.float32)
    assert layer._workspace(64, whole, torch.device("cpu"))[1:] == (whole.data_ptr(), 256)


def test_stream_by_keyword(layer):  # noqa: F811
    """A stream's handle with all tensors by keyword, and with none."""
    x = torch.zeros(1, 4, 64)
    for call in (lambda: layer.gated_fwd(X=x, G=x, stream=0), lambda: layer.norm_fwd(X=x[0], eps=0., stream=5),
                 lambda: layer.matmul_fp8(A=x[0], sa=x, B=x[0], sb=x, stream=0), lambda: layer.quant_fp8(x[0], stream=0)):
        with pytest.raises(ValueError, match="no CPU path"):
            call()
    with pytest.raises(ValueError, match="no tensor"):
        layer.quant_fp8(X=None, stream=0)
