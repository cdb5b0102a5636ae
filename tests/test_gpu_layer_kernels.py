"""The gated recurrence of one sequence alone and among a thousand others, which other kernels take (tiles, tiles of which more are listened to;
a workgroup to a chain, over many rounds): each within the bounds of test_gpu_layer.py, and all the others alike."""
import pytest
import torch

from test_gpu_layer import BF, F32, HALF, gated_grads, gated_ref, gates, layer, near, rnd  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

MANY = 1030


def near_all(got, want, halves):
    for out, (ref, tol), half in zip(got, want, halves):
        near(out[:1], ref, tol + half * ref.abs())
        assert torch.equal(out, out[:1].expand_as(out))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("gate,mix", [("value", False), ("log", True), ("logit", True)])
@pytest.mark.parametrize("L,D", [(257, 16), (700, 5), (3001, 16), (12500, 8)])
def test_alone_and_among_many(layer, L, D, gate, mix, dt):  # noqa: F811
    x, g, h0 = rnd(1, 1, L, D, dt=dt), gates(2, 1, L, D, gate, dt), rnd(3, 1, D)
    y, dy, dh = rnd(4, 1, L, D, dt=dt), rnd(5, 1, L, D, dt=dt), rnd(6, 1, D)
    ref, tol = gated_ref(x, g, h0, gate, mix)
    fwd, bwd = ((ref, tol), (ref[:, -1], tol[:, -1])), gated_grads(x, g, h0, y, dy, dh, gate, mix)
    for B in (1, MANY):
        shared = lambda t: t.cuda().expand(B, *t.shape[1:])  # noqa: E731
        h, d = shared(h0).contiguous(), shared(dh).contiguous()
        near_all(layer.gated_fwd(shared(x), shared(g), h, gate=gate, mix=mix), fwd, (HALF[dt], 0))
        back = layer.gated_bwd(shared(x) if mix else None, shared(g), shared(y).contiguous(), shared(dy), h, d, gate=gate, mix=mix)
        near_all(back, bwd, (HALF[dt], HALF[dt], 0))
