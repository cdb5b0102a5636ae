"""The gated recurrence where the product of some tokens' gates is far outside fp32 and no state is: growth and decay that take each
other back, and gates of zero behind gates that grow.  Formulas and error bounds in 64 bits are those of test_gpu_layer.py; every state
and every step of the bounds stays inside fp32's normal range, so they hold as they are."""
import pytest
import torch

from test_gpu_layer import BF, F32, HALF, gate_ref, gated_grads, gated_ref, layer, near, rnd  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

# a few tokens; a workgroup to a chain: one round, two, and several with many chains; tiles; tiles of which more are listened to
SHAPES = [(2, 12, 70), (2, 60, 130), (1, 250, 33), (1024, 600, 4), (3, 600, 72), (1, 3000, 33), (2, 1700, 260), (1, 20000, 64)]


def pattern(case, B, L, D):
    """Logarithms (base 2) of the gates [B, L, D] (minus infinity: zero), the size of what is added at each token, the incoming state."""
    n = min(145, L // 3)
    if case == "reset":      # 2^66 twice, then zero, behind a state of 2^-100; nothing is added before that
        lg, x = torch.zeros(L), torch.ones(L)
        at = L // 2 if L < 1000 else L // 2 // 224 * 224 + 3
        lg[:at], lg[at:at + 2], lg[at + 2], lg[at + 3:] = 0, 66, float("-inf"), -0.2
        x[:at + 2] = 0
        return lg.view(1, L, 1).expand(B, L, D), x, 2.0 ** -100
    # up (or down) over n tokens, as it is over some, and back
    whole, x, h = {"up": (140.0, 1e-7, 1e-6), "down": (-170.0, 1e-23, 1e30)}[case]
    flat, lg = min(400, (L - 2 * n) // 2), torch.zeros(L)
    lg[:n], lg[n + flat:2 * n + flat] = whole / n, -whole / n
    lg = lg.roll(min(100, L - 2 * n - flat))
    return lg.view(1, L, 1) * (1 + 0.01 * rnd(9, B, 1, D).clamp(-1, 1)), torch.full((L,), x), h


def inputs(case, B, L, D, gate, dt):
    lg, x, h = pattern(case, B, L, D)
    G = (lg * 0.6931471805599453 if gate == "log" else torch.exp2(lg)).to(dt)
    return rnd(1, B, L, D).mul(x.view(1, L, 1)).to(dt), G, torch.full((B, D), h) * (1 + 0.1 * rnd(3, B, D).clamp(-1, 1))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("case,gate,mix", [(c, g, m) for c in ("up", "down", "reset") for g, m in (("value", False), ("value", True), ("log", False))
                                           if not (c == "reset" and m)])      # (what the mix adds at a gate of 2^66 is of that size)
@pytest.mark.parametrize("B,L,D", SHAPES)
def test_gated_products_outside_fp32(layer, B, L, D, case, gate, mix, dt):  # noqa: F811
    x, g, h0 = inputs(case, B, L, D, gate, dt)
    ref, tol = gated_ref(x, g, h0, gate, mix)
    assert ref.abs().max() < 2.0 ** 126
    Y, hL = layer.gated_fwd(x.cuda(), g.cuda(), h0.cuda(), gate=gate, mix=mix)
    near(Y, ref, tol + HALF[dt] * ref.abs())
    near(hL, ref[:, -1], tol[:, -1])


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("gate,mix", [("value", False), ("value", True), ("log", False)])
@pytest.mark.parametrize("case", ["up", "down", "reset"])
@pytest.mark.parametrize("B,L,D", SHAPES)
def test_gated_backward_products_outside_fp32(layer, B, L, D, case, gate, mix, dt):  # noqa: F811
    """The same gates from the other end."""
    dy, g, dh = inputs(case, B, L, D, gate, dt)
    dy, g = dy.flip(1), g.flip(1)
    x, y, h0 = rnd(5, B, L, D, dt=dt), rnd(6, B, L, D, dt=dt), rnd(7, B, D)
    got = layer.gated_bwd(x.cuda() if mix else None, g.cuda(), y.cuda(), dy.cuda(), h0.cuda(), dh.cuda(), gate=gate, mix=mix)
    want = list(gated_grads(x, g, h0, y, dy, dh, gate, mix))
    if mix:      # that bound takes 1 - a for its size, and here it is below zero: db's bound times the size
        (db, tol), rest = gated_grads(x, g, h0, y, dy, dh, gate, False)[0], gate_ref(g.double(), gate)[1]
        want[0] = db * rest, tol * rest.abs()
    for out, (ref, tol), half in zip(got, want, (HALF[dt], HALF[dt], 0)):
        assert ref.abs().max() < 2.0 ** 126
        near(out, ref, tol + half * ref.abs())
