"""Gradients of the gated delta rule where its gates are strong, head by head against the definition in 64 bits.

The gradient of a token's log gate is a_t <R_t', S_{t-1}>: what reaches a later token, or the state behind, from an earlier one or the state
before, so it has the gate for a factor and is as small.  Tolerances are those of test_gpu_gated_delta, of each head's own gradients, since
every term of the sums carries that factor and none is a difference of larger ones: (d_k + 128) rounded sums and as much again in
fp32, and for bf16 the output's rounding and four operands of 16 bits."""
import pytest
import torch

import gated_delta_ref as ref
from test_gpu_gated_delta import DT, bound, f32_bound, layer, make, wide  # noqa: F401  (layer: fixture)

pytestmark = pytest.mark.gpu

GATES = (-0.1, -2.0, -5.0, -8.0, -12.0, -16.0, -30.0, -60.0)


def by_heads(layer, args, S0, dO, dSL, dk):  # noqa: F811
    got = layer.gated_delta_bwd(*args, dO, S0, dSL)
    want = ref.delta_grads(wide(*args, S0), *wide(dO, dSL))
    for name, a, b in zip(("dV", "dG", "dbeta"), got[2:5], want[2:5]):
        for h in range(b.shape[2]):
            tol, off = bound(a.dtype, dk), ref.off(a[:, :, h], b[:, :, h])
            assert off <= tol, (name, h, off, tol)
    return got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L,Hk,dk,dv", [(64, 8, 64, 64), (130, 4, 128, 32), (70, 8, 72, 40), (150, 2, 256, 64), (2100, 1, 64, 32)])
def test_each_head_a_gate_of_its_own(layer, L, Hk, dk, dv, dtype):  # noqa: F811
    """Around each of GATES; the last size is cut into segments and has two of them."""
    dt = DT[dtype]
    gates = GATES if L < 2000 else GATES[3:5]
    (Q, K, V, G, beta), S0, dO, dSL = make(1, L, Hk, len(gates), dk, dv, dt, seed=L)
    g = torch.Generator().manual_seed(L)
    G = (torch.tensor(gates, dtype=torch.float64) * (1 + 0.1 * torch.rand(1, L, len(gates), generator=g, dtype=torch.float64))).to(dt).cuda()
    by_heads(layer, (Q, K, V, G, beta), S0, dO, dSL, dk)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_gate_that_lets_nothing_through_has_no_gradient(layer, dtype):  # noqa: F811
    """At -256 and below a is 0, and so is its gradient: exactly, among gates of every strength, at a chunk's ends and in its middle, token upon token."""
    dt = DT[dtype]
    (Q, K, V, G, beta), S0, dO, dSL = make(2, 200, 2, 4, 64, 64, dt, seed=3)
    shut = torch.zeros(2, 200, 4, dtype=torch.bool)
    for t in (0, 1, 15, 16, 31, 47, 48, 63, 64, 100, 127, 128, 199):
        shut[:, t, t % 4] = shut[1, t, (t + 1) % 4] = True
    shut[0, 80:90, 2] = True
    G[shut.cuda()] = torch.tensor([-256.0, -300.0, -1e4, -float("inf")] * 200)[:int(shut.sum())].to(dt).cuda()
    got = by_heads(layer, (Q, K, V, G, beta), S0, dO, dSL, 64)
    assert not bool(got[3][shut.cuda()].any()) and bool((got[3][~shut.cuda()] != 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L,dk,dv", [(60, 64, 64), (100, 128, 32), (200, 256, 40), (40, 72, 16)])
def test_gradient_of_beta_where_the_state_knows_the_values(layer, L, dk, dv, dtype):  # noqa: F811
    """e_t = v_t - S k_t is 2^-12 of either, and dbeta_t = e_t.R k_t as small.  Keys are unit vectors, each token its own, g = 0 and beta a power of two or 0, so that
    e_t comes out exact in fp32, and what is left are the roundings that the tolerances count."""
    g, dt = torch.Generator().manual_seed(L), DT[dtype]
    n = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    i = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=g).double()  # noqa: E731
    Q, K = torch.nn.functional.normalize(n(1, L, 1, dk), dim=-1), torch.eye(dk, dtype=torch.float64)[torch.randperm(dk, generator=g)[:L]][None, :, None]
    V = i(-120, 121, 1, L, 1, dv) / 64
    e = (i(0, 2, L, dv) * 2 - 1) * (1 + i(0, 64, L, dv) / 64) * 2.0 ** -12
    beta = 2.0 ** -i(0, 3, 1, L, 1)
    beta[0, ::7] = 0
    S0 = 0.3 * n(1, 1, dv, dk)
    S0[0, 0] = torch.where(K[0, :, 0].sum(0) > 0, (V[0, :, 0] - e).t() @ K[0, :, 0], S0[0, 0])
    dO, dSL = n(1, L, 1, dv), n(1, 1, dv, dk)
    args = [t.to(dt).cuda() for t in (Q, K, V, torch.zeros(1, L, 1), beta)]
    dO, S0, dSL = dO.to(dt).cuda(), S0.float().cuda(), dSL.float().cuda()
    got = layer.gated_delta_bwd(*args, dO, S0, dSL)[4]
    want = ref.delta_grads(wide(*args, S0), *wide(dO, dSL))[4]
    some = beta[0, :, 0] > 0
    assert ref.off(got[0, some], want[0, some]) <= bound(dt, dk)
    # where beta is 0 the difference is taken of sums over d_v and pairs of tokens: its terms are |z| |v| at most, z = R k
    R = float(dSL.double().norm()) + float(dO.double().norm(dim=-1).sum())
    tol = (4 * 2.0 ** -17 if dtype == "bf16" else f32_bound(dk)) * R * float(V.norm(dim=-1).max()) + bound(dt, dk) * float(want[0, ~some].norm())
    assert float((got[0, ~some].double().cpu() - want[0, ~some]).norm()) <= tol


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("s", [0.5, 3.0])
def test_gates_above_zero(layer, s, dtype):  # noqa: F811
    """Sums of gates of a chunk up to s: the tolerances times e^s, as a chunk's products have e^s for a factor also where beta erases what the gates let grow."""
    dt = DT[dtype]
    (Q, K, V, _, beta), S0, dO, dSL = make(1, 130, 1, 2, 64, 32, dt, seed=5)
    beta[:, :, 1] = 1.0
    g = torch.Generator().manual_seed(5)
    G = (torch.rand(1, 130, 2, generator=g) * (s / 64)).to(dt).cuda()
    O, SL = layer.gated_delta_fwd(Q, K, V, G, beta, S0)
    grads = layer.gated_delta_bwd(Q, K, V, G, beta, dO, S0, dSL)
    wide_args = wide(Q, K, V, G, beta, S0)
    want = (*ref.delta(*wide_args), *ref.delta_grads(wide_args, *wide(dO, dSL)))
    for i, (a, b) in enumerate(zip((O, SL, *grads), want)):
        assert ref.off(a, b) <= bound(a.dtype, 64) * 2.718281828 ** s, i


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_token_by_token_gates_may_be_large(layer, dtype):  # noqa: F811
    """k = 1, beta = 1: every token erases what its gate of e^2 let grow, S_t = v_t, over any number of tokens."""
    dt = DT[dtype]
    V = torch.randn(2, 200, 1, 5, generator=torch.Generator().manual_seed(1)).to(dt).cuda()
    one, two, S = (torch.full(s, v, dtype=t, device="cuda") for s, v, t in (((2, 1, 1), 1.0, dt), ((2, 1), 2.0, dt), ((2, 1, 5, 1), 0.0, torch.float32)))
    for t in range(200):
        o = layer.gated_delta_step(one, one, V[:, t], two, one[..., 0], S)
        # v - a S + a S: three roundings of a S, at most e^2 times the token's before
        tol = 4 * 2.0 ** -24 * 7.39 * float(V.abs().max()) * 2
        assert float((S[..., 0] - V[:, t].float()).abs().max()) <= tol and float((o.float() - V[:, t].float()).abs().max()) <= tol + 2.0 ** -8 * float(V.abs().max())
