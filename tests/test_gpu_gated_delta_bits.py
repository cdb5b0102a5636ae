"""How many bits the gated delta rule keeps with bf16 inputs: 24 of states and of their gradients, 16 at least of what enters the other outputs.

Whole numbers, unit gates (g = 0) and keys that have few entries make every exact result a whole number too, and every product and sum of 24 (16) bits
exact: so results are equal to those in 64 bits where the bits are kept, and off by hundreds where they are not, by up to 2^-17 of numbers of
24 bits with two bf16 parts in the place of three, 2^-9 of numbers of 16 bits with one in the place of two.  Outputs in bf16 are small differences of
large terms, so that their own rounding takes nothing."""
import pytest
import torch

import gated_delta_ref as ref
from test_gpu_gated_delta import layer, wide  # noqa: F401  (layer: fixture)

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def whole(*shape, most, g):
    return torch.randint(-most, most + 1, shape, generator=g).double()


def tokens(L, Hv, dk, dv, g, busy):
    """Q, K, V, G, beta [1, L, ..] of zeros but at the busy tokens: keys of two entries of 1 or -1 out of the first half of d_k, small whole values."""
    Q, K, V, G, beta = (torch.zeros(1, L, *s, dtype=torch.float64) for s in ((1, dk), (1, dk), (Hv, dv), (Hv,), (Hv,)))
    half = max(2, dk // 2)
    for t in busy:
        for X in (Q, K):
            X[0, t, 0, torch.randperm(half, generator=g)[:2]] = (torch.randint(0, 2, (2,), generator=g) * 2 - 1).double()
        V[0, t], beta[0, t] = whole(Hv, dv, most=100, g=g), 1.0
    return Q, K, V, G, beta


@pytest.mark.parametrize("L,Hv,dk,dv", [(8, 1, 64, 16), (64, 2, 128, 40), (130, 2, 64, 32), (90, 1, 256, 16), (70, 1, 72, 16), (2100, 1, 64, 32)])
def test_states_and_their_gradients_keep_24_bits(layer, L, Hv, dk, dv):  # noqa: F811
    """Eight tokens change the state (|v - S k| stays within 2^24 then), before and behind chunks' ends and, in the last size, in several segments."""
    g = torch.Generator().manual_seed(L + dk)
    busy = range(8) if L == 8 else [2, 3, 40, 60, 61, 62, 63, L - 1] if L < 128 else [2, 60, 63, 64, 65, 100, L - 2, L - 1]
    Q, K, V, G, beta = tokens(L, Hv, dk, dv, g, busy)
    S0, dSL, dO = whole(1, Hv, dv, dk, most=1 << 18, g=g), whole(1, Hv, dv, dk, most=1 << 18, g=g), whole(1, L, Hv, dv, most=3, g=g)
    S0[..., -1], dSL[..., -1] = (1 << 23) + 1, -(1 << 23) - 1      # (a column that no key touches)
    args = [t.to(BF).cuda() for t in (Q, K, V, G, beta)]
    s0, dsl = S0.float().cuda(), dSL.float().cuda()
    want = ref.delta(Q, K, V, G, beta, S0)[1]
    back = ref.delta_grads([Q, K, V, G, beta, S0], dO, dSL)[5]
    assert float(want.abs().max()) < 1 << 24 and float(back.abs().max()) < 1 << 24 and float(want[..., :-1].abs().max()) > 1 << 17
    got = layer.gated_delta_fwd(*args, s0)[1]
    assert torch.equal(got.double().cpu(), want)
    assert torch.equal(layer.gated_delta_bwd(*args, dO.to(BF).cuda(), s0, dsl)[5].double().cpu(), back)


@pytest.mark.parametrize("dk,dv", [(64, 16), (128, 40), (256, 16), (72, 16)])
def test_outputs_keep_16_bits(layer, dk, dv):  # noqa: F811
    """Out of the state alone, out of the state and what the tokens write, and out of pairs of tokens."""
    g = torch.Generator().manual_seed(dk)
    L = 70
    Q, K, V, G, beta = (torch.zeros(1, L, *s, dtype=torch.float64) for s in ((1, dk), (1, dk), (1, dv), (1,), (1,)))
    S0 = torch.zeros(1, 1, dv, dk, dtype=torch.float64)
    S0[0, 0, :, 0] = whole(dv, most=(1 << 16) - 256, g=g)
    S0[0, 0, :, 1] = S0[0, 0, :, 0] + whole(dv, most=100, g=g)
    Q[0, 3, 0, 0], Q[0, 3, 0, 1] = 1, -1                                # S of 16 bits
    S0[0, 0, :, 2] = whole(dv, most=(1 << 15) - 256, g=g)
    V[0, 5], beta[0, 5], K[0, 5, 0, 2] = whole(1, dv, most=100, g=g), 1, 1
    for t in (5, 9, 20, 63, 64):
        Q[0, t, 0, 2] = 1                                               # S q and u = v - S k of 16 bits, far above their sum
    K[0, 10, 0, 4:6], K[0, 11, 0, 6] = torch.tensor([200.0, 1.0], dtype=torch.float64), -200
    Q[0, 40, 0, 4:7] = torch.tensor([200.0, 1.0, 200.0], dtype=torch.float64)      # q.k = 40001 and -40000
    V[0, 10:12], beta[0, 10:12] = 1, 1
    args = [t.to(BF).cuda() for t in (Q, K, V, G, beta)]
    want = ref.delta(Q, K, V, G, beta, S0)[0]
    assert float(want.abs().max()) <= 200 and all(bool(want[0, t].any()) for t in (3, 5, 64, 40)) and bool((want[0, 40] == 1).all())
    assert torch.equal(layer.gated_delta_fwd(*args, S0.float().cuda())[0].double().cpu(), want)


@pytest.mark.parametrize("dk", [64, 128, 256, 72])
def test_gradients_keep_16_bits(layer, dk):  # noqa: F811
    """One token behind a state, with k = e_0 and beta = 1: u = v - S k, z = R k, dk = R^T u - S^T z, dbeta = z.u, dg = <R, S> - z.S k, and
    dq = S^T do + (u.do) k, each of two terms of 16 bits that leave a few units (dk in the columns behind the first)."""
    dv = 16

    def one(v, S, R, q, do):
        """First two rows of v, S and R given, S and R by columns."""
        Q, K, V, dO = (torch.zeros(1, 1, 1, n, dtype=torch.float64) for n in (dk, dk, dv, dv))
        G, beta = torch.zeros(1, 1, 1, dtype=torch.float64), torch.ones(1, 1, 1, dtype=torch.float64)
        S0, dSL = torch.zeros(1, 1, dv, dk, dtype=torch.float64), torch.zeros(1, 1, dv, dk, dtype=torch.float64)
        K[..., 0] = 1
        V[..., :2], dO[..., :2] = torch.tensor(v).double(), torch.tensor(do).double()
        Q[..., :len(q)] = torch.tensor(q).double()
        for X, x in ((S0, S), (dSL, R)):
            X[0, 0, :2, :len(x[0])] = torch.tensor(x).double()
        want = ref.delta_grads([Q, K, V, G, beta, S0], dO, dSL)
        low = [t.to(BF).cuda() for t in (Q, K, V, G, beta)]
        got = layer.gated_delta_bwd(*low, dO.to(BF).cuda(), S0.float().cuda(), dSL.float().cuda())
        return [t.double().cpu() for t in got], want

    # u = (40001, 1), z = (1, 39999): dk_1 = 40001 - 39999 + 40001 - 39999
    got, want = one([1, 1], [[-40000, 39999], [0, 1]], [[1, 1], [39999, 40001]], [0], [0, 0])
    assert float(want[1][0, 0, 0, 1]) == 4 and torch.equal(got[1][..., 1:], want[1][..., 1:])
    # v of 16 bits as bf16 has them, S k beside it: dbeta = 40192 - 40190 + 2 (300 * 128 - 38399)
    got, want = one([40192, 300 * 128], [[40190], [38399]], [[1], [2]], [0], [0, 0])
    assert float(want[4]) == 4 and torch.equal(got[4], want[4])
    # R k = 1, S k = 40001 and its neighbour's 3
    got, want = one([0, 0], [[40001, 3], [-20001, 2]], [[1, 1], [2, 1]], [0], [0, 0])
    assert float(want[3]) == 5 and torch.equal(got[3], want[3])
    # q = k: dq_0 = 40001 + (3 - 40001), dq_1 of rows that differ by one
    got, want = one([3, 0], [[40001, 20001], [0, 20000]], [[0], [0]], [1], [1, 0])
    assert float(want[0][0, 0, 0, 0]) == 3 and torch.equal(got[0][..., :1], want[0][..., :1])
    got, want = one([0, 0], [[0, 40001], [0, 40000]], [[0], [0]], [0], [1, -1])
    assert float(want[0][0, 0, 0, 1]) == 1 and torch.equal(got[0], want[0])


@pytest.mark.parametrize("dk", [64, 128, 256])
def test_gradients_of_pairs_of_tokens_keep_16_bits(layer, dk):  # noqa: F811
    """Two tokens, q_2 = k_1 = e_0 and k_2 = e_1: what the second reads of what the first wrote, u_1 = 40001, and of the state, -40000 beside it."""
    dv = 16
    Q, K, V, dO = (torch.zeros(1, 2, 1, n, dtype=torch.float64) for n in (dk, dk, dv, dv))
    G, beta = torch.zeros(1, 2, 1, dtype=torch.float64), torch.ones(1, 2, 1, dtype=torch.float64)
    S0 = torch.zeros(1, 1, dv, dk, dtype=torch.float64)
    K[0, 0, 0, 0] = K[0, 1, 0, 1] = Q[0, 1, 0, 0] = 1
    V[0, 0, 0, 0], S0[0, 0, 0, 0] = 1, -40000
    dO[0, 1, 0, 0] = 1
    want = ref.delta_grads([Q, K, V, G, beta, S0], dO, torch.zeros_like(S0))
    low = [t.to(BF).cuda() for t in (Q, K, V, G, beta)]
    got = layer.gated_delta_bwd(*low, dO.to(BF).cuda(), S0.float().cuda())
    assert float(want[0][0, 1, 0, 0]) == 1 and torch.equal(got[0].double().cpu(), want[0])
    assert torch.equal(got[2].double().cpu(), want[2]) and torch.equal(got[5].double().cpu(), want[5])
