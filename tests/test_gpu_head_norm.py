"""Norm of heads with rotation against its definition in 64 bits, forward and backward.

Tolerances: a sum of d squares, a root, a division, two products and a sum for the rotation in fp32, (d + 8) 2^-24 of a row's largest
partial sums; one rounding of 2^-8 where bf16 comes out.  The backward has a second sum of d products.  dw sums over M H rows: as
many roundings at most, of sums that need not grow with them: the bound is 2^-24 times the rows' number, times the sum of sizes."""
import pytest
import torch

import gated_delta_ref as ref

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6


@pytest.fixture(scope="module")
def layer():
    assert torch.cuda.is_available()
    from paper_2504_00492_amd import layer
    return layer


def make(M, Hq, Hk, d, rot, dt, weights=True, seed=0, far=1000):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g).to(dt).cuda()  # noqa: E731
    Q, K = n(M, Hq, d), n(M, Hk, d) if Hk else None
    wq, wk = ((1 + 0.1 * n(d).float()).to(dt), (1 + 0.1 * n(d).float()).to(dt) if Hk else None) if weights else (None, None)
    at = torch.randint(0, far, (M,), generator=g).int().cuda() if rot else None
    return Q, K, wq, wk, at, n(M, Hq, d), n(M, Hk, d) if Hk else None


def check(layer, Q, K, wq, wk, table, at, dYq, dYk, how):
    d, dt = Q.shape[-1], Q.dtype
    M = Q.shape[0]
    low = 2.0 ** -8 if dt == torch.bfloat16 else 0.0
    Y = layer.head_norm_fwd(Q, K, wq, wk, table, at, **how)
    got = layer.head_norm_bwd(Q, K, dYq, dYk, wq, wk, table, at, **how)
    for i, (x, w, dy, scale) in enumerate(((Q, wq, dYq, how["q_scale"]), (K, wk, dYk, 1.0))):
        if x is None:
            assert Y[i] is None and got[i] is None and got[2 + i] is None
            continue
        X, W = x.double().requires_grad_(), None if w is None else w.double().requires_grad_()
        want = ref.heads(X, W, table, at, how["norm"], how["eps"], scale, how["pairs"])
        assert ref.off(Y[i], want.detach()) <= (d + 8) * 2.0 ** -24 + low, (i, "y")
        if M:
            (want * dy.double()).sum().backward()
            # dx = (g - xh m) / n: where the two terms cancel (wholly at d = 1) the roundings of each stay, so fp32's share goes by
            # their sizes; |xh m| is |g| at most, as xh m is g's projection on xh
            n = torch.sqrt((X.detach() ** 2).sum(-1, keepdim=True) / (d if how["norm"] == "rms" else 1) + EPS)
            terms = 2 * float((dy.double().norm(dim=-1) * abs(scale) * (1 if w is None else float(w.double().abs().max())) / n[..., 0]).norm())
            off = float((got[i].double() - X.grad).norm())
            assert off <= 4 * (d + 8) * 2.0 ** -24 * terms + low * float(X.grad.norm()), (i, "dx", off)
        if w is None:
            assert got[2 + i] is None
        elif M:
            size = float(M * x.shape[1])
            o = (got[2 + i].double() - W.grad).abs()
            xh = X.detach() / X.detach().norm(dim=-1, keepdim=True) * d ** 0.5
            # each term is xh times the turned gradient, whose size is that of its pair at most
            most = (xh.abs() * abs(scale) * (dy.double().abs().amax(-1, keepdim=True) * 2 ** 0.5)).sum((0, 1)) * (1 if how["norm"] == "rms" else d ** -0.5)
            assert bool((o <= (size + d + 8) * 2.0 ** -24 * most).all()), (i, "dw", float((o / most).max()))
        else:
            assert not bool(got[2 + i].any())


SIZES = [
    # M, Hq, Hk, d, rot
    (1, 1, 1, 128, 128), (4, 32, 32, 128, 128), (3, 4, 2, 64, 64), (17, 3, 1, 128, 64), (5, 2, 2, 72, 40), (33, 5, 3, 80, 80), (2, 1, 0, 16, 0),
    (7, 2, 1, 256, 256), (9, 3, 2, 256, 64), (3, 2, 1, 512, 512), (4, 1, 1, 504, 2), (6, 2, 2, 33, 10), (5, 1, 1, 1, 0), (8, 1, 2, 2, 2), (5, 3, 3, 20, 6),
    (1000, 6, 2, 128, 96), (300, 1, 1, 40, 24), (0, 2, 2, 64, 64),
    (3, 2, 1, 1024, 1024), (2, 3, 1, 1010, 2), (5, 1, 1, 640, 256), (2, 70, 9, 32, 16), (3000, 1, 1, 16, 16),
]


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("norm", ["rms", "l2"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_against_the_definition(layer, size, dtype, norm, pairs):
    M, Hq, Hk, d, rot = size
    Q, K, wq, wk, at, dYq, dYk = make(*size, DT[dtype], weights=norm == "rms", seed=sum(size))
    table = layer.rotary_table(1000, rot) if rot else None
    check(layer, Q, K, wq, wk, table, at, dYq, dYk, dict(norm=norm, eps=EPS, q_scale=d ** -0.5, pairs=pairs))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_slices_of_a_projection(layer, dtype):
    """Rows at any element, other orders, gradients too: the same bits as dense ones."""
    dt = DT[dtype]
    how = dict(norm="rms", eps=EPS, q_scale=0.5, pairs=False)
    Q, K, wq, wk, at, dYq, dYk = make(50, 4, 2, 64, 64, dt)
    table = layer.rotary_table(1000, 64)
    want = (*layer.head_norm_fwd(Q, K, wq, wk, table, at, **how), *layer.head_norm_bwd(Q, K, dYq, dYk, wq, wk, table, at, **how))
    both = torch.empty(50, 1 + 6 * 64, dtype=dt, device="cuda")
    both[:, 1:257], both[:, 257:] = Q.flatten(1), K.flatten(1)
    q, k = both[:, 1:257].unflatten(1, (4, 64)), both[:, 257:].unflatten(1, (2, 64))
    swap = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    for a in ((q, k, dYq, dYk), (swap(Q), swap(K), swap(dYq), swap(dYk)), (q, swap(K), swap(dYq), dYk)):
        got = (*layer.head_norm_fwd(*a[:2], wq, wk, table, at, **how), *layer.head_norm_bwd(*a, wq, wk, table, at, **how))
        for x, y in zip(got, want):
            assert torch.equal(x, y)


def test_far_positions_and_none(layer):
    Q, K, wq, wk, at, _, _ = make(4, 2, 1, 128, 64, torch.float32, far=131072)
    table = layer.rotary_table(131072, 64)
    at[:] = torch.tensor([131071, 0, 131072, -1], dtype=torch.int32)
    Yq, Yk = layer.head_norm_fwd(Q, K, wq, wk, table, at, norm="l2", eps=EPS)
    want = ref.heads(Q.double(), wq.double(), table, at.clamp(0, 131071), "l2", EPS, 1.0, False)
    assert ref.off(Yq[:2], want[:2]) <= 136 * 2.0 ** -24
    assert bool(Yq[2:, :, :64].isnan().all()) and ref.off(Yq[2:, :, 64:], want[2:, :, 64:]) <= 136 * 2.0 ** -24
    # the table's own angles: 64-bit ones, rounded once
    p = torch.tensor([131071.0], dtype=torch.float64)
    angle = p * 10000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64)
    assert torch.equal(table[131071, :32].cpu(), angle.cos().float()) and torch.equal(table[131071, 32:].cpu(), angle.sin().float())


def test_a_row_of_zeros_and_large_numbers(layer):
    Q = torch.zeros(2, 2, 64, device="cuda")
    Q[1] = 1e15
    Yq, _ = layer.head_norm_fwd(Q, norm="l2", eps=EPS)
    assert not bool(Yq[0].any()) and bool((Yq[1] - 0.125).abs().max() <= 0.125 * 72 * 2.0 ** -24)
    dQ = layer.head_norm_bwd(Q, None, torch.ones_like(Q), None, norm="l2", eps=EPS)[0]
    assert bool(torch.isfinite(dQ).all()) and bool((dQ[0] - EPS ** -0.5).abs().max() <= 1e3 * 80 * 2.0 ** -24)


def test_an_infinity_stays_in_its_place(layer):
    """As the formula has it: NaN where the infinity lies and at its partner of a turn, zeros elsewhere."""
    Q = torch.ones(3, 2, 96, device="cuda")
    Q[1, 0, 90] = Q[2, 1, 5] = float("inf")
    Yq, _ = layer.head_norm_fwd(Q, None, None, None, layer.rotary_table(10, 32), torch.arange(3, dtype=torch.int32, device="cuda"), norm="rms", eps=EPS)
    nan = torch.zeros(3, 2, 96, dtype=torch.bool, device="cuda")
    nan[1, 0, 90] = nan[2, 1, 5] = nan[2, 1, 5 + 16] = True
    assert torch.equal(Yq.isnan(), nan)
    assert not bool(Yq[1, 0][~nan[1, 0]].any()) and not bool(Yq[2, 1][~nan[2, 1]].any()) and bool((Yq[0] != 0).all())


def test_in_place(layer):
    Q, K, wq, wk, at, dYq, dYk = make(20, 4, 2, 128, 128, torch.bfloat16)
    table = layer.rotary_table(1000, 128)
    how = dict(norm="rms", eps=EPS, q_scale=1.0, pairs=False)
    Yq, Yk = layer.head_norm_fwd(Q, K, wq, wk, table, at, **how)
    dQ, dK = layer.head_norm_bwd(Q, K, dYq, dYk, wq, wk, table, at, **how)[:2]
    s = torch.cuda.current_stream().cuda_stream
    q, k, gq, gk = Q.clone(), K.clone(), dYq.clone(), dYk.clone()
    sizes = (20, 4, 2, 128, 128, 0, 0, EPS, 1.0, layer.PF_BF16)
    assert layer.pf_head_norm_bwd(Q, 512, 128, K, 256, 128, gq, 512, 128, gk, 256, 128, wq, wk, table, 1000, at, gq, gk, None, None, *sizes, None, 0, s) == 0
    assert layer.pf_head_norm_fwd(q, 512, 128, k, 256, 128, wq, wk, table, 1000, at, q, k, *sizes, s) == 0
    assert torch.equal(q, Yq) and torch.equal(k, Yk) and torch.equal(gq, dQ) and torch.equal(gk, dK)


def test_gradients_against_differences(layer):
    """As for the gated delta rule: slopes of <y, dy> along a direction, h = 2^-8; the weights' too."""
    how = dict(norm="rms", eps=EPS, q_scale=0.3, pairs=True)
    Q, K, wq, wk, at, dYq, dYk = make(40, 3, 2, 48, 32, torch.float32)
    table = layer.rotary_table(1000, 32)
    every = [Q, K, wq, wk]
    grads = layer.head_norm_bwd(Q, K, dYq, dYk, wq, wk, table, at, **how)

    def f(x):
        a, b = layer.head_norm_fwd(*x, table, at, **how)
        return float((a.double() * dYq.double()).sum() + (b.double() * dYk.double()).sum())

    for i, (x, grad) in enumerate(zip(every, grads)):
        u = grad * (0.5 / float(grad.abs().max()))
        h = 2.0 ** -8
        up, down = list(every), list(every)
        up[i], down[i] = x + h * u, x - h * u
        slope, want = (f(up) - f(down)) / (2 * h), float((grad.double() * u.double()).sum())
        assert abs(slope - want) <= 1e-2 * abs(want), (i, slope, want)


def test_captured_and_on_another_stream(layer):
    how = dict(norm="rms", eps=EPS, q_scale=0.3, pairs=False)
    Q, K, wq, wk, at, dYq, dYk = make(300, 4, 2, 64, 64, torch.bfloat16)
    table = layer.rotary_table(1000, 64)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = (*layer.head_norm_fwd(Q, K, wq, wk, table, at, stream=s, **how), *layer.head_norm_bwd(Q, K, dYq, dYk, wq, wk, table, at, stream=s, **how))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = (*layer.head_norm_fwd(Q, K, wq, wk, table, at, **how), *layer.head_norm_bwd(Q, K, dYq, dYk, wq, wk, table, at, **how))
    for k in range(3):
        if k:
            Q.mul_(0.5).add_(0.1), at.add_(k)
        graph.replay()
        torch.cuda.synchronize()
        want = (*layer.head_norm_fwd(Q, K, wq, wk, table, at, **how), *layer.head_norm_bwd(Q, K, dYq, dYk, wq, wk, table, at, **how))
        for a, b in zip(out, want):
            assert torch.equal(a, b) or bool(torch.equal(a.isnan(), b.isnan()))
        if k == 0:
            for a, b in zip(other, want):
                assert torch.equal(a, b)


def test_every_replay_is_the_eager_call(layer):
    """A captured call replayed with other inputs, and positions that the table has: the eager call's bits each time, and others than the time before."""
    how = dict(norm="rms", eps=EPS, q_scale=0.3, pairs=False)
    Q, K, wq, wk, at, dYq, dYk = make(300, 4, 2, 64, 64, torch.bfloat16, far=900)
    table = layer.rotary_table(1000, 64)

    def both():
        return (*layer.head_norm_fwd(Q, K, wq, wk, table, at, **how), *layer.head_norm_bwd(Q, K, dYq, dYk, wq, wk, table, at, **how))

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    before = None
    for k in range(4):
        if k:
            Q.mul_(0.5).add_(0.1), K.neg_().add_(0.2), at.add_(k), dYq.mul_(1.5), dYk.mul_(-0.5)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, both()):
            assert bool(torch.isfinite(a).all()) and torch.equal(a, b)
        if before is not None:
            assert not any(torch.equal(a, b) for a, b in zip(out, before))
        before = [t.clone() for t in out]


def test_gradients_at_a_position_that_the_table_does_not_have(layer):
    """NaN in the token's own rows and in what dw sums over them, of the turned values; every other number is as without the token."""
    how = dict(norm="rms", eps=EPS, q_scale=0.5, pairs=False)
    Q, K, wq, wk, at, dYq, dYk = make(9, 2, 1, 64, 32, torch.float32)
    table = layer.rotary_table(1000, 32)
    at[4] = -1
    dQ, dK, dwq, dwk = layer.head_norm_bwd(Q, K, dYq, dYk, wq, wk, table, at, **how)
    there = [0, 1, 2, 3, 5, 6, 7, 8]
    want = layer.head_norm_bwd(*(t[there] for t in (Q, K, dYq, dYk)), wq, wk, table, at[there], **how)
    for got, w in ((dQ, want[0]), (dK, want[1])):
        assert bool(got[4].isnan().all()) and torch.equal(got[there], w)
    for got in (dwq, dwk):
        assert bool(got[:32].isnan().all()) and bool(torch.isfinite(got[32:]).all())
