"""The gated delta rule on the GPU against its definition in 64 bits, forward, backward and token by token.

Tolerances (2-norms, relative).  With unit keys, beta in (0, 1) and gates up to 1 a token's transition never makes a difference larger, so
an error is what a chunk adds: sums of d_k + 64 + 64 rounded products in fp32, at most (d_k + 128) 2^-24 of their
largest partial sums, for which the same again is allowed: F32 below.  Where bf16 is what comes out, a rounding of 2^-8 at most joins it, and for O and
the gradients operands of 16 bits, 2^-17 each, four of them one after another at most: BF."""
import pytest
import torch

import gated_delta_ref as ref

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def f32_bound(dk):
    return 2 * (dk + 128) * 2.0 ** -24


def bound(t, dk):
    return f32_bound(dk) if t == torch.float32 else 2.0 ** -8 + 4 * 2.0 ** -17 + f32_bound(dk)


@pytest.fixture(scope="module")
def layer():
    assert torch.cuda.is_available()
    from paper_2504_00492_amd import layer
    return layer


def make(B, L, Hk, Hv, dk, dv, dt, *, s0=True, seed=0, gate=1.0, rows=None):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    unit = torch.nn.functional.normalize
    lead = rows or (B, L)
    Q, K, V = unit(n(*lead, Hk, dk), dim=-1), unit(n(*lead, Hk, dk) + 0.4 * n(Hk, dk), dim=-1), n(*lead, Hv, dv)
    G = -torch.nn.functional.softplus(n(*lead, Hv) * 0.5 - torch.arange(Hv) % 4 * 1.5) * gate
    beta = n(*lead, Hv).sigmoid()
    S0 = 0.3 * n(B, Hv, dv, dk) if s0 else None
    dO, dSL = n(*lead, Hv, dv), n(B, Hv, dv, dk)
    low = [t.to(dt).cuda() for t in (Q, K, V, G, beta)]
    return low, None if S0 is None else S0.float().cuda(), dO.to(dt).cuda(), dSL.float().cuda()


def wide(*tensors):
    return [None if t is None else t.double().cpu() for t in tensors]


def check(layer, args, S0, dO, dSL, dt, dk, offsets=None, ends=None):
    """Forward and backward of packed or plain sequences against the definition, each sequence by itself."""
    O, SL = layer.gated_delta_fwd(*args, S0, offsets=offsets)
    got = layer.gated_delta_bwd(*args, dO, S0, dSL, offsets=offsets)
    if ends is None:
        wO, wS = ref.delta(*wide(*args, S0))
        want = ref.delta_grads(wide(*args, S0), *wide(dO, dSL))
        pairs = [(O, wO, "O"), (SL, wS, "SL")] + [(a, b, n) for a, b, n in zip(got, want, ("dQ", "dK", "dV", "dG", "dbeta", "dS0")) if b is not None]
    else:
        pairs = []
        for n, (a, b) in enumerate(zip(ends, ends[1:])):
            one = [t[:, a:b] for t in args]
            s0, dsl = None if S0 is None else S0[n:n + 1], dSL[n:n + 1]
            wO, wS = ref.delta(*wide(*one, s0))
            want = ref.delta_grads(wide(*one, s0), *wide(dO[:, a:b], dsl))
            pairs += [(O[:, a:b], wO, f"O {n}"), (SL[n:n + 1], wS, f"SL {n}")]
            pairs += [(t[:, a:b], w, f"grad {i} {n}") for i, (t, w) in enumerate(zip(got[:5], want)) if b > a]
            if s0 is not None and want[5] is not None:
                pairs.append((got[5][n:n + 1], want[5], f"dS0 {n}"))
    for a, b, name in pairs:
        tol = bound(a.dtype, dk)
        o = ref.off(a, b)
        assert o <= tol, (name, o, tol)


SIZES = [
    # B, L, Hk, Hv, dk, dv
    (1, 1, 1, 1, 64, 64), (2, 1, 2, 2, 128, 128), (1, 2, 1, 1, 16, 16), (1, 15, 1, 1, 64, 32), (1, 16, 1, 1, 128, 16), (1, 17, 2, 2, 32, 48),
    (2, 63, 1, 2, 64, 64), (1, 64, 2, 2, 128, 128), (1, 65, 1, 1, 128, 64), (2, 127, 1, 3, 72, 40), (1, 128, 2, 4, 64, 128), (1, 200, 1, 1, 128, 128),
    (1, 129, 1, 1, 256, 256), (1, 70, 1, 2, 256, 24), (1, 66, 1, 1, 200, 130), (3, 90, 2, 2, 1, 1), (1, 100, 1, 1, 3, 7), (1, 300, 1, 1, 65, 33),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_against_the_definition(layer, size, dtype):
    dt = DT[dtype]
    args, S0, dO, dSL = make(*size, dt, s0=size[1] % 2 == 0, seed=sum(size))
    check(layer, args, S0, dO, dSL, dt, size[4])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lengths,behind", [((5, 0, 64, 1, 65, 130), 0), ((0, 0, 3), 9), ((200,), 0), ((64, 64, 128), 3), ((1,) * 20, 1)])
def test_packed_sequences(layer, lengths, behind, dtype):
    dt = DT[dtype]
    ends = [0]
    for n in lengths:
        ends.append(ends[-1] + n)
    args, S0, dO, dSL = make(len(lengths), 0, 1, 2, 64, 48, dt, seed=len(lengths), rows=(1, ends[-1] + behind))
    off = torch.tensor(ends, dtype=torch.int32).cuda()
    check(layer, args, S0, dO, dSL, dt, 64, off, ends)


@pytest.mark.parametrize("gate", [1.0, 0.01])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [(1, 1600, 1, 1, 64, 64), (1, 2000, 1, 2, 128, 128), (2, 1700, 1, 1, 72, 40), (1, 1537, 1, 1, 256, 130), (1, 4100, 1, 1, 128, 16),
                                  (3, 0, 1, 1, 64, 48)], ids=lambda s: "x".join(map(str, s)))
def test_few_long_sequences(layer, size, dtype, gate, monkeypatch):
    """Cut into segments that run side by side.  To what a chunk adds come the errors of what a segment makes of the unit matrix, of the same size, and
    the d_k rounded products of joining them: three times F32 in all.  The last size: packed ones, one of them empty, one shorter than a segment."""
    monkeypatch.setitem(globals(), "f32_bound", lambda dk: 6 * (dk + 128) * 2.0 ** -24)
    B, L, *heads = size
    if L:
        args, S0, dO, dSL = make(B, L, *heads, DT[dtype], seed=sum(size), gate=gate)
        check(layer, args, S0, dO, dSL, DT[dtype], heads[2])
    else:
        ends = [3, 2603, 2603, 2643]
        args, S0, dO, dSL = make(B, 0, *heads, DT[dtype], seed=sum(size), gate=gate, rows=(1, 2650))
        check(layer, args, S0, dO, dSL, DT[dtype], heads[2], torch.tensor(ends, dtype=torch.int32).cuda(), ends)


def test_rows_of_no_sequence_are_left_alone(layer):
    args, S0, dO, dSL = make(2, 0, 1, 2, 64, 48, torch.bfloat16, rows=(1, 100))
    for t in (*args, dO):
        t[:, 90:] = float("nan")      # (nobody's: not read)
        t[:, :7] = float("nan")
    off = torch.tensor([7, 40, 90], dtype=torch.int32).cuda()
    L, Hk, Hv, dk, dv = 100, 1, 2, 64, 48
    marked = lambda *s: torch.full(s, 7.0, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    O, dQ, dK, dV, dG, db = marked(1, L, Hv, dv), marked(1, L, Hk, dk), marked(1, L, Hk, dk), marked(1, L, Hv, dv), marked(1, L, Hv), marked(1, L, Hv)
    SL, dS0 = torch.empty_like(S0), torch.empty_like(S0)
    sizes = (2, L, Hk, Hv, dk, dv)
    st = lambda t: (t, 0, t.stride(1), t.stride(2))  # noqa: E731
    arrays = [x for t in args for x in st(t)]
    need = layer.pf_gated_delta_workspace_bytes(*sizes, 1, 1, layer.PF_BF16)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    assert layer.pf_gated_delta_fwd(*arrays, S0, off, O, SL, *sizes, layer.PF_BF16, ws, need, stream) == 0
    assert layer.pf_gated_delta_bwd(*arrays, *st(dO), S0, dSL, off, dQ, dK, dV, dG, db, dS0, *sizes, layer.PF_BF16, ws, need, stream) == 0
    torch.cuda.synchronize()
    for t in (O, dQ, dK, dV, dG, db):
        assert bool((t[:, 90:] == 7).all()) and bool((t[:, :7] == 7).all()) and bool(torch.isfinite(t).all())
    assert bool(torch.isfinite(SL).all()) and bool(torch.isfinite(dS0).all())


@pytest.mark.parametrize("offsets", [[0, 50, 20, 70], [-5, 10, 2000, 2000], [70, 0, 0, 0], [0, 0, 0, 0]])
def test_offsets_out_of_order_are_brought_into_it(layer, offsets):
    args, S0, dO, dSL = make(3, 0, 1, 1, 64, 32, torch.float32, rows=(1, 70))
    ends, top = [], 0
    for o in offsets:
        top = max(top, min(max(o, 0), 70))
        ends.append(top)
    check(layer, args, S0, dO, dSL, torch.float32, 64, torch.tensor(offsets, dtype=torch.int32).cuda(), ends)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_orders_and_strides(layer, dtype):
    """Heads before tokens, slices of one projection, a beta that all heads share, tokens backwards in memory are the same numbers."""
    dt = DT[dtype]
    (Q, K, V, G, beta), S0, dO, dSL = make(2, 77, 2, 4, 64, 64, dt)
    beta = beta[:, :, :1].expand(2, 77, 4)
    want = (*layer.gated_delta_fwd(Q, K, V, G, beta.contiguous(), S0), *layer.gated_delta_bwd(Q, K, V, G, beta.contiguous(), dO, S0, dSL))
    swap = lambda t: t.transpose(1, 2).contiguous().transpose(1, 2)  # noqa: E731
    batch = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    both = torch.cat((Q.flatten(2), K.flatten(2), V.flatten(2), G), 2)      # rows of 516 values: not whole 16 bytes apart
    q, k, v, g = both.split([128, 128, 256, 4], 2)
    for a in ((swap(Q), swap(K), swap(V), swap(G), beta, swap(dO)), (q.unflatten(2, (2, 64)), k.unflatten(2, (2, 64)), v.unflatten(2, (4, 64)), g, beta, batch(dO))):
        got = (*layer.gated_delta_fwd(*a[:5], S0), *layer.gated_delta_bwd(*a, S0, dSL))
        for x, y in zip(got, want):
            assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_token_by_token(layer, dtype):
    dt = DT[dtype]
    (Q, K, V, G, beta), S0, _, _ = make(3, 70, 2, 4, 128, 96, dt)
    S = S0.clone()
    steps = torch.stack([layer.gated_delta_step(Q[:, t], K[:, t], V[:, t], G[:, t], beta[:, t], S) for t in range(70)], 1)
    wO, wS = ref.delta(*wide(Q, K, V, G, beta, S0))
    assert ref.off(steps, wO) <= bound(dt, 128)
    assert ref.off(S, wS) <= 70 * 140 * 2.0 ** -24      # 70 tokens, 140 roundings each
    O, SL = layer.gated_delta_fwd(Q, K, V, G, beta, S0)
    assert ref.off(O, wO) <= bound(dt, 128) and ref.off(SL, wS) <= f32_bound(128)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,Hk,Hv,dk,dv", [(1, 1, 1, 128, 128), (5, 2, 4, 64, 64), (3, 1, 1, 72, 40), (2, 1, 1, 7, 5), (70, 1, 2, 256, 200), (1, 1, 1, 1, 1), (300, 1, 1, 64, 17)])
def test_step(layer, B, Hk, Hv, dk, dv, dtype):
    dt = DT[dtype]
    (Q, K, V, G, beta), _, _, _ = make(B, 1, Hk, Hv, dk, dv, dt, seed=B)
    g = torch.Generator().manual_seed(B + dk)
    pool = torch.randn(B + 2, Hv, dv, dk, generator=g).cuda()
    slots = torch.randperm(B + 2, generator=g)[:B].int().cuda()
    before = pool.clone()
    O = layer.gated_delta_step(Q[:, 0], K[:, 0], V[:, 0], G[:, 0], beta[:, 0], pool, slots)
    wO, wS = ref.delta(*wide(Q, K, V, G, beta, before[slots.long()]))
    # Two sums of d_k products and four roundings behind them, each of a term a S, a beta (S k) k^T or beta v k^T: with |k| = |q| = 1, a and beta
    # up to 1 these are |S|, |S| and |v| at most, also where they cancel in the result.  Then the rounding of o.
    tol = (dk + 4) * 2.0 ** -24 * (2 * float(before[slots.long()].double().norm()) + float(V.double().norm()))
    assert float((O.double().cpu() - wO[:, 0]).norm()) <= tol + (2.0 ** -8 if dtype == "bf16" else 0) * float(wO.norm())
    assert float((pool[slots.long()].double().cpu() - wS).norm()) <= tol
    rest = torch.ones(B + 2, dtype=torch.bool)
    rest[slots.long().cpu()] = False
    assert torch.equal(pool[rest.cuda()], before[rest.cuda()])


def test_step_without_a_state(layer):
    """Padding, slots beyond the pool and a slot that an earlier sequence has: o is zero, no state changes."""
    (Q, K, V, G, beta), S0, _, _ = make(6, 1, 1, 2, 64, 64, torch.float32)
    a = [t[:, 0] for t in (Q, K, V, G, beta)]
    pool = S0[:4].clone()
    slots = torch.tensor([2, -1, 0, 2, 4, 1], dtype=torch.int32).cuda()
    O = layer.gated_delta_step(*a, pool, slots)
    served = [0, 2, 5]
    alone = S0[:4].clone()
    want = layer.gated_delta_step(*(t[served] for t in a), alone, slots[served])
    assert torch.equal(O[served], want) and torch.equal(pool, alone) and not bool(O[[1, 3, 4]].any()) and torch.equal(pool[3], S0[3])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gates_at_their_ends(layer, dtype):
    """Log gates of 0, of a large negative number, of the type's lowest and of minus infinity: sequences anew in the middle of chunks,
    which sums of logs may not blur."""
    dt = DT[dtype]
    (Q, K, V, G, beta), S0, dO, dSL = make(1, 150, 1, 4, 64, 32, dt)
    for t, h, v in ((0, 0, -1e30), (10, 0, -float("inf")), (11, 0, -1e4), (63, 0, torch.finfo(dt).min), (64, 1, -float("inf")), (100, 1, -200.0), (149, 2, -float("inf"))):
        G[:, t, h] = v
    G[:, 20:40, 3] = -300.0
    G[:, 70:, 2] = 0.0
    check(layer, [Q, K, V, G, beta], S0, dO, dSL, dt, 64)


def test_a_beta_of_zero_and_of_one(layer):
    (Q, K, V, G, beta), S0, dO, dSL = make(1, 140, 1, 2, 64, 32, torch.float32)
    beta[:, :70, 0], beta[:, 70:, 0] = 0.0, 1.0
    beta[:, :, 1] = 1.0
    check(layer, [Q, K, V, G, beta], S0, dO, dSL, torch.float32, 64)


def test_the_same_key_again_and_again(layer):
    """64 equal keys with beta = 1 and no decay: the chunk's triangular system is all ones, its powers are not."""
    (Q, K, V, G, beta), S0, dO, dSL = make(1, 128, 1, 1, 64, 32, torch.float32)
    K[:] = K[:, :1]
    beta[:], G[:] = 1.0, 0.0
    check(layer, [Q, K, V, G, beta], S0, dO, dSL, torch.float32, 64)


def test_no_tokens_and_no_sequences(layer):
    (Q, K, V, G, beta), S0, dO, dSL = make(2, 0, 1, 2, 64, 32, torch.float32)
    O, SL = layer.gated_delta_fwd(Q, K, V, G, beta, S0)
    assert O.shape == V.shape and torch.equal(SL, S0)
    assert not bool(layer.gated_delta_fwd(Q, K, V, G, beta)[1].any())
    assert torch.equal(layer.gated_delta_bwd(Q, K, V, G, beta, dO, S0, dSL)[5], dSL)
    none = [t[:0] for t in (Q, K, V, G, beta)]
    assert layer.gated_delta_fwd(*none)[1].shape == (0, 2, 32, 64)
    empty = torch.zeros(4, dtype=torch.int32, device="cuda")
    S3 = torch.randn(3, 2, 32, 64, device="cuda")
    args = [t[:1] for t in (Q, K, V, G, beta)]
    assert torch.equal(layer.gated_delta_fwd(*args, S3, offsets=empty)[1], S3)
    assert torch.equal(layer.gated_delta_bwd(*args, dO[:1], S3, S3 + 1, offsets=empty)[5], S3 + 1)


def test_the_state_in_place(layer):
    (Q, K, V, G, beta), S0, dO, dSL = make(2, 100, 1, 2, 64, 64, torch.bfloat16)
    O, SL = layer.gated_delta_fwd(Q, K, V, G, beta, S0)
    sizes = (2, 100, 1, 2, 64, 64)
    arrays = [x for t in (Q, K, V, G, beta) for x in (t, *t.stride()[:3])]
    need = layer.pf_gated_delta_workspace_bytes(*sizes, 0, 0, layer.PF_BF16)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    S, O2 = S0.clone(), torch.empty_like(O)
    assert layer.pf_gated_delta_fwd(*arrays, S, None, O2, S, *sizes, layer.PF_BF16, ws, need, torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(S, SL) and torch.equal(O, O2)


@pytest.mark.parametrize("packed", [False, True])
def test_gradients_against_differences(layer, packed):
    """Along a random direction: (f(x + h u) - f(x - h u)) / 2 h with f = <O, dO> + <S_L, dSL> of the library's own forward in fp32, summed
    in 64 bits.  h = 2^-6 leaves curvature h^2 of the third derivative's size, and 2^-20 of f for its rounding, divided by 2 h: 1e-2 of
    the slope is beyond both where the direction is not nearly level."""
    args, S0, dO, dSL = make(2, 130, 1, 2, 64, 32, torch.float32, rows=(1, 130) if packed else None)
    off = torch.tensor([0, 60, 130], dtype=torch.int32).cuda() if packed else None
    grads = layer.gated_delta_bwd(*args, dO, S0, dSL, offsets=off)
    g = torch.Generator().manual_seed(3)

    def f(x):
        O, S = layer.gated_delta_fwd(*x[:5], x[5], offsets=off)
        return float((O.double() * dO.double()).sum() + (S.double() * dSL.double()).sum())

    every = [*args, S0]
    for i, (x, grad) in enumerate(zip(every, grads)):
        u = torch.randn(x.shape, generator=g).cuda() * 0.1 + grad * (0.1 / float(grad.abs().max()))      # (a direction with a slope)
        h = 2.0 ** -6
        up, down = list(every), list(every)
        up[i], down[i] = x + h * u, x - h * u
        slope, want = (f(up) - f(down)) / (2 * h), float((grad.double() * u.double()).sum())
        assert abs(slope - want) <= 1e-2 * abs(want), (i, slope, want)


def test_a_captured_call_replayed(layer):
    args, S0, dO, dSL = make(2, 150, 1, 2, 128, 64, torch.bfloat16)
    off = torch.tensor([0, 70, 150], dtype=torch.int32).cuda()
    flat = [t[:1] for t in args]
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        layer.gated_delta_bwd(*flat, dO[:1], S0, dSL, offsets=off)
        layer.gated_delta_fwd(*flat, S0, offsets=off)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = (*layer.gated_delta_fwd(*flat, S0, offsets=off), *layer.gated_delta_bwd(*flat, dO[:1], S0, dSL, offsets=off))
    for k in range(4):
        if k:
            for t, u in zip(flat, make(2, 150, 1, 2, 128, 64, torch.bfloat16, seed=k)[0]):
                t.copy_(u[:1])
            off[1] = 70 + 10 * k
        graph.replay()
        torch.cuda.synchronize()
        want = (*layer.gated_delta_fwd(*flat, S0, offsets=off), *layer.gated_delta_bwd(*flat, dO[:1], S0, dSL, offsets=off))
        for a, b in zip(out, want):
            assert torch.equal(a, b)


def test_two_streams_and_the_same_bits_again(layer):
    """Calls side by side with workspaces of their own give what they give alone, and always the same bits."""
    args, S0, dO, dSL = make(4, 333, 2, 4, 128, 128, torch.bfloat16)
    torch.cuda.synchronize()
    want = (*layer.gated_delta_fwd(*args, S0), *layer.gated_delta_bwd(*args, dO, S0, dSL))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [(*layer.gated_delta_fwd(*args, S0, stream=s), *layer.gated_delta_bwd(*args, dO, S0, dSL, stream=s)) for s in streams]
    torch.cuda.synchronize()
    for g in got:
        for a, b in zip(g, want):
            assert torch.equal(a, b)


def test_a_workspace_with_anything_in_it(layer):
    args, S0, dO, dSL = make(1, 100, 1, 1, 40, 24, torch.float32)
    want = layer.gated_delta_bwd(*args, dO, S0, dSL)
    need = layer.pf_gated_delta_workspace_bytes(1, 100, 1, 1, 40, 24, 0, 1, layer.PF_F32)
    ws = torch.full((need // 4,), float("nan"), device="cuda")
    for a, b in zip(layer.gated_delta_bwd(*args, dO, S0, dSL, workspace=ws), want):
        assert torch.equal(a, b)


def test_segments_in_place_captured_and_with_anything_in_the_workspace(layer):
    """One long sequence, cut: S_L in the place of S0 and dS0 in that of dS_L, NaN in the workspaces, captured, on another stream, slices of a projection:
    the same bits always."""
    sizes = (1, 2500, 1, 2, 64, 64)
    args, S0, dO, dSL = make(*sizes, torch.bfloat16, gate=0.1)
    want = (*layer.gated_delta_fwd(*args, S0), *layer.gated_delta_bwd(*args, dO, S0, dSL))
    wide = torch.zeros(1, 2500, 1024, dtype=torch.bfloat16, device="cuda")
    low, parts = 8, []
    for t in args:
        n = t[0, 0].numel()
        wide[..., low:low + n] = t.flatten(2)
        parts.append(wide[..., low:low + n].unflatten(2, t.shape[2:]))
        low += n
    ws = [torch.full((layer.pf_gated_delta_workspace_bytes(*sizes, 0, b, layer.PF_BF16) // 4,), float("nan"), device="cuda") for b in (0, 1)]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    others = [(*layer.gated_delta_fwd(*parts, S0, workspace=ws[0]), *layer.gated_delta_bwd(*parts, dO, S0, dSL, workspace=ws[1])),
              (*layer.gated_delta_fwd(*args, S0, stream=s), *layer.gated_delta_bwd(*args, dO, S0, dSL, stream=s))]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        others.append((*layer.gated_delta_fwd(*args, S0), *layer.gated_delta_bwd(*args, dO, S0, dSL)))
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        for got in others:
            for a, b in zip(got, want):
                assert torch.equal(a, b)
        others[2][0].zero_(), others[2][2].zero_()
    graph.replay()
    arrays = [x for t in args for x in (t, *t.stride()[:3])]
    stream = torch.cuda.current_stream().cuda_stream
    S, R, O = S0.clone(), dSL.clone(), torch.empty_like(want[0])
    assert layer.pf_gated_delta_fwd(*arrays, S, None, O, S, *sizes, layer.PF_BF16, ws[0], 4 * ws[0].numel(), stream) == 0
    grads = [torch.empty_like(t) for t in want[2:7]]
    assert layer.pf_gated_delta_bwd(*arrays, dO, *dO.stride()[:3], S0, R, None, *grads, R, *sizes, layer.PF_BF16, ws[1], 4 * ws[1].numel(), stream) == 0
    for a, b in zip((O, S, *grads, R), want):
        assert torch.equal(a, b)


def test_offsets_beyond_32_bits(layer):
    """Rows that lie 120 KB apart, 4.8 GB in all, and a pool of 9 GB: the same bits as dense ones."""
    L, W = 40000, 60000
    args, _, dO, _ = make(1, L, 1, 2, 64, 64, torch.bfloat16, s0=False)
    wide = torch.empty(1, L, W, dtype=torch.bfloat16, device="cuda")
    low, parts = W - 1024, []
    for t in (*args, dO):
        n = t[0, 0].numel()
        wide[..., low:low + n] = t.flatten(2)
        parts.append(wide[..., low:low + n].unflatten(2, t.shape[2:]))
        low += n + -n % 8
    for a, b in zip(layer.gated_delta_fwd(*parts[:5]), layer.gated_delta_fwd(*args)):
        assert torch.equal(a, b)
    for a, b in zip(layer.gated_delta_bwd(*parts), layer.gated_delta_bwd(*args, dO)):
        assert torch.equal(a, b)
    table, at = layer.rotary_table(L, 64), torch.arange(L, dtype=torch.int32, device="cuda")
    for a, b in zip(layer.head_norm_fwd(parts[0][0], parts[1][0], None, None, table, at, norm="l2", eps=1e-6),
                    layer.head_norm_fwd(args[0][0], args[1][0], None, None, table, at, norm="l2", eps=1e-6)):
        assert torch.equal(a, b)
    del wide, parts
    pool = torch.zeros(2150, 64, 128, 128, device="cuda")
    (Q, K, V, G, beta), S0, _, _ = make(3, 1, 64, 64, 128, 128, torch.bfloat16)
    tokens, slots = [t[:, 0] for t in (Q, K, V, G, beta)], torch.tensor([2149, 0, 2148], dtype=torch.int32).cuda()
    pool[slots.long()] = S0
    O = layer.gated_delta_step(*tokens, pool, slots)
    assert torch.equal(O, layer.gated_delta_step(*tokens, S0)) and torch.equal(pool[slots.long()], S0) and not bool(pool[1:2148].any())


@pytest.mark.parametrize("packed", [False, True])
def test_a_workspace_of_more_sequences(layer, packed):
    """One that was sized for ten sequences, none of which is cut then, does for two, which are: the same bits as with its own."""
    heads, dt = (1, 1, 64, 64), torch.bfloat16
    args, S0, dO, dSL = make(2, 2500, *heads, dt, gate=0.1, rows=(1, 5000) if packed else None)
    off = torch.tensor([0, 2600, 5000], dtype=torch.int32).cuda() if packed else None
    want = (*layer.gated_delta_fwd(*args, S0, offsets=off), *layer.gated_delta_bwd(*args, dO, S0, dSL, offsets=off))
    ws = [torch.empty(layer.pf_gated_delta_workspace_bytes(10, 5000 if packed else 2500, *heads, packed, b, layer.PF_BF16), dtype=torch.uint8, device="cuda") for b in (0, 1)]
    got = (*layer.gated_delta_fwd(*args, S0, offsets=off, workspace=ws[0]), *layer.gated_delta_bwd(*args, dO, S0, dSL, offsets=off, workspace=ws[1]))
    for a, b in zip(got, want):
        assert torch.equal(a, b)
