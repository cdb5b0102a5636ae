"""The operators of include/pf_layer.h on the GPU against plain statements of their definitions in 64 bits.

Tolerances, from the arithmetic (u = 2^-24, half a unit of fp32; half a unit of bf16 is 2^-8 of the value at most):
  norm       a sum of D positive squares in fp32, at most 32 additions deep, a division, a root, three products: 64 u of y;
             the gradient adds one more sum of D terms of either sign, whose error goes by the sum of their sizes
  8 bits     half a step of e4m3: 2^-4 of the value, 2^-10 of the scale below 2^-6; a value that lies within the norm's error
             of the middle of two may go either way.  From given values (the quantiser) the bits are those of the definition
  matmul     a block's sum of 128 products is taken to be off by 2^-16 of the sum of their sizes at most, blocks by u each
             (fp32 results come from exact products and are far inside; bf16 ones add their rounding)
  gated      errors run through the recurrence with the values: e_t = |a| e_{t-1} + u (c |a h_{t-1}| + 4 |b| + |h_t|), c = 8 + 4 |g| for
             the gate's exponential; twice that, since spans are joined as well as stepped through
  outputs in bf16 add their one rounding."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}
BF, F32, E4 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
EPS = 1e-5


@pytest.fixture(scope="module")
def layer():
    from paper_2504_00492_amd import layer
    return layer


def rnd(seed, *shape, dt=F32, std=1.0, mean=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std + mean).to(dt)


def near(x, ref, tol):
    """Every element of x within tol of ref (64 bits), NaN and infinities in the same places."""
    x, tol = x.double().cpu(), torch.as_tensor(tol, dtype=torch.float64).expand(ref.shape)
    assert x.shape == ref.shape
    fine = ref.isfinite()
    assert torch.equal(x.isnan(), ref.isnan()) and torch.equal(x[~fine & ~ref.isnan()], ref[~fine & ~ref.isnan()])
    over = ((x - ref).abs() > tol) & fine
    i = over.nonzero()
    assert not len(i), (len(i), over.numel(), i[0].tolist(), float(x[tuple(i[0])]), float(ref[tuple(i[0])]), float(tol[tuple(i[0])]))


def apart(t, gap):
    """The same matrix on the GPU with its rows `gap` elements further apart, and NaN between them."""
    wide = torch.full((*t.shape[:-1], t.shape[-1] + gap), float("nan"), dtype=t.dtype)
    wide[..., :t.shape[-1]] = t
    return wide.cuda()[..., :t.shape[-1]]


# ---- norm

def norm_ref(x, r, w):
    s = x if r is None else (x.double() + r.double()).to(x.dtype)
    s64 = s.double()
    rho = 1 / ((s64 ** 2).mean(1, keepdim=True) + EPS).sqrt()
    return s, s64 * rho * (1 if w is None else w.double())


def check_e4m3(q, scale, y, extra=64 * U):
    """q, scale (GPU) stand for y [M, D] in blocks of 128 columns."""
    M, D = y.shape
    nb = -(-D // 128)
    full = torch.nn.functional.pad(y, (0, nb * 128 - D)).view(M, nb, 128)
    want = full.abs().amax(2).clamp(min=1e-30) / 448
    near(scale.t(), want, want * (extra + 4 * U))
    s = scale.t().double().cpu().repeat_interleave(128, 1)[:, :D]
    assert q.dtype == E4
    near(q.double().cpu() * s, y, torch.maximum(y.abs() * 2.0 ** -4, s * 2.0 ** -10) * (1 + 1e-3))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("M,D", [(1, 1), (3, 7), (5, 64), (2, 128), (33, 130), (9, 256), (4, 500), (17, 512), (6, 1000), (3, 1024),
                                 (7, 1999), (5, 2048), (3, 4096), (2, 4097), (3, 8192), (2, 8200), (2, 16384), (700, 72)])
def test_norm(layer, M, D, dt):
    x, r, w = rnd(1, M, D, dt=dt), rnd(2, M, D, dt=dt, std=3), rnd(3, D, dt=dt, std=0.1, mean=1)
    for R in (r, None):
        s, y = norm_ref(x, R, w)
        S, Y, Q, scale = layer.norm_fwd(x.cuda(), w.cuda(), None if R is None else R.cuda(), eps=EPS, fp8=True)
        assert torch.equal(S.cpu(), s) and Q.stride(0) % 16 == 0
        near(Y, y, y.abs() * (64 * U + HALF[dt]))
        check_e4m3(Q, scale, y)
        only = layer.norm_fwd(x.cuda(), w.cuda(), None if R is None else R.cuda(), eps=EPS, y=False, fp8=True)
        assert only[1] is None and torch.equal(only[2].view(torch.uint8), Q.view(torch.uint8)) and torch.equal(only[3], scale)


@pytest.mark.parametrize("dt,gap", [(BF, 8), (BF, 3), (F32, 4), (F32, 1)])
@pytest.mark.parametrize("D", [96, 1000, 3000])
def test_norm_rows_apart(layer, D, dt, gap):
    """Rows of a wider array, at places that allow wide loads and at such that do not; no w."""
    x, r = rnd(1, 6, D, dt=dt), rnd(2, 6, D, dt=dt)
    s, y = norm_ref(x, r, None)
    S, Y, Q, scale = layer.norm_fwd(apart(x, gap), None, apart(r, gap), eps=EPS, fp8=True)
    assert torch.equal(S.cpu(), s)
    near(Y, y, y.abs() * (64 * U + HALF[dt]))
    check_e4m3(Q, scale, y)
    dy, ds = rnd(4, 6, D, dt=dt), rnd(5, 6, D, dt=dt)
    one = layer.norm_bwd(s.cuda(), dy.cuda(), None, ds.cuda(), eps=EPS)
    two = layer.norm_bwd(apart(s, gap), apart(dy, gap), None, apart(ds, gap), eps=EPS)
    for a, b in zip(one, two):
        assert torch.allclose(a.float(), b.float(), rtol=2.0 ** -7, atol=1e-5)


def test_norm_special_values(layer):
    x = rnd(1, 6, 300)
    x[1] = 0                     # y = 0, scale of an empty block
    x[2, 5] = float("nan")       # the whole row, and no other
    x[3, 5] = float("inf")       # finite values go to 0, the infinity to NaN
    x[4, :128] = 0
    x[5, 130] = 1e18
    s, y = norm_ref(x, None, None)
    _, Y, Q, scale = layer.norm_fwd(x.cuda(), eps=EPS, fp8=True)
    assert Y[3, 5].isnan() and (Y[3].cpu()[torch.arange(300) != 5] == 0).all()
    rows = [0, 1, 2, 4, 5]
    near(Y[rows], y[rows], y[rows].nan_to_num().abs() * 64 * U)
    rows = [0, 1, 4]
    check_e4m3(Q[rows], scale[:, rows], y[rows])
    assert Q[2].float().isnan().all() and Q[3, :128].float().isnan().all() and (Q[3, 128:].float() == 0).all()
    assert (Q[1].float() == 0).all() and torch.allclose(scale[:, 1].cpu(), torch.tensor(1e-30 / 448), rtol=1e-5)


def norm_grads(x, w, dy, ds):
    x, w, dy = x.double(), w.double(), dy.double()
    D = x.shape[1]
    rho = 1 / ((x ** 2).mean(1, keepdim=True) + EPS).sqrt()
    g, xh = dy * w, x * rho
    part = g - xh * (g * xh).mean(1, keepdim=True)
    size = g.abs() + xh.abs() * (g * xh).abs().mean(1, keepdim=True)
    return (0 if ds is None else ds.double()) + rho * part, rho * size, (dy * xh).sum(0), (dy * xh).abs().sum(0)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("M,D", [(1, 1), (3, 7), (40, 64), (1000, 128), (33, 200), (5, 512), (70, 1000), (600, 2048), (1030, 4096), (3, 4097),
                                 (5, 8192), (2, 16384), (1, 4096)])
def test_norm_backward(layer, M, D, dt):
    x, w, dy, ds = rnd(1, M, D, dt=dt, std=2), rnd(2, D, dt=dt, std=0.2, mean=1), rnd(3, M, D, dt=dt), rnd(4, M, D, dt=dt)
    for dS in (ds, None):
        dx, size, dw, wsize = norm_grads(x, w, dy, dS)
        X, W = layer.norm_bwd(x.cuda(), dy.cuda(), w.cuda(), None if dS is None else dS.cuda(), eps=EPS)
        near(X, dx, 128 * U * (size + dx.abs()) + HALF[dt] * dx.abs())
        near(W, dw, 128 * U * wsize)
        assert layer.norm_bwd(x.cuda(), dy.cuda(), w.cuda(), eps=EPS, want_dw=False)[1] is None


def test_norm_backward_is_the_forwards_derivative(layer):
    """Differences of the forward's definition (64 bits) along random directions."""
    x, w, dy = rnd(1, 5, 300), rnd(2, 300, mean=1), rnd(3, 5, 300)
    dx, dw = (t.double().cpu() for t in layer.norm_bwd(x.cuda(), dy.cuda(), w.cuda(), eps=EPS))
    loss = lambda x, w: float((x / ((x ** 2).mean(1, keepdim=True) + EPS).sqrt() * w * dy.double()).sum())  # noqa: E731
    for seed in range(3):
        ex, ew, h = rnd(10 + seed, 5, 300).double(), rnd(20 + seed, 300).double(), 1e-5
        diff = (loss(x.double() + h * ex, w.double() + h * ew) - loss(x.double() - h * ex, w.double() - h * ew)) / (2 * h)
        assert abs(diff - float((dx * ex).sum() + (dw * ew).sum())) < 1e-4 * (1 + abs(diff))


def test_norm_in_place_and_no_rows(layer):
    x, r = rnd(1, 9, 640, dt=BF).cuda(), rnd(2, 9, 640, dt=BF).cuda()
    want = layer.norm_fwd(x, None, r, eps=EPS)
    keep = r.clone()
    got = layer.norm_fwd(x, None, keep, eps=EPS, inplace=True)
    assert got[0].data_ptr() == keep.data_ptr() and torch.equal(keep, want[0]) and torch.equal(got[1], want[1])
    S, Y, Q, scale = layer.norm_fwd(x[:0], None, eps=EPS, fp8=True)
    assert Y.shape == (0, 640) and Q.shape == (0, 640) and scale.shape == (5, 0)
    dX, dw = layer.norm_bwd(x[:0], x[:0], None, eps=EPS)
    assert dX.shape == (0, 640) and (dw == 0).all()


# ---- 8 bits

def quant_ref(x, rows):
    """e4m3 values (fp32) and scales [ceil(R/rows), ceil(C/128)] in the steps that the header prints."""
    R, C = x.shape
    nr, nc = -(-R // rows), -(-C // 128)
    full = torch.nn.functional.pad(x.float(), (0, nc * 128 - C, 0, nr * rows - R)).view(nr, rows, nc, 128)
    top = full.abs().amax((1, 3))
    top = torch.where(top < 1e-30, torch.tensor(1e-30), top)
    inv = (torch.tensor(1.0) / top) * torch.tensor(448.0)
    q = (full * inv[:, None, :, None]).to(E4).float().reshape(nr * rows, nc * 128)[:R, :C]
    return q, top * torch.tensor(np.float32(1) / np.float32(448))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("M,K", [(1, 1), (5, 16), (128, 128), (129, 127), (64, 300), (300, 64), (257, 264), (16, 1000), (1000, 24), (127, 8)])
def test_quant(layer, M, K, rows, dt):
    x = rnd(1, M, K, dt=dt)
    x[0] *= 100
    x[M // 2] *= 1e-3
    if M > 3:
        x[3] = 0
    Q, scale, QT, scaleT = layer.quant_fp8(x.cuda(), rows=rows, transposed=True)
    q, s = quant_ref(x, rows)
    assert torch.equal(Q.float().cpu(), q) and torch.equal(scale.t().cpu(), s)
    q, s = quant_ref(x.t().contiguous(), rows)
    assert torch.equal(QT.float().cpu(), q) and torch.equal(scaleT.t().cpu(), s)
    for gap in (8, 3):
        for plain, turned in ((True, False), (False, True)):
            got = layer.quant_fp8(apart(x, gap), rows=rows, plain=plain, transposed=turned)
            for a, b in zip(got, (Q, scale, QT, scaleT)):
                assert a is None or torch.equal(a.view(torch.uint8) if a.dtype == E4 else a, b.view(torch.uint8) if b.dtype == E4 else b)


def test_quant_special_values(layer):
    x = rnd(1, 130, 260)
    x[2, 3], x[5, 200] = float("nan"), float("-inf")
    x[7] = 1e-38
    Q, scale = layer.quant_fp8(x.cuda())[:2]
    q, s = quant_ref(x, 1)
    assert torch.equal(Q.float().cpu().isnan(), q.isnan()) and Q[2, :128].float().isnan().all() and not Q[2, 128:].float().isnan().any()
    assert torch.equal(Q.float().cpu().nan_to_num(), q.nan_to_num()) and torch.equal(scale.t().cpu().nan_to_num(), s.nan_to_num())
    wide = torch.full((4, 48), 77, dtype=torch.uint8, device="cuda").view(E4)      # what lies behind a row stays
    st = layer.pf_quant_fp8(x[:4, :33].contiguous().cuda(), 33, wide, 48, scale, None, 0, None, 4, 33, 1, 0)
    torch.cuda.synchronize()
    assert st == 0 and (wide.view(torch.uint8)[:, 33:] == 77).all()


# ---- matmul

def e4m3(seed, R, C, std=60.0):
    """Random e4m3 values in rows of whole 16 bytes with NaN behind them, on the GPU, and as 64-bit numbers."""
    q = (rnd(seed, R, C) * std).clamp(-448, 448).to(E4)
    to = torch.full((R, (C + 15) // 16 * 16), 0x7f, dtype=torch.uint8)
    to[:, :C] = q.view(torch.uint8)
    return to.cuda().view(E4)[:, :C], q.double()


def check_matmul(layer, M, N, K, b_rows, dt, seed=1, **more):
    A, a = e4m3(seed, M, K)
    B, b = e4m3(seed + 1, N, K)
    nk, nb = -(-K // 128), N if b_rows == 1 else -(-N // 128)
    sa, sb = rnd(seed + 2, nk, M).exp() * 1e-2, rnd(seed + 3, nk, nb).exp() * 1e-2
    C = layer.matmul_fp8(A, sa.cuda(), B, sb.cuda(), b_rows=b_rows, out_dtype=dt, **more)
    a = a * sa.double().t().repeat_interleave(128, 1)[:, :K]
    b = b * sb.double().t().repeat_interleave(b_rows, 0)[:N].repeat_interleave(128, 1)[:, :K]
    ref = a @ b.t()
    near(C, ref, (2.0 ** -16 + (nk + 4) * U) * (a.abs() @ b.abs().t()) + HALF[dt] * ref.abs())
    return C


@pytest.mark.parametrize("b_rows", [1, 128])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 16, 128), (3, 100, 200), (16, 256, 1024), (17, 300, 129), (40, 64, 144), (64, 1000, 2080),
                                   (65, 130, 500), (100, 128, 4096), (128, 128, 128), (129, 257, 384), (200, 600, 1000), (256, 256, 256),
                                   (257, 255, 640), (300, 513, 96), (512, 1030, 1111), (1000, 40, 2500)])
def test_matmul(layer, M, N, K, b_rows):
    check_matmul(layer, M, N, K, b_rows, F32)
    check_matmul(layer, M, N, K, b_rows, BF)


@pytest.mark.parametrize("M,N,K", [(2048, 1024, 512), (1025, 2049, 1000), (2, 8192, 8192), (33, 4096, 4096), (300, 300, 8192), (130, 700, 8000)])
def test_matmul_large(layer, M, N, K):
    """Sizes of the large tiles, of few rows with many columns, and of K shared out between workgroups."""
    check_matmul(layer, M, N, K, 128, BF)
    check_matmul(layer, M, N, K, 1, F32)


@pytest.mark.parametrize("b_rows", [1, 128])
@pytest.mark.parametrize("N", [2112, 2050])
def test_matmul_last_columns_apart(layer, N, b_rows):
    """More tiles than compute units by a last column of them that is hardly there: a product of its own."""
    check_matmul(layer, 8192, N, 1024, b_rows, BF)


@pytest.mark.parametrize("M,N", [(5, 24), (300, 264), (300, 265)])
def test_matmul_into_wider_rows(layer, M, N):
    """C as columns of a wider array, where rows allow wide stores and where they do not; what is beside them stays."""
    A, _ = e4m3(1, M, 256)
    B, _ = e4m3(2, N, 256)
    sa, sb = torch.ones(2, M, device="cuda"), torch.ones(2, N, device="cuda")
    want = layer.matmul_fp8(A, sa, B, sb, b_rows=1)
    need = layer.pf_matmul_fp8_workspace_bytes(M, N, 256, 1)
    work = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    for wide in (N + 8, N + 3):
        C = torch.full((M, wide), 7.0, dtype=BF, device="cuda")
        assert layer.pf_matmul_fp8(A, 256, sa, B, 256, sb, 1, C, wide, M, N, 256, 1, work, need) == 0
        torch.cuda.synchronize()
        assert torch.equal(C[:, :N], want) and (C[:, N:] == 7).all()


def test_matmul_special_values(layer):
    """NaN in a row of A reaches that row of C and no other; scales of 0 and infinity count as they are."""
    for M, N in ((4, 48), (200, 300)):
        A, _ = e4m3(1, M, 256)
        B, _ = e4m3(2, N, 256)
        sa, sb = torch.ones(2, M, device="cuda"), torch.ones(2, N, device="cuda")
        want = layer.matmul_fp8(A, sa, B, sb, b_rows=1, out_dtype=F32)
        A.view(torch.uint8)[1, 130] = 0x7f
        sa[:, 2] = 0
        sb[1, 7] = float("inf")
        got = layer.matmul_fp8(A, sa, B, sb, b_rows=1, out_dtype=F32)
        assert got[1].isnan().all() and (got[2, torch.arange(N) != 7] == 0).all()
        rows = torch.tensor([i for i in range(M) if i not in (1, 2)], device="cuda")
        cols = torch.tensor([i for i in range(N) if i != 7], device="cuda")
        assert torch.equal(got[rows][:, cols], want[rows][:, cols]) and not got[rows, 7].isfinite().any()


def test_training_products(layer):
    """Forward, gradient of the input and of the weights from the quantiser's outputs, against the products of what these
    stand for."""
    M, N, K = 150, 200, 300
    x, w, dy = rnd(1, M, K, dt=BF), rnd(2, N, K, std=0.05), rnd(3, M, N, dt=BF, std=1e-3)
    value = lambda q, s, rows: q.double().cpu() * s.double().cpu().t().repeat_interleave(rows, 0)[:q.shape[0]].repeat_interleave(128, 1)[:, :q.shape[1]]  # noqa: E731
    X, sx, XT, sxT = layer.quant_fp8(x.cuda(), transposed=True)
    W, sw, WT, swT = layer.quant_fp8(w.cuda(), rows=128, transposed=True)
    Y, sy, YT, syT = layer.quant_fp8(dy.cuda(), transposed=True)
    assert torch.equal(value(W, sw, 128), value(WT, swT, 128).t())
    for got, a, b in ((layer.matmul_fp8(X, sx, W, sw, out_dtype=F32), value(X, sx, 1), value(W, sw, 128)),
                      (layer.matmul_fp8(Y, sy, WT, swT, out_dtype=F32), value(Y, sy, 1), value(WT, swT, 128)),
                      (layer.matmul_fp8(YT, syT, XT, sxT, b_rows=1, out_dtype=F32), value(YT, syT, 1), value(XT, sxT, 1))):
        near(got, a @ b.t(), 2.0 ** -15 * (a.abs() @ b.abs().t()))
    # and of the unrounded ones: an operand is off by 2^-4 of its size at most, about
    ref, size = dy.double().t() @ x.double(), dy.double().abs().t() @ x.double().abs()
    assert ((got.double().cpu() - ref).abs() <= size * 2.0 ** -3).all()


# ---- gated recurrence

def gate_ref(g, gate):
    a = g if gate == "value" else g.exp() if gate == "log" else g.sigmoid()
    return a, {"value": 1 - a, "log": -torch.expm1(g), "logit": torch.sigmoid(-g)}[gate], {"value": torch.ones_like(a), "log": a, "logit": a * torch.sigmoid(-g)}[gate]


def gated_ref(x, g, h0, gate, mix):
    """h [B, L, D] in 64 bits and its error bound."""
    x, g = x.double(), g.double()
    a, rest, _ = gate_ref(g, gate)
    b = rest * x if mix else x
    h = torch.zeros(x.shape[0], x.shape[2], dtype=torch.float64) if h0 is None else h0.double()
    e, hs, es = torch.zeros_like(h), torch.empty_like(x), torch.empty_like(x)
    c = 8 + 4 * g.abs().clamp(max=100) if gate != "value" else torch.full_like(g, 8.0)
    for t in range(x.shape[1]):
        e = a[:, t].abs() * e + U * (c[:, t] * (a[:, t] * h).abs() + c[:, t] * b[:, t].abs())
        h = a[:, t] * h + b[:, t]
        e = e + U * h.abs()
        hs[:, t], es[:, t] = h, 2 * e
    return hs, es


def gates(seed, B, L, D, gate, dt):
    g = rnd(seed, B, L, D, std=0.5) - torch.linspace(0, 6, D)      # log of 1 - a, about
    return ((-g) if gate == "logit" else -torch.nn.functional.softplus(g) if gate == "log" else torch.exp(-torch.nn.functional.softplus(g))).to(dt)


SHAPES = [(1, 1, 1), (2, 3, 5), (64, 1, 96), (1, 2, 64), (3, 17, 130), (2, 100, 64), (1, 255, 128), (2, 256, 256), (1, 257, 72), (2, 700, 33),
          (5, 1030, 48), (1, 4099, 264), (1, 9000, 16), (3, 513, 1000), (40, 300, 8)]


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("gate,mix", [("value", False), ("log", False), ("logit", True), ("log", True)])
@pytest.mark.parametrize("B,L,D", SHAPES)
def test_gated(layer, B, L, D, gate, mix, dt):
    x, g, h0 = rnd(1, B, L, D, dt=dt), gates(2, B, L, D, gate, dt), rnd(3, B, D)
    for h in (h0, None):
        ref, tol = gated_ref(x, g, h, gate, mix)
        Y, hL = layer.gated_fwd(x.cuda(), g.cuda(), None if h is None else h.cuda(), gate=gate, mix=mix)
        near(Y, ref, tol + HALF[dt] * ref.abs())
        near(hL, ref[:, -1], tol[:, -1])


def gated_grads(x, g, h0, y, dy, dh, gate, mix):
    """dX, dG, dh0 in 64 bits and their error bounds."""
    g, y, dy = g.double(), y.double(), dy.double()
    a, rest, slope = gate_ref(g, gate)
    h = torch.cat((h0.double()[:, None], y[:, :-1]), 1) - (x.double() if mix else 0)
    l = dh.double()
    e, ls, es = torch.zeros_like(l), torch.empty_like(dy), torch.empty_like(dy)
    c = 8 + 4 * g.abs().clamp(max=100) if gate != "value" else torch.full_like(g, 8.0)
    for t in range(g.shape[1] - 1, -1, -1):
        l = l + dy[:, t]
        e = e + U * (l.abs() + dy[:, t].abs())
        ls[:, t], es[:, t] = l, 2 * e
        e = a[:, t].abs() * e + U * c[:, t] * (a[:, t] * l).abs()
        l = a[:, t] * l
    k = rest if mix else 1
    size = torch.cat((h0.double()[:, None], y[:, :-1]), 1).abs() + (x.double().abs() if mix else 0)
    return ((ls * k, es * k + 16 * U * (c * ls * k).abs()), (ls * h * slope, (es * size * slope).abs() + 16 * U * (c * ls * slope).abs() * size),
            (l, 2 * e + 4 * U * l.abs()))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("gate,mix", [("value", True), ("log", False), ("logit", True)])
@pytest.mark.parametrize("B,L,D", SHAPES)
def test_gated_backward(layer, B, L, D, gate, mix, dt):
    x, g, h0 = rnd(1, B, L, D, dt=dt), gates(2, B, L, D, gate, dt), rnd(3, B, D)
    y, dy, dh = rnd(4, B, L, D, dt=dt), rnd(5, B, L, D, dt=dt), rnd(6, B, D)
    got = layer.gated_bwd(x.cuda() if mix else None, g.cuda(), y.cuda(), dy.cuda(), h0.cuda(), dh.cuda(), gate=gate, mix=mix)
    for out, (ref, tol), half in zip(got, gated_grads(x, g, h0, y, dy, dh, gate, mix), (HALF[dt], HALF[dt], 0)):
        near(out, ref, tol + half * ref.abs())


@pytest.mark.parametrize("gate,mix", [("value", False), ("value", True), ("log", False), ("log", True), ("logit", False), ("logit", True)])
def test_gated_backward_is_the_forwards_derivative(layer, gate, mix):
    B, L, D = 2, 300, 20
    x, g, h0 = rnd(1, B, L, D), gates(2, B, L, D, gate, F32), rnd(3, B, D)
    dy, dh = rnd(5, B, L, D), rnd(6, B, D)
    Y, _ = layer.gated_fwd(x.cuda(), g.cuda(), h0.cuda(), gate=gate, mix=mix)
    got = [t.double().cpu() for t in layer.gated_bwd(x.cuda(), g.cuda(), Y, dy.cuda(), h0.cuda(), dh.cuda(), gate=gate, mix=mix)]

    def loss(x, g, h0):
        h, _ = gated_ref(x, g, h0, gate, mix)
        return float((h * dy.double()).sum() + (h[:, -1] * dh.double()).sum())
    for k in range(3):      # x, g, h0 each along a direction of its own
        at, step = [x.double(), g.double(), h0.double()], 1e-6
        e = rnd(30 + k, *at[k].shape).double()
        up, down = list(at), list(at)
        up[k], down[k] = at[k] + step * e, at[k] - step * e
        diff = (loss(*up) - loss(*down)) / (2 * step)
        assert abs(diff - float((got[k] * e).sum())) < 2e-4 * (1 + float((got[k] * e).abs().sum()) ** 0.5 + abs(diff))


@pytest.mark.parametrize("dt", [BF, F32])
def test_gated_strides(layer, dt):
    """Parts of a wider array, tokens before sequences, and inputs that all sequences share."""
    B, L, D = 3, 140, 40
    x, g, dy, y, h0 = rnd(1, B, L, D, dt=dt), gates(2, B, L, D, "log", dt), rnd(5, B, L, D, dt=dt), rnd(4, B, L, D, dt=dt).cuda(), rnd(3, B, D).cuda()
    want = layer.gated_fwd(x.cuda(), g.cuda(), h0, mix=True)
    back = layer.gated_bwd(x.cuda(), g.cuda(), y, dy.cuda(), h0, mix=True)
    turn = lambda t: t.cuda().transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    for f in (lambda t: apart(t, 8), lambda t: apart(t, 5), turn):
        for a, b in zip(layer.gated_fwd(f(x), f(g), h0, mix=True), want):
            assert torch.equal(a, b)
        for a, b in zip(layer.gated_bwd(f(x), f(g), y, f(dy), h0, mix=True), back):
            assert torch.equal(a, b)
    same = x[:1].cuda().expand(B, L, D)
    for a, b in zip(layer.gated_fwd(same, g.cuda(), h0), layer.gated_fwd(same.contiguous(), g.cuda(), h0)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("L", [70, 1500, 5000])
def test_gated_packed_sequences(layer, L, dt):
    """A log of minus infinity (the type's lowest value does the same) starts anew: the parts are independent calls."""
    D, cut = 24, L // 3
    x, g = rnd(1, 1, L, D, dt=dt), gates(2, 1, L, D, "log", dt)
    for low in (float("-inf"), torch.finfo(dt).min):
        g[:, cut] = low
        ref, tol = gated_ref(x, g, None, "log", False)
        one, _ = gated_ref(x[:, cut:], g[:, cut:], None, "log", False)
        assert torch.equal(one, ref[:, cut:])
        near(layer.gated_fwd(x.cuda(), g.cuda())[0], ref, tol + HALF[dt] * ref.abs())
        dy, y = rnd(3, 1, L, D, dt=dt), ref.to(dt)
        zero = torch.zeros(1, D)
        got = layer.gated_bwd(None, g.cuda(), y.cuda(), dy.cuda())
        for out, (r, t), half in zip(got, gated_grads(x, g.clamp(min=-1e4), zero, y, dy, zero, "log", False), (HALF[dt], HALF[dt], 0)):
            near(out, r, t + half * r.abs())
        assert (got[1][:, cut] == 0).all()


FEW_CHAINS = [(1, 6000, 33), (2, 5500, 131), (1, 4099, 768), (1, 3500, 1030)]


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("B,L,D", FEW_CHAINS)
def test_gated_few_chains(layer, B, L, D, dt):
    """Long sequences of few channels against the formula, and bit for bit against the same ones among many."""
    x, g, h0, y, dy, dh = (rnd(1, B, L, D, dt=dt), gates(2, B, L, D, "log", dt), rnd(3, B, D), rnd(4, B, L, D, dt=dt), rnd(5, B, L, D, dt=dt),
                           rnd(6, B, D))
    ref, tol = gated_ref(x, g, h0, "log", True)
    Y, hL = layer.gated_fwd(x.cuda(), g.cuda(), h0.cuda(), mix=True)
    near(Y, ref, tol + HALF[dt] * ref.abs())
    near(hL, ref[:, -1], tol[:, -1])
    back = layer.gated_bwd(x.cuda(), g.cuda(), y.cuda(), dy.cuda(), h0.cuda(), dh.cuda(), mix=True)
    for out, (r, t), half in zip(back, gated_grads(x, g, h0, y, dy, dh, "log", True), (HALF[dt], HALF[dt], 0)):
        near(out, r, t + half * r.abs())
    many = lambda t: t.repeat(12, *[1] * (t.dim() - 1)).cuda()  # noqa: E731
    for one, all_ in zip((Y, hL), layer.gated_fwd(many(x), many(g), many(h0), mix=True)):
        assert torch.equal(all_, one.repeat(12, *[1] * (one.dim() - 1)))
    for one, all_ in zip(back, layer.gated_bwd(many(x), many(g), many(y), many(dy), many(h0), many(dh), mix=True)):
        assert torch.equal(all_, one.repeat(12, *[1] * (one.dim() - 1)))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("gate,mix", [("log", False), ("logit", True)])
@pytest.mark.parametrize("B,L,D", [(1, 12289, 256), (1, 14400, 33), (2, 17000, 131), (1, 16500, 900)])
def test_gated_few_chains_longer(layer, B, L, D, gate, mix, dt):
    """The lengths from which more tiles in front are listened to."""
    test_gated(layer, B, L, D, gate, mix, dt)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("gate,mix", [("value", False), ("logit", True)])
@pytest.mark.parametrize("B,L,D", [(1, 8300, 33), (1, 8193, 256), (1, 10000, 1024), (2, 8200, 514)])
def test_gated_backward_few_chains(layer, B, L, D, gate, mix, dt):
    """Both sides of the lengths and channels from which the backward's tiles are longer."""
    test_gated_backward(layer, B, L, D, gate, mix, dt)


@pytest.mark.parametrize("L", [40, 3000])
def test_gated_special_values(layer, L):
    """NaN stays in its channel and sequence and reaches no earlier token; gates above one that overflow a span's product."""
    B, D = 2, 70
    x, g = rnd(1, B, L, D), gates(2, B, L, D, "log", F32)
    clean = layer.gated_fwd(x.cuda(), g.cuda())[0]
    bad = x.clone()
    bad[1, L // 2, 33] = float("nan")
    Y = layer.gated_fwd(bad.cuda(), g.cuda())[0]
    assert Y[1, L // 2:, 33].isnan().all()
    hit = torch.zeros(B, L, D, dtype=torch.bool, device="cuda")
    hit[1, L // 2:, 33] = True
    assert torch.equal(Y[~hit], clean[~hit])
    # products of gates far above fp32's range, on a state that is zero until late
    a, x = torch.full((1, L, 4), 8.0), torch.zeros(1, L, 4)
    x[0, L - 5:] = 1.0
    near(layer.gated_fwd(x.cuda(), a.cuda(), gate="value")[0], gated_ref(x, a, None, "value", False)[0], 1e-2)
    dy = torch.zeros(1, L, 4)
    dy[0, :4] = 1.0
    back = layer.gated_bwd(None, a.cuda(), torch.zeros(1, L, 4, device="cuda"), dy.cuda(), gate="value")
    assert back[0].isfinite().all() and torch.equal(back[0][0, 0].cpu(), torch.full((4,), 585.0))


def test_gated_states(layer):
    """Token by token with the state carried on is the whole call; no tokens hand the state through; hL may be h0."""
    B, L, D = 5, 9, 130
    x, g, h0 = rnd(1, B, L, D).cuda(), gates(2, B, L, D, "log", F32).cuda(), rnd(3, B, D).cuda()
    Y, hL = layer.gated_fwd(x, g, h0)
    h = h0
    for t in range(L):
        y, h = layer.gated_fwd(x[:, t:t + 1], g[:, t:t + 1], h)
        assert torch.allclose(y[:, 0], Y[:, t], rtol=1e-5, atol=1e-6)
    assert torch.allclose(h, hL, rtol=1e-5, atol=1e-6)
    y, h = layer.gated_fwd(x[:, :0], g[:, :0], h0)
    assert y.shape == (B, 0, D) and torch.equal(h, h0)
    assert (layer.gated_fwd(x[:, :0], g[:, :0])[1] == 0).all()
    out = layer.gated_bwd(None, g[:, :0], x[:, :0].contiguous(), x[:, :0], h0, h0)
    assert out[0].shape == (B, 0, D) and torch.equal(out[2], h0)
    keep, y = h0.clone(), torch.empty_like(x)
    need = layer.pf_gated_workspace_bytes(B, L, D, 0)
    work = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    assert layer.pf_gated_fwd(x, L * D, D, g, L * D, D, keep, y, keep, B, L, D, 1, 0, 0, work, need) == 0
    torch.cuda.synchronize()
    assert torch.equal(keep, hL) and torch.equal(y, Y)


# ---- more values than 32 bits count: the last rows, on zeros before them, are those of a call of their own

def tail(rows, *shape, seed, dt=BF):
    t = torch.zeros(rows, *shape, dtype=dt, device="cuda")
    t[-300:] = rnd(seed, 300, *shape, dt=dt).cuda()
    return t


def test_norm_past_32_bits(layer):
    M, D = 2 ** 31 // 4096 + 301, 4096
    x, w, dy = tail(M, D, seed=1), rnd(2, D, dt=BF).cuda(), tail(M, D, seed=3)
    for one, all_ in zip(layer.norm_fwd(x[-300:], w, eps=EPS, fp8=True)[1:3], layer.norm_fwd(x, w, eps=EPS, fp8=True)[1:3]):
        assert torch.equal(one.view(torch.uint8), all_[-300:].view(torch.uint8))
    dx, dw = layer.norm_bwd(x, dy, w, eps=EPS)
    one, dw1 = layer.norm_bwd(x[-300:], dy[-300:], w, eps=EPS)
    assert torch.equal(dx[-300:], one)
    assert (dw - dw1).abs().max() < 1e-5 * dw1.abs().max() + 300 * U * (dy[-300:].float() * x[-300:].float()).abs().sum(0).max()


@pytest.mark.parametrize("rows", [1, 128])
def test_quantiser_past_32_bits(layer, rows):
    M, K = 2 ** 31 // 4096 + 320, 4096      # (a multiple of 128 and 64 more)
    x = tail(M, K, seed=1)
    Q, s, QT, sT = layer.quant_fp8(x, rows=rows, transposed=True)
    part = M // 128 * 128 - 128
    q1, s1, qt1, st1 = layer.quant_fp8(x[part:], rows=rows, transposed=True)
    bits = lambda t: t.view(torch.uint8)  # noqa: E731
    assert torch.equal(bits(Q[part:]), bits(q1)) and torch.equal(bits(QT[:, part:]), bits(qt1[:, :M - part]))
    assert torch.equal(s[:, part // rows:], s1) and torch.equal(sT[part // 128:], st1)


@pytest.mark.parametrize("M,N,K", [(2 ** 31 // 4096 + 333, 64, 4096), (64, 2 ** 31 // 4096 + 333, 4096), (2 ** 31 // 4096 + 333, 4160, 128)])
def test_matmul_past_32_bits(layer, M, N, K):
    A = torch.zeros(M, K, dtype=torch.float8_e4m3fn, device="cuda")
    B = torch.zeros(N, K, dtype=torch.float8_e4m3fn, device="cuda")
    A[-40:], B[-40:] = rnd(1, 40, K).cuda().to(A.dtype), rnd(2, 40, K).cuda().to(B.dtype)
    sa, sb = torch.ones(K // 128, M, device="cuda"), torch.ones(K // 128, N, device="cuda")
    for dt in (F32, BF):
        C = layer.matmul_fp8(A, sa, B, sb, b_rows=1, out_dtype=dt)
        a, b = A[-40:].double().cpu(), B[-40:].double().cpu()
        ref = a @ b.t()
        near(C[-40:, -40:], ref, (HALF[dt] + 2 ** -10 * (dt == BF) + K * U) * (a.abs() @ b.abs().t()))
        assert (C[:-40, -40:][:4].float() == 0).all() and (C[-40:, :4].float() == 0).all()


@pytest.mark.parametrize("B,L,D", [(1, 2 ** 31 // 2048 + 301, 2048), (2 ** 31 // 4096 + 301, 1, 4096), (2 ** 31 // 32768 + 301, 32, 1024)])
def test_gated_past_32_bits(layer, B, L, D):
    x, dy = (tail(B * L, D, seed=s).view(B, L, D) for s in (1, 2))
    g = torch.full_like(x, -0.5)
    Y, hL = layer.gated_fwd(x, g)
    dX, dG, dh0 = layer.gated_bwd(None, g, Y, dy)
    cut = (lambda t: t[:, -300:].contiguous()) if B == 1 else (lambda t: t[-9:].contiguous())
    ref, tol = gated_ref(cut(x).cpu(), cut(g).cpu(), None, "log", False)
    near(cut(Y), ref, tol + HALF[BF] * ref.abs())
    near(hL[-1], ref[-1, -1], tol[-1, -1])
    zero = torch.zeros(ref.shape[0], D)
    for out, (r, t) in zip((dX, dG), gated_grads(cut(x).cpu(), cut(g).cpu(), zero, cut(Y).cpu(), cut(dy).cpu(), zero, "log", False)):
        near(cut(out), r, t + HALF[BF] * r.abs())


# ---- as a user calls them

def _calls(layer):
    x, r, w = rnd(1, 600, 1024, dt=BF).cuda(), rnd(2, 600, 1024, dt=BF).cuda(), rnd(3, 1024, dt=BF).cuda()
    W, sw, _, _ = layer.quant_fp8(rnd(4, 640, 1024, std=0.03).cuda(), rows=128)
    g = gates(5, 2, 3000, 256, "log", BF).cuda()
    z, dz = rnd(6, 2, 3000, 256, dt=BF).cuda(), rnd(7, 2, 3000, 256, dt=BF).cuda()

    def go():
        S, Y, Q, scale = layer.norm_fwd(x, w, r, eps=EPS, fp8=True)
        C = layer.matmul_fp8(Q, scale, W, sw)
        few = layer.matmul_fp8(Q[:3], scale[:, :3].contiguous(), W, sw)
        h, hL = layer.gated_fwd(z, g)
        return [S, Y, Q.view(torch.uint8), scale, C, few, h, hL, *layer.norm_bwd(S, Y, w, r, eps=EPS),
                *layer.gated_bwd(None, g, h, dz), *(t.view(torch.uint8) for t in layer.quant_fp8(x, transposed=True))]
    return go


def test_the_same_bits_again_and_on_another_stream(layer):
    go = _calls(layer)
    want = go()
    torch.cuda.synchronize()
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(go(), want))
    other = torch.cuda.Stream()
    with torch.cuda.stream(other):
        got = go()
    other.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_stream_argument(layer):
    """`stream` (a stream or its handle) is where the call runs and whose memory it takes: work queued on the current stream, which
    still uses memory that is freed at once, is not disturbed, and the result does not wait for it."""
    x, g = rnd(1, 2, 4000, 256, dt=BF).cuda(), gates(2, 2, 4000, 256, "log", BF).cuda()
    want = layer.gated_fwd(x, g)
    back = layer.gated_bwd(None, g, want[0], x)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    for stream in (other, other.cuda_stream, torch.cuda.default_stream().cuda_stream):
        busy = torch.zeros(1 << 22, device="cuda")
        for _ in range(50):
            busy = busy + 1
        got = layer.gated_fwd(x, g, stream=stream)
        grads = layer.gated_bwd(None, g, want[0], x, stream=stream)
        torch.cuda.synchronize()
        assert (busy == 50).all()
        assert all(torch.equal(a, b) for a, b in zip((*got, *grads), (*want, *back)))


def test_in_a_graph(layer):
    """Captured once, replayed with eager work between: every replay gives the eager bits."""
    go = _calls(layer)
    want = [t.clone() for t in go()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        go()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = go()
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        go()
        torch.cuda.synchronize()
