"""What the product of 8-bit matrices adds up, on values of very different sizes.

Into fp32 every product of two e4m3 numbers is exact and sums are fp32 ones: a block of 128 takes at most 127 additions, blocks are joined by
one fma each, and the product of the scales is rounded once: (128 + blocks + 4) u of the sum of the sizes, u = 2^-24; and where every partial
sum is a whole number below 2^24, in whatever order, there is no error at all.

Into bf16 the 8-bit instruction adds eight neighbouring products at a time and keeps of each what is 2^-13 of the largest's power of two or
more: of the other seven at most that much each is lost, 7 * 2^-13 of the largest of every eight, besides the bound above and the result's own
rounding.  The last test shows, without a GPU, that the first two bounds tell the one from the other."""
import pytest
import torch

from test_gpu_layer import BF, E4, F32, HALF, U, layer, near, rnd  # noqa: F401  (fixture)

gpu = pytest.mark.gpu

# few rows of A (three kernels), every tile, K shared out, a last column of tiles apart
SIZES = [(1, 40, 128), (3, 100, 200), (16, 256, 1024), (32, 64, 640), (40, 64, 144), (64, 1000, 384), (65, 130, 500), (128, 128, 2048), (200, 600, 1000),
         (257, 255, 640), (300, 300, 4096), (512, 1030, 1111), (1100, 2049, 256), (4096, 2112, 256)]


def rows(q):
    """e4m3 values in rows of whole 16 bytes, NaN behind them, on the GPU."""
    R, C = q.shape
    to = torch.full((R, (C + 15) // 16 * 16), 0x7f, dtype=torch.uint8)
    to[:, :C] = q.to(E4).view(torch.uint8)
    return to.cuda().view(E4)[:, :C]


def loud(M, N, K):
    """Whole numbers up to 15, and in every eight columns two loud ones whose products cancel."""
    a, b = rnd(1, M, K).mul(6).round().clamp(-15, 15), rnd(2, N, K).mul(6).round().clamp(-15, 15)
    k = torch.arange(K)
    a[:, k % 8 == 0], b[:, k % 8 == 0], a[:, k % 8 == 5], b[:, k % 8 == 5] = 448, 448, -448, 448
    return a, b


def patterns(seed, R, C):
    """Every finite e4m3 number alike: sizes from 2^-9 to 448."""
    g = torch.Generator().manual_seed(seed)
    t = torch.randint(0, 256, (R, C), generator=g, dtype=torch.int16)
    return torch.where(t % 128 == 127, t - 1, t).to(torch.uint8).view(E4).float()


def scaled(q, s, by):
    return q.double() * s.double().t().repeat_interleave(by, 0)[:q.shape[0]].repeat_interleave(128, 1)[:, :q.shape[1]]


def bounds(a, b, blocks):
    """The product in 64 bits and the two bounds."""
    ref, size = a @ b.t(), a.abs() @ b.abs().t()
    exact = (128 + blocks + 4) * U * size
    K = a.shape[1]
    pad = torch.nn.functional.pad
    aa, bb = (pad(t.abs(), (0, -K % 8)).view(t.shape[0], -1, 8) for t in (a, b))
    largest = torch.zeros_like(ref)
    for i in range(aa.shape[1]):
        top = aa[:, None, i, 0] * bb[None, :, i, 0]
        for e in range(1, 8):
            top = torch.maximum(top, aa[:, None, i, e] * bb[None, :, i, e])
        largest += top
    return ref, exact, exact + 7 * 2.0 ** -13 * largest


@gpu
@pytest.mark.parametrize("b_rows", [1, 128])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_whole_numbers_are_exact_in_fp32(layer, M, N, K, b_rows):  # noqa: F811
    a, b = loud(M, N, K)
    nk = -(-K // 128)
    sa, sb = torch.ones(nk, M, device="cuda"), torch.ones(nk, N if b_rows == 1 else -(-N // 128), device="cuda")
    C = layer.matmul_fp8(rows(a), sa, rows(b), sb, b_rows=b_rows, out_dtype=F32)
    assert torch.equal(C.double().cpu(), a.double() @ b.double().t())


@gpu
@pytest.mark.parametrize("b_rows", [1, 128])
@pytest.mark.parametrize("M,N,K", [s for s in SIZES if s[0] * s[1] <= 200 * 600])
def test_all_sizes_of_numbers(layer, M, N, K, b_rows):  # noqa: F811
    a, b = patterns(1, M, K), patterns(2, N, K)
    nk = -(-K // 128)
    sa, sb = rnd(3, nk, M).exp() * 1e-2, rnd(4, nk, N if b_rows == 1 else -(-N // 128)).exp() * 1e-2
    ref, exact, eights = bounds(scaled(a, sa, 1), scaled(b, sb, b_rows), nk)
    for dt, tol in ((F32, exact), (BF, eights)):
        C = layer.matmul_fp8(rows(a), sa.cuda(), rows(b), sb.cuda(), b_rows=b_rows, out_dtype=dt)
        near(C, ref, tol + HALF[dt] * (ref.abs() + tol))


@gpu
@pytest.mark.parametrize("M,N,K", [(3, 100, 200), (65, 130, 500), (200, 600, 1000)])
def test_loud_columns_into_bf16(layer, M, N, K):  # noqa: F811
    a, b = loud(M, N, K)
    nk = -(-K // 128)
    ref, _, tol = bounds(a.double(), b.double(), nk)
    C = layer.matmul_fp8(rows(a), torch.ones(nk, M, device="cuda"), rows(b), torch.ones(nk, N, device="cuda"), b_rows=1, out_dtype=BF)
    near(C, ref, tol + HALF[BF] * (ref.abs() + tol))


def test_the_bounds_tell_the_sums_apart():
    """Sums that drop what the 8-bit instruction drops are outside both bounds of fp32 results and inside that of bf16 ones."""
    def dropping(a, b):
        p = (a[:, None, :] * b[None, :, :]).view(a.shape[0], b.shape[0], -1, 8)
        unit = 2.0 ** (torch.floor(torch.log2(p.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -40))) - 13)
        return (torch.trunc(p / unit) * unit).sum((-1, -2))
    a, b = (t.double() for t in loud(9, 17, 128))
    assert not torch.equal(dropping(a, b), a @ b.t())
    assert ((dropping(a, b) - a @ b.t()).abs() <= bounds(a, b, 1)[2]).all()
    a, b = patterns(1, 20, 256).double(), patterns(2, 30, 256).double()
    ref, exact, eights = bounds(a, b, 2)
    off = (dropping(a, b) - ref).abs()
    assert (off > 4 * exact).sum() > 10 and (off <= eights).all()
