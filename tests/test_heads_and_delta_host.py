"""Norm of heads with rotation and gated delta rule, without a GPU: what the C calls refuse on the host, before any pointer is looked at and any
work is enqueued, how large their workspaces are, and what the functions on tensors say of tensors that are not on a GPU."""
import pytest
import torch

from test_layer_host import layer  # noqa: F401  (fixture)

P = 1 << 20      # an address that is never followed
F32, BF16 = 0, 1
NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE = 1, 2, 3, 4, 5
BIG = (1 << 31) - 1


def _heads_fwd(pf, **k):
    a = dict(Q=P, qt=256, qh=64, K=P, kt=128, kh=64, wq=P, wk=P, table=P, far=100, positions=P, Yq=P, Yk=P, M=5, Hq=4, Hk=2, d=64, rot=32,
             norm=0, pairs=0, eps=1e-6, q_scale=1.0, dt=BF16, stream=0) | k
    return pf.pf_head_norm_fwd(*a.values())


def _heads_bwd(pf, **k):
    a = dict(Q=P, qt=256, qh=64, K=P, kt=128, kh=64, dYq=P, dyqt=256, dyqh=64, dYk=P, dykt=128, dykh=64, wq=P, wk=P, table=P, far=100, positions=P,
             dQ=P, dK=P, dwq=P, dwk=P, M=5, Hq=4, Hk=2, d=64, rot=32, norm=0, pairs=0, eps=1e-6, q_scale=1.0, dt=BF16, workspace=P,
             workspace_bytes=1 << 40, stream=0) | k
    return pf.pf_head_norm_bwd(*a.values())


def _arrays(names, outer):
    a = {}
    for n in names:
        a[n] = P
        for s in outer:
            a[n.lower() + s] = 64
    return a


def _delta_fwd(pf, **k):
    a = _arrays(("Q", "K", "V", "G", "beta"), "bth") | dict(S0=P, offsets=None, O=P, SL=P, N=2, L=100, Hk=2, Hv=4, dk=64, dv=64, dt=BF16, workspace=P,
                                                             workspace_bytes=1 << 40, stream=0)
    assert not set(k) - set(a)
    return pf.pf_gated_delta_fwd(*(a | k).values())


def _delta_bwd(pf, **k):
    a = _arrays(("Q", "K", "V", "G", "beta", "dO"), "bth") | dict(S0=P, dSL=P, offsets=None, dQ=P, dK=P, dV=P, dG=P, dbeta=P, dS0=P, N=2, L=100, Hk=2, Hv=4,
                                                                   dk=64, dv=64, dt=BF16, workspace=P, workspace_bytes=1 << 40, stream=0)
    assert not set(k) - set(a)
    return pf.pf_gated_delta_bwd(*(a | k).values())


def _delta_step(pf, **k):
    a = _arrays(("Q", "K", "V", "G", "beta"), "bh") | dict(S=P, slots=None, O=P, B=3, pool=3, Hk=2, Hv=4, dk=64, dv=64, dt=BF16, stream=0)
    assert not set(k) - set(a)
    return pf.pf_gated_delta_step(*(a | k).values())


REFUSED = [
    *[(_heads_fwd, {n: None}, NULL) for n in ("Q", "K", "table", "positions", "Yq", "Yk")],
    *[(_heads_bwd, {n: None}, NULL) for n in ("Q", "K", "dYq", "dYk", "table", "positions", "dQ", "dK")],
    *[(c, w, SHAPE) for c in (_heads_fwd, _heads_bwd) for w in (dict(M=-1), dict(Hq=-1), dict(Hk=-1), dict(d=0), dict(rot=-2), dict(rot=66), dict(rot=31),
                                                                 dict(far=-1), dict(qt=-1), dict(qh=-64), dict(kt=-1), dict(kh=-1))],
    (_heads_bwd, dict(dyqt=-1), SHAPE), (_heads_bwd, dict(dykh=-1), SHAPE),
    *[(c, w, UNSUPPORTED) for c in (_heads_fwd, _heads_bwd) for w in (dict(d=1025), dict(d=1011, rot=2), dict(d=BIG), dict(d=BIG, rot=BIG - 1), dict(norm=2),
                                                                       dict(norm=-1), dict(dt=2), dict(Hq=1 << 24), dict(Hq=BIG, Hk=BIG))],
    *[(c, w, ALIGN) for c in (_heads_fwd, _heads_bwd) for w in (dict(Q=P + 1), dict(K=P + 1), dict(Q=P + 2, dt=F32), dict(wq=P + 2), dict(wk=P + 8),
                                                                 dict(table=P + 4), dict(positions=P + 2))],
    (_heads_fwd, dict(Yq=P + 2), ALIGN), (_heads_fwd, dict(Yk=P + 8), ALIGN), (_heads_bwd, dict(dYq=P + 1), ALIGN), (_heads_bwd, dict(dQ=P + 8), ALIGN),
    (_heads_bwd, dict(dwk=P + 4), ALIGN), (_heads_bwd, dict(workspace=P + 4), ALIGN), (_heads_bwd, dict(workspace=None), WORKSPACE),
    (_heads_bwd, dict(workspace_bytes=255), WORKSPACE),
    *[(c, {n: None}, NULL) for c in (_delta_fwd, _delta_bwd, _delta_step) for n in ("Q", "K", "V", "G", "beta")],
    (_delta_fwd, dict(O=None), NULL), (_delta_step, dict(O=None), NULL), (_delta_step, dict(S=None), NULL),
    *[(_delta_bwd, {n: None}, NULL) for n in ("dO", "dQ", "dK", "dV", "dG", "dbeta")],
    *[(c, w, SHAPE) for c in (_delta_fwd, _delta_bwd, _delta_step) for w in (dict(Hk=0), dict(Hv=0), dict(Hk=3), dict(Hk=-1), dict(dk=0), dict(dv=0),
                                                                             dict(qh=-1), dict(kb=-1), dict(vh=-1), dict(gb=-1), dict(betah=-1))],
    *[(c, w, SHAPE) for c in (_delta_fwd, _delta_bwd) for w in (dict(N=-1), dict(L=-1), dict(qt=-1), dict(gt=-5))],
    (_delta_bwd, dict(dot=-1), SHAPE), (_delta_step, dict(B=-1), SHAPE), (_delta_step, dict(pool=-1), SHAPE), (_delta_step, dict(pool=2), SHAPE),
    *[(c, w, UNSUPPORTED) for c in (_delta_fwd, _delta_bwd, _delta_step) for w in (dict(dk=257), dict(dv=257), dict(dt=2), dict(dt=-1))],
    *[(c, w, ALIGN) for c in (_delta_fwd, _delta_bwd, _delta_step) for w in (dict(Q=P + 1), dict(K=P + 1), dict(V=P + 1), dict(G=P + 1), dict(beta=P + 2, dt=F32))],
    *[(c, w, ALIGN) for c in (_delta_fwd, _delta_bwd) for w in (dict(S0=P + 4), dict(offsets=P + 2), dict(workspace=P + 8))],
    (_delta_fwd, dict(O=P + 2), ALIGN), (_delta_fwd, dict(SL=P + 4), ALIGN), (_delta_bwd, dict(dSL=P + 4), ALIGN), (_delta_bwd, dict(dG=P + 2), ALIGN),
    (_delta_bwd, dict(dS0=P + 8), ALIGN), (_delta_step, dict(S=P + 4), ALIGN), (_delta_step, dict(O=P + 2), ALIGN), (_delta_step, dict(slots=P + 1), ALIGN),
]


@pytest.mark.parametrize("call,wrong,status", REFUSED)
def test_refusals(layer, call, wrong, status):  # noqa: F811
    assert call(layer, **wrong) == status


@pytest.mark.parametrize("call,sizes", [
    (_delta_fwd, dict(N=1, L=(1 << 30) + 1)), (_delta_bwd, dict(N=1, L=BIG)), (_delta_fwd, dict(N=1 << 24, L=64, Hk=1, Hv=1)),
    (_delta_fwd, dict(N=BIG, L=0, Hk=1, Hv=1)), (_delta_fwd, dict(N=1 << 19, L=1, Hk=1, Hv=1, dv=256)), (_delta_bwd, dict(N=1 << 16, L=1, Hk=1, Hv=8, dv=250)), (_delta_bwd, dict(N=1 << 20, L=1024, Hk=1, Hv=1)), (_delta_fwd, dict(N=BIG, L=1 << 30, Hk=1, Hv=1, offsets=P)),
    (_delta_bwd, dict(N=1, L=64, Hk=1, Hv=1 << 24)), (_delta_step, dict(B=1 << 24, pool=1 << 24, Hk=1, Hv=1)), (_delta_step, dict(B=BIG, pool=BIG)),
    (_delta_step, dict(B=1, pool=1, Hk=1, Hv=BIG)), (_heads_fwd, dict(M=BIG, Hq=1 << 23)), (_heads_fwd, dict(M=BIG, Hq=64, Hk=64, d=1024, rot=0))])
def test_more_than_a_launch_holds(layer, call, sizes):  # noqa: F811
    """Refused on the host, before any work."""
    assert call(layer, **sizes) == UNSUPPORTED


def test_nothing_to_do(layer):  # noqa: F811
    """Empty calls return at once, with no pointer looked at."""
    none = dict.fromkeys(("Q", "K"))
    assert _heads_fwd(layer, M=0, **none, table=None, positions=None, Yq=None, Yk=None) == 0
    assert _heads_fwd(layer, Hq=0, Hk=0, **none) == 0
    assert _heads_bwd(layer, M=0, **none, dYq=None, dYk=None, dwq=None, dwk=None, workspace=None) == 0
    none = dict.fromkeys(("Q", "K", "V", "G", "beta"))
    assert _delta_fwd(layer, N=0, **none, O=None, workspace=None) == 0
    assert _delta_fwd(layer, L=0, **none, O=None, SL=None, workspace=None) == 0
    assert _delta_bwd(layer, N=0, **none, dO=None, workspace=None) == 0
    assert _delta_bwd(layer, L=0, **none, dO=None, dS0=None, workspace=None) == 0
    assert _delta_step(layer, B=0, **none, S=None, O=None, pool=0) == 0


def test_workspaces(layer):  # noqa: F811
    """Refused one byte below what is asked for; no more than is written of them; none where there is nothing to do."""
    for N, L, Hk, Hv, dk, dv in ((1, 64, 1, 1, 64, 64), (3, 1000, 2, 4, 128, 128), (1, 65, 1, 3, 256, 40), (2, 1, 1, 1, 1, 1)):
        sizes = dict(N=N, L=L, Hk=Hk, Hv=Hv, dk=dk, dv=dv)
        for packed in (0, 1):
            for call, back in ((_delta_fwd, 0), (_delta_bwd, 1)):
                need = layer.pf_gated_delta_workspace_bytes(*sizes.values(), packed, back, BF16)
                chunks = (L + 63) // 64 * N if not packed else (L + 63 * min(N, L)) // 64
                rows = max(64, (dv + 31) // 32 * 32) * max(64, 1 << (dk - 1).bit_length())
                per = (3 if back else 2) * 18432 + 4096 + back * (2 * 4 * rows + 2 * 4 * 64 * ((dv + 31) // 32 * 32))
                assert 0 < need <= chunks * Hv * per + 4 * (3 * N + chunks) + 10 * 256, (sizes, packed, back)
                # (a packed call asks for its sequences' bounds besides)
                given = dict(workspace_bytes=need - 1, offsets=P if packed else None)
                assert call(layer, **sizes, **given) == WORKSPACE and call(layer, **sizes, **given | dict(workspace=None)) == WORKSPACE
    for sizes in ((0, 10, 1, 1, 64, 64), (1, 0, 1, 1, 64, 64), (1, 10, 1, 1, 257, 64), (1, 10, 2, 3, 64, 64), (BIG, BIG, 1, 1, 64, 64), (-1, 10, 1, 1, 64, 64)):
        assert layer.pf_gated_delta_workspace_bytes(*sizes, 0, 1, BF16) == 0
    for M, Hq, Hk, d, rot in ((1, 1, 0, 1, 0), (100, 4, 2, 64, 64), (1 << 20, 64, 8, 128, 128), (BIG, 1 << 23, 1, 1024, 0)):
        need = layer.pf_head_norm_bwd_workspace_bytes(M, Hq, Hk, d, rot)
        assert 0 < need <= 2048 * d * 4
        assert _heads_bwd(layer, M=M, Hq=Hq, Hk=Hk, d=d, rot=rot, workspace_bytes=need - 1) == WORKSPACE
    for sizes in ((0, 1, 1, 64, 64), (5, 0, 0, 64, 64), (5, -1, 1, 64, 64), (5, BIG, BIG, 64, 64), (5, 1, 1, 64, 65)):
        assert layer.pf_head_norm_bwd_workspace_bytes(*sizes) == 0


def test_supported(layer):  # noqa: F811
    assert all(layer.pf_head_norm_supported(d, r, t) for d, r in ((1, 0), (2, 2), (1010, 0), (1010, 2), (1010, 1010), (1024, 1024), (1024, 16)) for t in (F32, BF16))
    assert not any(layer.pf_head_norm_supported(*a) for a in ((0, 0, F32), (1025, 0, F32), (1024, 2, F32), (64, 3, F32), (64, 66, F32), (64, 64, 2), (64, -2, F32)))
    assert all(layer.pf_gated_delta_supported(*a, t) for a in ((1, 1, 1, 1), (2, 6, 256, 256), (5, 5, 72, 40)) for t in (F32, BF16))
    assert not any(layer.pf_gated_delta_supported(*a) for a in ((0, 1, 64, 64, F32), (2, 3, 64, 64, F32), (1, 1, 257, 64, F32), (1, 1, 64, 0, F32), (1, 1, 64, 64, 3), (1, 0, 64, 64, F32)))


def test_tensor_checks(layer):  # noqa: F811
    """The functions on tensors say what is wrong with an argument; there is no CPU path."""
    x, g, s = torch.zeros(1, 4, 2, 16), torch.zeros(1, 4, 2), torch.zeros(1, 2, 16, 16)
    for call in (lambda **k: layer.head_norm_fwd(x[0], eps=0.0, **k), lambda **k: layer.head_norm_bwd(x[0], None, x[0], None, eps=0.0, **k),
                 lambda **k: layer.gated_delta_fwd(x, x, x, g, g, **k), lambda **k: layer.gated_delta_bwd(x, x, x, g, g, x, **k),
                 lambda **k: layer.gated_delta_step(x[0], x[0], x[0], g[0], g[0], s, **k)):
        for k in ({}, {"stream": 0}, {"stream": 5}):
            with pytest.raises(ValueError, match="no CPU path"):
                call(**k)


def test_rotary_table(layer):  # noqa: F811
    """Angles in 64 bits, rounded once; an empty table and one of no columns too."""
    t = layer.rotary_table(7, 6, base=100.0, device="cpu")
    angle = torch.arange(7, dtype=torch.float64)[:, None] * 100.0 ** (-torch.tensor([0.0, 2.0, 4.0], dtype=torch.float64) / 6)
    assert t.dtype is torch.float32 and torch.equal(t, torch.cat((angle.cos(), angle.sin()), 1).float())
    assert layer.rotary_table(0, 4, device="cpu").shape == (0, 4) and layer.rotary_table(3, 0, device="cpu").shape == (3, 0)


@pytest.mark.parametrize("packed", [0, 1])
@pytest.mark.parametrize("back", [0, 1])
def test_a_workspace_does_for_smaller_calls(layer, packed, back):  # noqa: F811
    """Sized for the most sequences and tokens it is large enough for fewer of either, though what a call takes goes by how its sequences are cut."""
    for heads in ((1, 1, 128, 128), (1, 1, 64, 32), (1, 2, 256, 256), (2, 6, 72, 40), (1, 1, 1, 1), (5, 5, 200, 16)):
        for L in (1, 64, 2047, 2048, 4100, 16384, 65536):
            needs = [layer.pf_gated_delta_workspace_bytes(n, L, *heads, packed, back, BF16) for n in (*range(1, 60), 100, 200)]
            assert needs == sorted(needs), (heads, L)
            longer = layer.pf_gated_delta_workspace_bytes(8, L + 1000, *heads, packed, back, BF16)
            assert longer >= needs[7]
    for M in (1, 100, 1000, 4096, 8192, 9000, 100000):
        for Hq, Hk, d in ((32, 8, 128), (17, 1, 72), (1, 0, 16), (70, 9, 256)):
            assert layer.pf_head_norm_bwd_workspace_bytes(M, Hq, Hk, d, 16) <= layer.pf_head_norm_bwd_workspace_bytes(M + M // 3 + 1, Hq, Hk, d, 16)


@pytest.mark.parametrize("length,rot", [(5, 3), (5, -2), (-1, 4), (5, 1)])
def test_rotary_table_refuses(layer, length, rot):  # noqa: F811
    """An odd number of columns would come out as one more, with another pair's angles."""
    with pytest.raises(ValueError, match="even"):
        layer.rotary_table(length, rot, device="cpu")
