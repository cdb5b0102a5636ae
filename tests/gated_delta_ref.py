"""The gated delta rule and the heads' norm with rotation in 64 bits, written from their definitions token by token; gradients are
autograd's of these.  Used by the tests; shares no code with the library."""
import torch

D = torch.float64


def delta(Q, K, V, G, beta, S0=None):
    """Q, K [B, L, Hk, dk], V [B, L, Hv, dv], G, beta [B, L, Hv], S0 [B, Hv, dv, dk] or None, all float64 -> O, S_L."""
    B, L, Hk, dk = Q.shape
    Hv, dv = V.shape[2:]
    Q, K = (t.repeat_interleave(Hv // Hk, 2) for t in (Q, K))
    S = torch.zeros(B, Hv, dv, dk, dtype=D, device=Q.device) if S0 is None else S0
    O = []
    for t in range(L):
        S = S * torch.exp(G[:, t])[..., None, None]
        e = V[:, t] - (S * K[:, t, :, None]).sum(-1)
        S = S + (beta[:, t, :, None] * e)[..., None] * K[:, t, :, None]
        O.append((S * Q[:, t, :, None]).sum(-1))
    return torch.stack(O, 1) if O else V.clone(), S


def delta_grads(args, dO, dSL):
    """Gradients of <O, dO> + <S_L, dSL> with respect to args (None stays None)."""
    args = [None if a is None else a.detach().clone().requires_grad_() for a in args]
    O, S = delta(*args)
    total = (O * dO).sum() + (0 if dSL is None else (S * dSL).sum())
    there = [a for a in args if a is not None]
    grads = iter(torch.autograd.grad(total, there, allow_unused=True))
    return [None if a is None else next(grads) for a in args]


def heads(X, w, table, positions, norm, eps, scale, pairs):
    """X [M, H, d] float64 -> scale * turn(X / n * w)."""
    d = X.shape[-1]
    size = torch.sqrt((X * X).sum(-1, keepdim=True) / (d if norm == "rms" else 1) + eps)
    y = X / size * (1 if w is None else w)
    if table is not None:
        rot = table.shape[1]
        row = table.to(D)[positions.long()][:, None]
        c, s = row[..., :rot // 2], row[..., rot // 2:]
        i = torch.arange(rot // 2, device=X.device)
        a, b = (2 * i, 2 * i + 1) if pairs else (i, i + rot // 2)
        out = y.clone()
        out[..., a] = y[..., a] * c - y[..., b] * s
        out[..., b] = y[..., a] * s + y[..., b] * c
        y = out
    return y * scale


def off(got, want):
    """2-norm of the difference over that of what is wanted (which alone decides where it is zero)."""
    got, want = got.double(), want.double().to(got.device)
    assert got.shape == want.shape, (got.shape, want.shape)
    assert bool(torch.isfinite(got).all()), "not finite"
    n = float(want.norm())
    return float((got - want).norm()) / (n if n else 1.0) if got.numel() else 0.0
