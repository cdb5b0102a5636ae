"""A block of a linear transformer from this library's calls: the delta rule over heads, then a gated recurrence over channels,
each behind a norm and between projections in 8 bits.  Prompt, token by token with the states carried on, and the gradients of
the gated half.

    python -m paper_2504_00492_amd.example_layer          # on the GPU: runs all three, prints what they agree to

Only the orders of the axes (heads before tokens for the delta rule) and the slicing of the projections are PyTorch's.
"""
from __future__ import annotations

import torch

from . import binding as pf, layer

EPS = 1e-5


class Weights:
    """One block's weights: norms in bf16; projections in 8 bits, and with `training` their transposed copies."""

    def __init__(self, heads: int, d: int, r: int, *, seed: int = 0, training: bool = False, device="cuda"):
        self.heads, self.d, self.r = heads, d, r
        self.width = D = heads * d
        g = torch.Generator().manual_seed(seed)
        normal = lambda *s: torch.randn(s, generator=g).to(device)      # noqa: E731
        self.norm_delta, self.norm_heads, self.norm_gated = ((1 + 0.1 * normal(n)).bfloat16() for n in (D, d, D))
        # the gate's rows start out remembering: sigmoid of about 3
        self.plain = dict(qkvb=normal(D * (1 + 2 * r) + heads * r, D) * D ** -0.5, out=normal(D, D) * D ** -0.5,
                          xg=normal(2 * D, D) * D ** -0.5, back=normal(D, D) * D ** -0.5)
        self.bias_gate = 3.0
        self.packed = {k: layer.quant_fp8(w, rows=128, transposed=training) for k, w in self.plain.items()}


def project(w: Weights, name: str, q, scale):
    return layer.matmul_fp8(q, scale, *w.packed[name][:2])


def delta_half(w: Weights, stream, branch, state, tokens: int):
    """stream, branch [B * tokens, D] (branch: what is still to be added, or None), state [B, H, d, d] or None ->
    (the stream with the branch in it, the new branch, state)."""
    stream, _, q8, scale = layer.norm_fwd(stream, w.norm_delta, branch, eps=EPS, y=False, fp8=True)
    B, H, d, r = stream.shape[0] // tokens, w.heads, w.d, w.r
    q, k, v, beta = project(w, "qkvb", q8, scale).view(B, tokens, -1).split([H * d, H * r * d, H * r * d, H * r], 2)
    heads_first = lambda t, *s: t.reshape(B, tokens, H, *s).transpose(1, 2).contiguous()      # noqa: E731
    k = heads_first(k, r, d)
    k = torch.nn.functional.normalize(k.float(), dim=-1).bfloat16()
    o, state = pf.delta_fwd(heads_first(q, d) * d ** -0.5, k, heads_first(v, r, d), heads_first(beta, r).sigmoid(), state, chunk=64)
    o = layer.norm_fwd(o.transpose(1, 2).reshape(B * tokens * H, d), w.norm_heads, eps=EPS)[1]
    q8, scale = layer.quant_fp8(o.view(B * tokens, H * d))[:2]
    return stream, project(w, "out", q8, scale), state


def gated_half(w: Weights, stream, branch, state, tokens: int, keep=None):
    """The same for the gated recurrence, state [B, D] or None; `keep` (a dict) receives what the backward needs."""
    given = state
    stream, y, q8, scale = layer.norm_fwd(stream, w.norm_gated, branch, eps=EPS, y=keep is not None, fp8=True)
    D, B = w.width, stream.shape[0] // tokens
    xg = project(w, "xg", q8, scale).view(B, tokens, 2 * D)
    xg[..., D:] += w.bias_gate
    h, state = layer.gated_fwd(xg[..., :D], xg[..., D:], given, gate="logit", mix=True)
    q8, scale = layer.quant_fp8(h.view(B * tokens, D))[:2]
    if keep is not None:
        keep.update(stream=stream, y=y, xg=xg, h=h, state=given)
    return stream, project(w, "back", q8, scale), state


def gated_half_backward(w: Weights, keep, d_branch, d_stream):
    """Gradients of gated_half from those of its branch and of the stream behind it (all tokens of all sequences):
    of what came in as stream (and branch), of the weights by name."""
    D = w.width
    y8, ys, yt, yts = layer.quant_fp8(d_branch, transposed=True)
    h = keep["h"].view(-1, D)
    grads = {"back": layer.matmul_fp8(yt, yts, *layer.quant_fp8(h, plain=False, transposed=True)[2:], b_rows=1, out_dtype=torch.float32)}
    dh = layer.matmul_fp8(y8, ys, *w.packed["back"][2:]).view_as(keep["h"])
    xg = keep["xg"]
    dx, dg, _ = layer.gated_bwd(xg[..., :D], xg[..., D:], keep["h"], dh, keep["state"], gate="logit", mix=True)
    d_xg = torch.cat((dx, dg), 2).view(-1, 2 * D)
    q8, qs, qt, qts = layer.quant_fp8(d_xg, transposed=True)
    grads["xg"] = layer.matmul_fp8(qt, qts, *layer.quant_fp8(keep["y"], plain=False, transposed=True)[2:], b_rows=1, out_dtype=torch.float32)
    d_stream, grads["norm_gated"] = layer.norm_bwd(keep["stream"], layer.matmul_fp8(q8, qs, *w.packed["xg"][2:]), w.norm_gated, d_stream, eps=EPS)
    return d_stream, grads


def block(w: Weights, x, states=(None, None), tokens: int = 1):
    """x [B * tokens, D] bf16 -> (the stream, the branch still to be added to it, the two states)."""
    stream, branch, delta = delta_half(w, x, None, states[0], tokens)
    stream, branch, gated = gated_half(w, stream, branch, states[1], tokens)
    return stream, branch, (delta, gated)


def main() -> None:
    B, tokens, w = 2, 192, Weights(heads=4, d=64, r=2, training=True)
    g = torch.Generator().manual_seed(1)
    x = torch.randn((B, tokens, w.width), generator=g).cuda().bfloat16()
    stream, branch, _ = block(w, x.view(-1, w.width), tokens=tokens)
    whole = (stream.float() + branch.float()).view(B, tokens, -1)
    states, steps = (None, None), []
    for t in range(tokens):
        s, b, states = block(w, x[:, t].contiguous(), states)
        steps.append(s.float() + b.float())
    off = float((torch.stack(steps, 1) - whole).norm() / whole.norm())
    print(f"prompt of {tokens} tokens against token by token: {off:.2e}")
    keep = {}
    flat = x.view(-1, w.width)
    out = gated_half(w, flat, None, None, tokens, keep)[1]
    d_x, grads = gated_half_backward(w, keep, out, torch.zeros_like(out))
    print("gradients of |branch|^2 / 2:", ", ".join(f"{k} {float(v.float().norm()):.3g}" for k, v in dict(x=d_x, **grads).items()))


if __name__ == "__main__":
    main()
