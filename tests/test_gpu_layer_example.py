"""The example block against the same block in plain float32 operations, whole and token by token, and its gradients
against automatic ones.

Bars: an 8-bit rounding is off by 2^-4 of a value at most, 2.7 % of it in the mean square (values spread over a binade), and
a product of two such operands by 3.8 % of its norm, as the errors are independent; a branch goes through two
products (5.4 %), what a recurrence makes of the first not counted, and weight gradients through three operands of that kind
and one forward.  0.12 and 0.2 leave a factor of two."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ex():
    from paper_2504_00492_amd import example_layer
    return example_layer


def rel(a, b):
    return float((a.float() - b.float()).norm() / b.float().norm())


def norm(x, w):
    return x / (x.square().mean(-1, keepdim=True) + 1e-5).sqrt() * w.float()


def plain_gated(w, x, tokens, norm_w=None, xg_w=None, back_w=None):
    D = w.width
    xg = norm(x, w.norm_gated if norm_w is None else norm_w) @ (w.plain["xg"] if xg_w is None else xg_w).t()
    xg = xg.view(-1, tokens, 2 * D)
    a = torch.sigmoid(xg[..., D:] + w.bias_gate)
    h, out = torch.zeros_like(a[:, 0]), []
    for t in range(tokens):
        h = a[:, t] * h + (1 - a[:, t]) * xg[:, t, :D]
        out.append(h)
    return torch.stack(out, 1).view(-1, D) @ (w.plain["back"] if back_w is None else back_w).t()


def plain_delta(w, x, tokens):
    H, d, r = w.heads, w.d, w.r
    B = x.shape[0] // tokens
    p = (norm(x, w.norm_delta) @ w.plain["qkvb"].t()).view(B, tokens, -1)
    q, k, v, beta = p.split([H * d, H * r * d, H * r * d, H * r], 2)
    q, k, v, beta = q.reshape(B, tokens, H, d), k.reshape(B, tokens, H, r, d), v.reshape(B, tokens, H, r, d), beta.reshape(B, tokens, H, r).sigmoid()
    k = torch.nn.functional.normalize(k, dim=-1)
    S, out = torch.zeros(B, H, d, d, device=x.device), []
    for t in range(tokens):
        old = (k[:, t] @ S.transpose(-1, -2).contiguous()).contiguous()                    # [B, H, r, d_v]: S k
        S = S + ((beta[:, t, ..., None] * (v[:, t] - old)).transpose(-1, -2).contiguous() @ k[:, t].contiguous())
        out.append((S @ (q[:, t] * d ** -0.5)[..., None].contiguous())[..., 0])
    o = norm(torch.stack(out, 1).reshape(-1, d), w.norm_heads).view(-1, H * d)
    return o @ w.plain["out"].t()


def test_block_against_plain_operations(ex):
    B, tokens, w = 2, 70, ex.Weights(heads=2, d=64, r=2, seed=3)
    x = torch.randn((B * tokens, w.width), generator=torch.Generator().manual_seed(4)).cuda().bfloat16()
    stream, branch, _ = ex.delta_half(w, x, None, None, tokens)
    assert torch.equal(stream, x) and rel(branch, plain_delta(w, x.float(), tokens)) < 0.12
    stream, out, _ = ex.gated_half(w, stream, branch, None, tokens)
    assert torch.equal(stream, (x.float() + branch.float()).bfloat16())
    assert rel(out, plain_gated(w, stream.float(), tokens)) < 0.12


def test_token_by_token_is_the_prompt(ex):
    """The same roundings to 8 bits in both; what is left is the rounding of intermediates to bf16 and what 8 bits make of it."""
    B, tokens, w = 3, 40, ex.Weights(heads=2, d=64, r=1, seed=5)
    x = torch.randn((B, tokens, w.width), generator=torch.Generator().manual_seed(6)).cuda().bfloat16()
    _, whole, states = ex.block(w, x.view(-1, w.width), tokens=tokens)
    step, outs = (None, None), []
    for t in range(tokens):
        _, b, step = ex.block(w, x[:, t].contiguous(), step)
        outs.append(b)
    assert rel(torch.stack(outs, 1).view_as(whole), whole) < 0.05
    for a, b in zip(step, states):
        assert rel(a, b) < 0.05


def test_gradients_against_automatic_ones(ex):
    B, tokens, w = 2, 90, ex.Weights(heads=2, d=64, r=2, seed=7, training=True)
    gen = torch.Generator().manual_seed(8)
    x, dy, ds = (torch.randn((B * tokens, w.width), generator=gen).cuda().bfloat16() for _ in range(3))
    keep = {}
    ex.gated_half(w, x, None, None, tokens, keep)
    d_x, grads = ex.gated_half_backward(w, keep, dy, ds)
    leaves = [t.clone().float().requires_grad_() for t in (x, w.norm_gated, w.plain["xg"], w.plain["back"])]
    out = plain_gated(w, leaves[0], tokens, *leaves[1:])
    want = torch.autograd.grad((out * dy.float()).sum() + (leaves[0] * ds.float()).sum(), leaves)
    for got, ref in zip((d_x, grads["norm_gated"], grads["xg"], grads["back"]), want):
        assert rel(got, ref) < 0.2


def test_main_runs(ex, capsys):
    ex.main()
    assert "token by token" in capsys.readouterr().out
