"""The gated delta rule and what stands in front of it, as sized cases: the norm of every head of queries and keys with the
rotation by position, the recurrence over whole and packed sequences, its gradients, and one token against a pool of states.
Everything goes through paper_2504_00492_amd.layer.

A case is a dict of plain values; "op" says which call it is:
  heads        M tokens, Hq heads of queries and Hk of keys, width d; norm "rms" (with weights) or "l2"; rot: how many of the
               d values are turned by the token's position (0: none), in halves or in neighbouring pairs
  heads_grad   its backward: gradients of the heads and of the weights
  delta        S_t = exp(g_t) S_{t-1} (I - beta_t k_t k_t^T) + beta_t v_t k_t^T, o_t = S_t q_t over B sequences of L tokens, Hv heads
               of d_v values, each Hv / Hk of which share a head of queries and keys of d_k; state in and out.  "tokens": packed
               instead, B sequences of different lengths in that many rows
  delta_grad   its backward
  step         one token of B sequences, their states in a pool, in place
"""
import math

import torch

own = False

DTYPES = {"bf16": (torch.bfloat16, 2), "f32": (torch.float32, 4)}
EPS = 1e-6
FAR = 131072     # positions of the rotation's table
BASE = 10000.0


def listed():
    return [
        # one new token of four sequences, 32 heads of 128 on either side: serving, what a call costs
        dict(name="heads, tokens", op="heads", dtype="bf16", M=4, Hq=32, Hk=32, d=128, norm="l2", rot=128, pairs=False),
        # a long prompt, queries and keys as configuration 4 has them
        dict(name="heads, prompt", op="heads", dtype="bf16", M=65536, Hq=32, Hk=32, d=128, norm="l2", rot=128, pairs=False),
        # odd sizes in fp32: few heads of keys, a part of each turned, in pairs
        dict(name="heads, ragged fp32", op="heads", dtype="f32", M=4099, Hq=14, Hk=3, d=72, norm="rms", rot=40, pairs=True),
        # training: a batch one token short of even, weights of the norm
        dict(name="heads backward", op="heads_grad", dtype="bf16", M=16383, Hq=32, Hk=16, d=128, norm="rms", rot=64, pairs=False),
        # one token of one sequence: serving, what a call costs
        dict(name="delta, token", op="step", dtype="bf16", B=1, Hk=16, Hv=32, dk=128, dv=128),
        # one token of 256 sequences out of a pool: the states are what is read and written
        dict(name="delta, tokens of many", op="step", dtype="bf16", B=256, Hk=16, Hv=32, dk=128, dv=128),
        # configuration 4's length, heads and widths: one long prompt
        dict(name="delta, long", op="delta", dtype="bf16", B=1, L=65536, tokens=0, Hk=32, Hv=32, dk=128, dv=128, s0=False),
        # configuration 2's, pairs of heads sharing queries and keys, states carried on
        dict(name="delta, batch", op="delta", dtype="bf16", B=4, L=4096, tokens=0, Hk=8, Hv=16, dk=128, dv=128, s0=True),
        # prompts of 37 requests as they come, packed one behind the other
        dict(name="delta, packed", op="delta", dtype="bf16", B=37, L=1024, tokens=8191, Hk=8, Hv=8, dk=64, dv=64, s0=True),
        # odd sizes in fp32
        dict(name="delta, ragged fp32", op="delta", dtype="f32", B=3, L=1023, tokens=0, Hk=5, Hv=5, dk=72, dv=40, s0=True),
        # training: configuration 3's length and heads
        dict(name="delta backward", op="delta_grad", dtype="bf16", B=2, L=8192, tokens=0, Hk=16, Hv=16, dk=128, dv=128, s0=False),
        # training at configuration 1's width, packed, with heads that share queries and keys
        dict(name="delta backward, packed", op="delta_grad", dtype="bf16", B=9, L=2048, tokens=8190, Hk=4, Hv=8, dk=64, dv=64, s0=True),
    ]


def draw(rng):
    def size(lo, hi):
        hi = max(lo, int(hi))
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return max(lo, min(hi, n if rng.random() < 0.5 else n // 16 * 16 or n))

    op = rng.choice(("heads", "heads_grad", "delta", "delta", "delta_grad", "delta_grad", "step"))
    dtype = "bf16" if rng.random() < 0.75 else "f32"
    wide = 1 if dtype == "bf16" else 2
    if op in ("heads", "heads_grad"):
        d = size(16, 256)
        Hk = size(1, 32)
        Hq = Hk * rng.choice((1, 1, 2, 4))
        M = size(1, min(131072, (65536 if op == "heads" else 16383) * 48 * 128 / (Hq + Hk) / d / wide))
        rot = rng.choice((0, d // 2 * 2, d // 4 * 2))
        return dict(op=op, dtype=dtype, M=M, Hq=Hq, Hk=Hk, d=d, norm=rng.choice(("l2", "rms")), rot=rot, pairs=rng.random() < 0.3)
    dk, dv = rng.choice((16, 32, 64, 64, 96, 128, 128, size(8, 256))), rng.choice((16, 32, 64, 64, 96, 128, 128, size(8, 256)))
    Hk = size(1, 16)
    Hv = Hk * rng.choice((1, 1, 2))
    if op == "step":
        return dict(op=op, dtype=dtype, B=size(1, min(1024, 256 * 32 * 128 * 128 / Hv / dk / dv)), Hk=Hk, Hv=Hv, dk=dk, dv=dv)
    # as much to do as the largest listed case at most: rows count for their padding to widths of 64 as well
    room = (65536 * 32 if op == "delta" else 8192 * 32) * 128 * 128 / Hv / (max(dk, 64) * max(dv, 64)) / wide / wide
    L = size(1, min(65536 if op == "delta" else 8192, room))
    B = size(1, min(64, room / L))
    packed = rng.random() < 0.4
    return dict(op=op, dtype=dtype, B=B, L=L, tokens=max(1, B * L // 2 + rng.randrange(7)) if packed else 0, Hk=Hk, Hv=Hv, dk=dk, dv=dv,
                s0=rng.random() < 0.5)


# ---- inputs

def _lengths(case):
    """Lengths of packed sequences: any from none to L, all together in the rows there are; the same ones for each seed, as sizes are."""
    g = torch.Generator()
    g.manual_seed(case["B"] * 1000003 + case["L"] * 1009 + case["tokens"])
    n = (torch.rand(case["B"], generator=g) * (case["L"] + 1)).long().clamp(max=case["L"])
    n = n * min(case["tokens"], int(n.sum())) // max(1, int(n.sum()))
    n[0] += int(n.sum()) == 0
    return n


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = DTYPES[case["dtype"]][0]

    def n(*shape, std=1.0, mean=0.0, to=dt):
        return torch.randn(shape, generator=g, device="cuda").mul_(std).add_(mean).to(to)

    op, s = case["op"], dict(case=case)
    if op in ("heads", "heads_grad"):
        M, Hq, Hk, d, rot = (case[k] for k in ("M", "Hq", "Hk", "d", "rot"))
        both = n(M, (Hq + Hk) * d)      # what one projection gives: queries and keys side by side
        s["Q"], s["K"] = both[:, :Hq * d].unflatten(1, (Hq, d)), both[:, Hq * d:].unflatten(1, (Hk, d))
        s["wq"], s["wk"] = (n(d, std=0.1, mean=1.0), n(d, std=0.1, mean=1.0)) if case["norm"] == "rms" else (None, None)
        s["table"] = s["positions"] = None
        if rot:
            turn = torch.arange(FAR, dtype=torch.float64, device="cuda")[:, None] * BASE ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
            s["table"] = torch.cat((turn.cos(), turn.sin()), 1).float()
            at = int(torch.randint(0, FAR - 1, (1,), generator=g, device="cuda"))
            s["positions"] = ((torch.arange(M, device="cuda") + at) % FAR).int()
        if op == "heads_grad":
            s["dQ"], s["dK"] = n(M, Hq, d, std=1e-2), n(M, Hk, d, std=1e-2)
        return s

    B, Hk, Hv, dk, dv = (case[k] for k in ("B", "Hk", "Hv", "dk", "dv"))
    packed = case.get("tokens", 0)
    rows = (1, packed) if packed else (B, 1 if op == "step" else case["L"])
    unit = torch.nn.functional.normalize
    # keys that lie somewhat together, as those of neighbouring tokens do; heads that remember from some tokens to some thousands
    q = unit(n(*rows, Hk, dk, to=torch.float32), dim=-1).mul_(dk ** -0.5)
    k = unit(n(*rows, Hk, dk, to=torch.float32).add_(n(Hk, dk, std=0.5, to=torch.float32)), dim=-1)
    both = torch.cat((q.flatten(2), k.flatten(2)), 2).to(dt)
    s["Q"], s["K"] = both[..., :Hk * dk].unflatten(2, (Hk, dk)), both[..., Hk * dk:].unflatten(2, (Hk, dk))
    s["V"] = n(*rows, Hv, dv)
    slow = torch.rand(Hv, generator=g, device="cuda").mul_(-6.0).sub_(1.0)
    s["G"] = (-torch.nn.functional.softplus(n(*rows, Hv, std=0.5, to=torch.float32).add_(slow))).to(dt)
    s["beta"] = n(*rows, Hv, to=torch.float32).sigmoid_().to(dt)
    if op == "step":
        for name in ("Q", "K", "V", "G", "beta"):
            s[name] = s[name][:, 0]
        s["S"] = n(B + 3, Hv, dv, dk, std=0.3, to=torch.float32)
        s["slots"] = torch.randperm(B + 3, generator=g, device="cuda")[:B].int()
        return s
    s["S0"] = n(B, Hv, dv, dk, std=0.3, to=torch.float32) if case["s0"] else None
    s["offsets"] = None
    if packed:
        lengths = _lengths(case)
        s["longest"] = int(lengths.max())
        s["offsets"] = torch.cat((torch.zeros(1, dtype=torch.long), torch.cumsum(lengths, 0))).int().cuda()
    if op == "delta_grad":
        s["dO"], s["dSL"] = n(*rows, Hv, dv, std=1e-2), n(B, Hv, dv, dk, std=1e-2, to=torch.float32)
    if packed:      # (rows behind the last sequence are nobody's: no output is looked at there)
        s["end"] = int(lengths.sum())
    return s


# ---- one pass

def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        from paper_2504_00492_amd import layer

        if op in ("heads", "heads_grad"):
            how = dict(norm=case["norm"], eps=EPS, q_scale=case["d"] ** -0.5, pairs=case["pairs"])
            heads, rest = (state["Q"], state["K"]), (state["wq"], state["wk"], state["table"], state["positions"])
            if op == "heads":
                return layer.head_norm_fwd(*heads, *rest, **how)
            return _present(layer.head_norm_bwd(*heads, state["dQ"], state["dK"], *rest, **how))
        if op == "step":
            return layer.gated_delta_step(state["Q"], state["K"], state["V"], state["G"], state["beta"], state["S"], state["slots"]), state["S"]
        given = (state["Q"], state["K"], state["V"], state["G"], state["beta"])
        if op == "delta":
            O, SL = layer.gated_delta_fwd(*given, state["S0"], offsets=state["offsets"])
            return _told(state, O), SL
        *grads, dS0 = layer.gated_delta_bwd(*given, state["dO"], state["S0"], state["dSL"], offsets=state["offsets"])
        return tuple(_told(state, t) for t in grads) + (dS0,)
    if op == "heads":
        return tuple(_heads(state, case, *x)[0] for x in (("Q", "wq", case["d"] ** -0.5), ("K", "wk", 1.0)))
    if op == "heads_grad":
        (dq, dwq), (dk, dwk) = (_heads_grad(state, case, *x) for x in (("Q", "dQ", "wq", case["d"] ** -0.5), ("K", "dK", "wk", 1.0)))
        return _present((dq, dk, dwq, dwk))
    if op == "step":
        return _step(state)
    return _delta(state, case) if op == "delta" else _delta_grad(state, case)


def _present(outputs):
    return tuple(t for t in outputs if t is not None)


def _told(state, t):
    return t[:, :state["end"]] if state["offsets"] is not None else t


def _turned(x, state, case, back=1):
    """x [M, H, d] with its first `rot` values turned by the angles of the rows' positions (back = -1: the other way)."""
    rot = case["rot"]
    if not rot:
        return x
    row = state["table"][state["positions"].long()].to(x.dtype)[:, None]
    c, s = row[..., :rot // 2], row[..., rot // 2:] * back
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if case["pairs"] else (x[..., :rot // 2], x[..., rot // 2:rot])
    a, b = a * c - b * s, a * s + b * c
    both = torch.stack((a, b), -1).flatten(-2) if case["pairs"] else torch.cat((a, b), -1)
    return torch.cat((both, x[..., rot:]), -1)


def _heads(state, case, name, weight, scale):
    x = state[name].float()
    squares = (x * x).sum(-1, keepdim=True)
    rho = 1 / torch.sqrt((squares / case["d"] if case["norm"] == "rms" else squares) + EPS)
    xh = x * rho
    w = 1.0 if state[weight] is None else state[weight].float()
    return (_turned(xh * w, state, case) * scale).to(state[name].dtype), xh, rho, w


def _heads_grad(state, case, name, grad, weight, scale):
    _, xh, rho, w = _heads(state, case, name, weight, scale)
    dy = _turned(state[grad].float() * scale, state, case, -1)
    g = dy * w
    along = (g * xh).sum(-1, keepdim=True)
    dx = rho * (g - xh * (along / case["d"] if case["norm"] == "rms" else along))
    return dx.to(state[name].dtype), None if state[weight] is None else (dy * xh).sum((0, 1))


def _step(state):
    dt, slots = state["Q"].dtype, state["slots"].long()
    share = state["V"].shape[1] // state["Q"].shape[1]
    q, k = (state[n].float().repeat_interleave(share, 1)[..., None] for n in ("Q", "K"))
    S = state["S"][slots] * torch.exp(state["G"].float())[..., None, None]
    e = (state["V"].float()[..., None] - S @ k) * state["beta"].float()[..., None, None]
    S = S + e * k.transpose(-1, -2)
    state["S"][slots] = S
    return (S @ q)[..., 0].to(dt), state["S"]


CHUNK = 64


def _sequences(state, case, *names):
    """The named arrays [.., tokens, H, ..] as [B, H, tokens, ..] in 32 bits, packed ones a sequence to a row; zeros behind each."""
    L = state["longest"] if state["offsets"] is not None else case["L"]
    whole = max(1, -(-L // CHUNK)) * CHUNK
    out = []
    for t in names:
        if state["offsets"] is not None:
            at, there = _places(state, whole)
            t = t[0][at] * there.view(*there.shape, *[1] * (t.dim() - 2)).to(t.dtype)
        elif whole > L:
            t = torch.cat((t, t.new_zeros(t.shape[0], whole - L, *t.shape[2:])), 1)
        out.append(t.float().transpose(1, 2))
    return out


def _places(state, whole):
    """Rows of the packed sequences' tokens [B, whole], and which of them there are."""
    first, last = state["offsets"][:-1, None].long(), state["offsets"][1:, None].long()
    at = first + torch.arange(whole, device="cuda")
    return at.clamp(max=state["V"].shape[1] - 1), at < last


def _back(state, case, t, dtype):
    """[B, H, tokens, ..] -> the outputs' layout and type."""
    t = t.transpose(1, 2)
    if state["offsets"] is not None:
        return t[_places(state, t.shape[1])[1]][None].to(dtype)
    return t[:, :case["L"]].to(dtype)


def _below(X):
    """(I + X)^-1 for X strictly below the diagonal, [.., CHUNK, CHUNK]: inverses of blocks of 1, 2, 4, ... joined."""
    T, s = torch.eye(CHUNK, device="cuda").expand(X.shape), 1
    row, col = torch.arange(CHUNK, device="cuda")[:, None], torch.arange(CHUNK, device="cuda")
    while s < CHUNK:
        pairs = (row // (2 * s) == col // (2 * s)) & (row // s > col // s)      # the lower left block of each two
        T = T - T @ (X * pairs) @ T
        s *= 2
    return T


def _flow(q, k, v, g, beta, S):
    """The recurrence over [B, H, tokens, ..] in 32 bits, a chunk at a time: (I + A) U = beta (V - decay K S^T) with
    A = beta (K K^T) decay strictly below the diagonal, o = decay S q + (Q K^T) decay U, S' = decay S + U^T K decay."""
    B, H, L, _ = q.shape
    q, k, v, g, beta = (t.unflatten(2, (L // CHUNK, CHUNK)) for t in (q, k, v, g, beta))
    total = torch.cumsum(g.double(), 3)      # (sums of many gates, whose differences are what counts)
    row, col = torch.arange(CHUNK, device="cuda")[:, None], torch.arange(CHUNK, device="cuda")
    decay = torch.exp((total[..., :, None] - total[..., None, :]).masked_fill(row < col, -math.inf).float())
    T = _below((k @ k.transpose(-1, -2)) * decay * beta[..., None] * (row > col)) * beta[..., None, :]
    P = (q @ k.transpose(-1, -2)) * decay
    since = torch.exp(total.float())[..., None]
    later = k * torch.exp((total[..., -1:] - total).float())[..., None]
    across, whole = k * since, since[..., -1:, :]
    out = []
    for c in range(L // CHUNK):      # (the chunks' states come one from the other)
        St = S.transpose(-1, -2)
        U = T[:, :, c] @ (v[:, :, c] - across[:, :, c] @ St)
        out.append(since[:, :, c] * (q[:, :, c] @ St) + P[:, :, c] @ U)
        S = whole[:, :, c] * S + U.transpose(-1, -2) @ later[:, :, c]
    return torch.cat(out, 2), S


def _first_state(state, case):
    if state["S0"] is not None:
        return state["S0"]
    return torch.zeros(case["B"], case["Hv"], case["dv"], case["dk"], device="cuda")


def _delta(state, case):
    share = case["Hv"] // case["Hk"]
    q, k, v, g, beta = _sequences(state, case, *(state[n] for n in ("Q", "K", "V", "G", "beta")))
    if share > 1:
        q, k = q.repeat_interleave(share, 1), k.repeat_interleave(share, 1)
    O, S = _flow(q, k, v, g, beta, _first_state(state, case))
    return _back(state, case, O, state["V"].dtype), S


def _delta_grad(state, case):
    share, dt = case["Hv"] // case["Hk"], state["V"].dtype
    *given, dO = _sequences(state, case, *(state[n] for n in ("Q", "K", "V", "G", "beta", "dO")))
    given = [t.detach().requires_grad_() for t in (*given, _first_state(state, case))]
    q, k, v, g, beta, S0 = given
    if share > 1:
        q, k = q.repeat_interleave(share, 1), k.repeat_interleave(share, 1)
    O, S = _flow(q, k, v, g, beta, S0)
    *grads, dS0 = torch.autograd.grad((O, S), given, (dO, state["dSL"]))
    return tuple(_back(state, case, t, dt) for t in grads) + (dS0,)


# ---- what a pass cannot do without

def work(case):
    e, op = DTYPES[case["dtype"]][1], case["op"]
    if op in ("heads", "heads_grad"):
        values = case["M"] * (case["Hq"] + case["Hk"]) * case["d"]
        turn = case["M"] * (4 + 4 * case["rot"]) if case["rot"] else 0
        return dict(bytes=values * e * (2 if op == "heads" else 3) + turn, flops=values * (8 if op == "heads" else 16))
    B, Hk, Hv, dk, dv = (case[k] for k in ("B", "Hk", "Hv", "dk", "dv"))
    if op == "step":
        return dict(bytes=B * (Hv * dv * dk * 8 + e * (2 * Hk * dk + 2 * Hv * dv + 2 * Hv) + 4), flops=7 * B * Hv * dk * dv)
    tokens = case["tokens"] or B * case["L"]      # (packed sequences may be some fewer)
    heads, values, states = tokens * 2 * Hk * dk * e, tokens * Hv * dv * e, B * Hv * dv * dk * 4
    gates = 2 * tokens * Hv * e
    if op == "delta":
        return dict(bytes=heads + 2 * values + gates + states * (1 + case["s0"]), flops=7 * tokens * Hv * dk * dv)
    return dict(bytes=2 * heads + 3 * values + 2 * gates + states * (2 + case["s0"]), flops=18 * tokens * Hv * dk * dv)


# ---- the definition in 64 bits, token by token

def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op in ("heads", "heads_grad"):
        return _exact_heads(s, case)
    if op == "step":
        return _exact_step(s, case)
    B, L, Hk, Hv = s["offsets"].numel() - 1 if s["offsets"] is not None else case["B"], case["L"], case["Hk"], case["Hv"]
    ends = s["offsets"].tolist() if s["offsets"] is not None else None
    if ends:
        L = max(b - a for a, b in zip(ends, ends[1:]))

    def rows(t, fill=0.0):      # [L, B, Hv, ..] in 64 bits
        t = t.double()
        if ends:
            to = torch.full((B, L, *t.shape[2:]), fill, dtype=torch.float64, device="cuda")
            for b in range(B):
                to[b, :ends[b + 1] - ends[b]] = t[0, ends[b]:ends[b + 1]]
            t = to
        t = t.transpose(0, 1)
        return (t if t.shape[2] == Hv else t.repeat_interleave(Hv // Hk, 2)).contiguous()

    q, k, v = rows(s["Q"]), rows(s["K"]), rows(s["V"])
    a, beta = torch.exp(rows(s["G"])), rows(s["beta"])
    S = torch.zeros(B, Hv, case["dv"], case["dk"], dtype=torch.float64, device="cuda") if s["S0"] is None else s["S0"].double()

    def token(S, t):
        S = S * a[t, :, :, None, None]
        e = v[t] - (S * k[t, :, :, None]).sum(-1)
        return torch.addcmul(S, (beta[t, :, :, None] * e)[..., None], k[t, :, :, None])

    def out(t):      # [L, B, H, ..] -> the outputs' layout
        t = t.transpose(0, 1)
        return torch.cat([t[b, :ends[b + 1] - ends[b]] for b in range(B)])[None] if ends else t

    if op == "delta":
        O = torch.empty_like(v)
        for t in range(L):
            S = token(S, t)
            O[t] = (S * q[t, :, :, None]).sum(-1)
        return out(O), S
    dO = rows(s["dO"])
    dq, dk, dv, dg, db = (torch.zeros_like(x) for x in (q, k, v, a, beta))
    span = 64
    marks = [S]
    for t in range(L):
        S = token(S, t)
        if (t + 1) % span == 0:
            marks.append(S)
    R = s["dSL"].double()
    for m in range(-(-L // span) - 1, -1, -1):
        last = min(L, (m + 1) * span)
        seen = [marks[m]]
        for t in range(m * span, last):
            seen.append(token(seen[-1], t))
        for t in range(last - 1, m * span - 1, -1):
            before, after = seen[t - m * span], seen[t - m * span + 1]
            dq[t] = (after * dO[t][..., None]).sum(-2)
            R = torch.addcmul(R, dO[t][..., None], q[t, :, :, None])
            kept = before * a[t, :, :, None, None]
            e = v[t] - (kept * k[t, :, :, None]).sum(-1)
            Rk = (R * k[t, :, :, None]).sum(-1)
            db[t] = (e * Rk).sum(-1)
            de = beta[t, :, :, None] * Rk
            dv[t] = de
            dk[t] = beta[t, :, :, None] * (R * e[..., None]).sum(-2) - (kept * de[..., None]).sum(-2)
            R = torch.addcmul(R, -de[..., None], k[t, :, :, None])
            dg[t] = (R * kept).sum((-1, -2))
            R = R * a[t, :, :, None, None]
    shared = lambda t: out(t).unflatten(2, (Hk, Hv // Hk)).sum(3)  # noqa: E731
    return shared(dq), shared(dk), out(dv), out(dg), out(db), R


def _exact_step(s, case):
    q, k, v, g, beta = (s[n].double() for n in ("Q", "K", "V", "G", "beta"))
    S, O = s["S"].double(), torch.empty_like(v)
    for h in range(case["Hv"]):
        hk = h // (case["Hv"] // case["Hk"])
        now = S[s["slots"].long(), h] * torch.exp(g[:, h, None, None])
        now += torch.einsum("b,bv,bk->bvk", beta[:, h], v[:, h] - torch.einsum("bvk,bk->bv", now, k[:, hk]), k[:, hk])
        S[s["slots"].long(), h] = now
        O[:, h] = torch.einsum("bvk,bk->bv", now, q[:, hk])
    return O, S


def _exact_heads(s, case):
    d, rot, M = case["d"], case["rot"], case["M"]
    turn = torch.eye(d, dtype=torch.float64, device="cuda").expand(M, d, d)
    if rot and M * d * d * 8 < 2 << 30:      # the rotation as a matrix for each token
        turn = turn.clone()
        row = s["table"][s["positions"].long()].double()
        i = torch.arange(rot // 2, device="cuda")
        a, b = (2 * i, 2 * i + 1) if case["pairs"] else (i, i + rot // 2)
        turn[:, a, a] = turn[:, b, b] = row[:, :rot // 2]
        turn[:, a, b], turn[:, b, a] = -row[:, rot // 2:], row[:, rot // 2:]
        turned = lambda x: torch.bmm(x, turn.transpose(1, 2).contiguous())  # noqa: E731
        unturned = lambda x: torch.bmm(x, turn)  # noqa: E731
    elif rot:      # as products of complex numbers
        row = s["table"][s["positions"].long()].double()
        z = torch.complex(row[:, :rot // 2], row[:, rot // 2:])[:, None]

        def by(x, z):
            y = x.clone()
            a, b = (slice(0, rot, 2), slice(1, rot, 2)) if case["pairs"] else (slice(0, rot // 2), slice(rot // 2, rot))
            p = torch.complex(x[..., a], x[..., b]) * z
            y[..., a], y[..., b] = p.real, p.imag
            return y
        turned, unturned = (lambda x: by(x, z)), (lambda x: by(x, z.conj()))
    else:
        turned = unturned = lambda x: x  # noqa: E731
    mean = d if case["norm"] == "rms" else 1
    outs, sums = [], []
    for x, w, dy, scale in ((s["Q"], s["wq"], s.get("dQ"), d ** -0.5), (s["K"], s["wk"], s.get("dK"), 1.0)):
        x = x.double()
        w = torch.ones(d, dtype=torch.float64, device="cuda") if w is None else w.double()
        size = torch.sqrt((x ** 2).sum(-1, keepdim=True) / mean + EPS)
        if case["op"] == "heads":
            outs.append(turned(x / size * w) * scale)
            continue
        back = unturned(dy.double() * scale)
        # y = x w / n, dn / dx = x / (mean n): dx = w dy / n - x (sum of w dy x) / (mean n^3)
        outs.append(back * w / size - x * (back * w * x).sum(-1, keepdim=True) / (mean * size ** 3))
        if case["norm"] == "rms":
            sums.append((back * x / size).sum((0, 1)))
    return tuple(outs + sums)
