"""The operators of a packed delta-rule block: what is measured of them.

  fwd    the gated delta rule over packed rows (delta_rule_fwd): a prompt, or the forward pass of training.
         States in and out where `states`.
  bwd    its backward pass (delta_rule_bwd): the gradients of q, k, v, the writing strengths, the log decays and,
         where `states`, the initial state.
  step   one token of each of `batch` sequences (delta_rule_step), the state updated in place.
  l2     each head's features divided by their length, as the rule wants its keys (head_l2norm_fwd).
  l2b    and backward (head_l2norm_bwd), from what the forward saved.
  ln     the layer norm before a mixer (layernorm_fwd).
  lnb    and backward (layernorm_bwd), with the residual's gradient where `residual`.

The rule, for every head, at token t of a row (pos: its place in its own sequence):
  S' = a_t S_{t-1},  a_t = exp(g_t), 0 where pos is 0
  S_t = S' + k_t u_t^T,  u_t = beta_t (v_t - S'^T k_t);   o_t = scale S_t^T q_t.
Shapes: q, k (batch, groups, dk, seqlen); v, o (batch, heads, dv, seqlen); beta (batch, heads, seqlen); g the same,
or (heads) where `fixed`; S (batch, heads, dk, dv).  The norms' activations are (batch, dim, seqlen).
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CHUNK = 64
L2_EPS, LN_EPS = 1e-6, 1e-5


def listed():
    return [
        # serving, a chat turn of odd length that continues a conversation: latency
        dict(name="prompt-turn", kind="fwd", batch=1, seqlen=77, heads=8, groups=8, dk=64, dv=64, dtype="bf16",
             fixed=False, states=True, mean=4000.0),
        # serving: one long document at the 130M width, q and k shared by three heads, an odd length
        dict(name="prompt-long", kind="fwd", batch=1, seqlen=30001, heads=24, groups=8, dk=128, dv=64, dtype="bf16",
             fixed=False, states=True, mean=20000.0),
        # training forward at the 1.4B width (d_inner 4096), packed rows
        dict(name="fwd-1.4b", kind="fwd", batch=8, seqlen=4096, heads=32, groups=16, dk=128, dv=128, dtype="bf16",
             fixed=False, states=False, mean=646.0),
        # the smallest training step (the 64-channel configuration), 32-bit, odd head sizes
        dict(name="bwd-tiny", kind="bwd", batch=1, seqlen=256, heads=2, groups=1, dk=24, dv=32, dtype="f32",
             fixed=True, states=True, mean=50.0),
        # training at the 130M width, a head's own q and k
        dict(name="bwd-130m", kind="bwd", batch=4, seqlen=2048, heads=24, groups=24, dk=64, dv=64, dtype="bf16",
             fixed=False, states=False, mean=400.0),
        # training at the 1.4B width, large heads, q and k shared by two heads, short and long sequences
        dict(name="bwd-1.4b", kind="bwd", batch=8, seqlen=4096, heads=32, groups=16, dk=128, dv=128, dtype="bf16",
             fixed=False, states=False, mean=646.0),
        # serving: one conversation's next token, where latency is all
        dict(name="step-one", kind="step", batch=1, heads=24, groups=8, dk=64, dv=64, dtype="bf16", fixed=False),
        # serving: the next tokens of 64 conversations at the 1.4B width
        dict(name="step-1.4b", kind="step", batch=64, heads=32, groups=16, dk=128, dv=128, dtype="bf16", fixed=False),
        # a prompt's keys at the 130M width, rows of odd length, 32-bit
        dict(name="l2-prompt", kind="l2", batch=2, seqlen=3001, dim=1536, groups=24, dtype="f32"),
        # training at the 1.4B width: the keys of 16 heads
        dict(name="l2-bwd-1.4b", kind="l2b", batch=8, seqlen=4096, dim=2048, groups=16, dtype="bf16"),
        # serving: the norm of 64 conversations' next tokens
        dict(name="ln-decode", kind="ln", batch=64, seqlen=1, dim=2048, dtype="bf16", residual=False),
        # training at the 1.4B width (d_model 2048), with the residual's gradient
        dict(name="ln-bwd-1.4b", kind="lnb", batch=8, seqlen=4096, dim=2048, dtype="bf16", residual=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _fitting(case):
    """No more work than the largest listed case has: shorter rows where it is."""
    while work(case)["bytes"] > 1.2e9 or case["batch"] * case["seqlen"] * case.get("heads", 1) > (1 << 20):
        case["seqlen"] //= 2
    return case


def draw(rng):
    kind = rng.choice(["fwd", "fwd", "fwd", "bwd", "bwd", "bwd", "step", "step", "l2", "l2b", "ln", "lnb"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    batch, seqlen = _log(rng, 1, 64), rng.choice([1, _log(rng, 2, 4096), _log(rng, 2, 4096)])
    if kind in ("l2", "l2b"):
        groups = _log(rng, 1, 64)
        return _fitting(dict(kind=kind, batch=batch, seqlen=seqlen, groups=groups, dtype=dtype,
                             dim=groups * rng.choice([32, 64, 128, _log(rng, 8, 256)])))
    if kind in ("ln", "lnb"):
        return _fitting(dict(kind=kind, batch=batch, seqlen=seqlen, dim=_log(rng, 64, 8192), dtype=dtype,
                             residual=rng.random() < 0.5))
    heads = _log(rng, 1, 64)
    groups = rng.choice([1, heads, max(g for g in range(1, heads + 1) if heads % g == 0 and g * g <= heads)])
    # head sizes: mostly those that models have, sometimes any
    dk, dv = (rng.choice([32, 64, 64, 128, 128, _log(rng, 8, 128)]) for _ in range(2))
    case = dict(kind=kind, batch=_log(rng, 1, 64 if kind == "step" else 8), heads=heads, groups=groups, dk=dk, dv=dv,
                dtype=dtype, fixed=rng.random() < 0.3)
    if kind == "step":
        return case
    mean = math.exp(rng.uniform(math.log(8), math.log(4096)))
    return _fitting(dict(case, seqlen=_log(rng, 1, 16384), states=rng.random() < 0.5, mean=mean))


def work(case):
    c = case
    size = 4 if c["dtype"] == "f32" else 2
    tok = c["batch"] * c.get("seqlen", 1)
    if c["kind"] in ("l2", "l2b", "ln", "lnb"):
        n = tok * c["dim"]
        if c["kind"] == "l2":
            return {"bytes": 2 * n * size + 4 * tok * c["groups"], "flops": 3 * n}
        if c["kind"] == "l2b":
            return {"bytes": 3 * n * size + 4 * tok * c["groups"], "flops": 6 * n}
        if c["kind"] == "ln":
            return {"bytes": 2 * n * size + 8 * tok + 8 * c["dim"], "flops": 8 * n}
        return {"bytes": (4 if c["residual"] else 3) * n * size + 8 * tok + 12 * c["dim"], "flops": 16 * n}
    qk, v = 2 * tok * c["groups"] * c["dk"] * size, tok * c["heads"] * c["dv"] * size
    b = 4 * tok * c["heads"]
    g = 4 * c["heads"] if c["fixed"] else b
    state = 4 * c["batch"] * c["heads"] * c["dk"] * c["dv"]
    mac = 2 * tok * c["heads"] * c["dk"] * c["dv"]
    if c["kind"] == "step":
        return {"bytes": qk + 2 * v + b + g + 2 * state, "flops": 3 * mac}
    if c["kind"] == "fwd":
        return {"bytes": qk + 2 * v + b + g + 4 * tok + (2 * state if c["states"] else 0), "flops": 3 * mac}
    # the errors and states again (2), the gradient of the state (2), of the errors (1), q (1) and k (2)
    return {"bytes": 2 * qk + 3 * v + 2 * (b + g) + 4 * tok + (3 * state if c["states"] else 0), "flops": 8 * mac}


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------

def _positions(case, seed):
    """Packed rows of sequences with lengths around `mean`; with `states` a row's first sequence
    continues another row's."""
    rng = np.random.default_rng(seed)
    B, L = case["batch"], case["seqlen"]
    pos = np.empty((B, L), np.int32)
    for b in range(B):
        t, first = 0, case["states"]
        while t < L:
            n = min(L - t, max(1, int(round(rng.lognormal(math.log(case["mean"]) - 0.5, 1.0)))))
            pos[b, t:t + n] = np.arange(n) + (int(rng.integers(1, 1000)) if first else 0)
            t, first = t + n, False
    return torch.from_numpy(pos).cuda()


def _decay(case, shape, gen):
    """Log decays: fixed for a head (memories from 32 tokens to thousands), or -dt A with dt in [1e-3, 1e-1]
    and A in [1, 16], as a discretised state space has them."""
    H = case["heads"]
    if case["fixed"]:
        return torch.log1p(-torch.exp2(-5 - 7 * torch.arange(H, device="cuda", dtype=torch.float32) / H))
    dt = torch.exp(torch.rand(shape, generator=gen, device="cuda") * math.log(100.0) + math.log(1e-3))
    A = 1 + 15 * torch.rand(H, generator=gen, device="cuda")
    return -dt * (A if len(shape) == 2 else A[:, None])


def prepare(case, seed):
    c, t = case, DTYPES[case["dtype"]]
    gen = torch.Generator(device="cuda").manual_seed(int(seed))

    def randn(*shape, dtype=t):
        return torch.randn(shape, generator=gen, device="cuda").to(dtype)

    B = c["batch"]
    if c["kind"] in ("l2", "l2b", "ln", "lnb"):
        D, L = c["dim"], c["seqlen"]
        s = dict(case=c)
        if c["kind"] in ("l2", "l2b"):
            s["x"] = randn(B, D, L)
            if c["kind"] == "l2b":
                s.update(dout=randn(B, D, L), rnorm=_rnorm(s))
            return s
        # a residual stream: every token its own size, and features that are off from 0 alike
        s["x"] = ((1 + torch.rand((B, 1, L), generator=gen, device="cuda")) *
                  (randn(B, D, L, dtype=torch.float32) + 0.5 * randn(D, 1, dtype=torch.float32) + 0.3)).to(t)
        s.update(w=1 + 0.1 * randn(D, dtype=torch.float32), b=0.1 * randn(D, dtype=torch.float32))
        if c["kind"] == "lnb":
            s["mean"], s["rstd"] = _moments(s)
            s.update(dout=randn(B, D, L), dres=randn(B, D, L) if c["residual"] else None)
        return s
    H, G, dk, dv = c["heads"], c["groups"], c["dk"], c["dv"]
    s = dict(case=c, scale=dk ** -0.5)
    state = (B, H, dk, dv)

    def unit(*shape):
        x = randn(*shape, dtype=torch.float32)
        return (x / x.square().sum(2, keepdim=True).add(L2_EPS).sqrt()).to(t)

    if c["kind"] == "step":
        s.update(q=unit(B, G, dk), k=unit(B, G, dk), v=randn(B, H, dv), beta=torch.sigmoid(randn(B, H, dtype=torch.float32)),
                 g=_decay(c, (B, H), gen), state=0.5 * randn(*state, dtype=torch.float32))
        return s
    L = c["seqlen"]
    s.update(q=unit(B, G, dk, L), k=unit(B, G, dk, L), v=randn(B, H, dv, L),
             beta=torch.sigmoid(randn(B, H, L, dtype=torch.float32)), g=_decay(c, (B, H, L), gen),
             pos=_positions(c, seed), h0=0.5 * randn(*state, dtype=torch.float32) if c["states"] else None)
    if c["kind"] == "bwd":
        s.update(dout=randn(B, H, dv, L), dfin=randn(*state, dtype=torch.float32) if c["states"] else None)
    return s


# ---------------------------------------------------------------------------------------------
# the plain forms: 32-bit products and sums, the rule over chunks of CHUNK tokens
# ---------------------------------------------------------------------------------------------

def _chunks(x, L):
    """(..., L) -> (..., chunks, CHUNK), padded with zeros."""
    n = -(-L // CHUNK)
    return torch.nn.functional.pad(x, (0, n * CHUNK - L)).unflatten(-1, (n, CHUNK))


def _tokens(x, L):
    """(batch, heads, features, L) -> (batch, heads, chunks, CHUNK, features)."""
    return _chunks(x, L).permute(0, 1, 3, 4, 2).contiguous()


def _back(x, L):
    """(batch, heads, chunks, CHUNK, features) -> (batch, heads, features, L)."""
    return x.flatten(2, 3)[:, :, :L].transpose(-1, -2)


def _mm(a, b):
    return torch.matmul(a, b.contiguous())


def _T(x):
    return x.transpose(-1, -2)


def _inverse(A):
    """(I + A)^-1 of strictly lower triangular A, blocks of one row joined to ones of two, four and so on."""
    X = torch.eye(CHUNK, device=A.device, dtype=A.dtype).expand(A.shape).clone()
    for n in (1, 2, 4, 8, 16, 32):
        blocks = [x.unflatten(-2, (-1, 2 * n)).unflatten(-1, (-1, 2 * n)).diagonal(dim1=-4, dim2=-2).movedim(-1, -3) for x in (A, X)]
        a, x = blocks[0][..., n:, :n], blocks[1]
        low = -_mm(_mm(x[..., n:, n:], a), x[..., :n, :n])
        X.unflatten(-2, (-1, 2 * n)).unflatten(-1, (-1, 2 * n)).diagonal(dim1=-4, dim2=-2)[..., n:, :n, :].copy_(low.movedim(-3, -1))
    return X


def _plan(s):
    """What the decays, the strengths and the sequence starts make: the weights between tokens of a chunk, into and out of
    chunks, and over them.  Sums of log decays in 64 bits."""
    c = s["case"]
    B, H, L = c["batch"], c["heads"], c["seqlen"]
    g = (s["g"][None, :, None] if c["fixed"] else s["g"]).double().expand(B, H, L)
    start = (s["pos"] == 0)[:, None]
    g = _chunks(torch.where(start, torch.zeros_like(g), g), L)
    cum = torch.cumsum(g, -1)                                               # since the chunk's start
    seq = torch.cumsum(_chunks(start.to(torch.int32), L), -1)               # the starts among those
    tri = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device="cuda").tril()
    zero = torch.zeros((), dtype=torch.float32, device="cuda")

    def decay(d, keep):
        return torch.where(keep, torch.exp(d).float(), zero)

    end, last = cum[..., -1], seq[..., -1]
    return {"within": decay(cum[..., :, None] - cum[..., None, :], (seq[..., :, None] == seq[..., None, :]) & tri),
            "in": decay(cum, seq == 0)[..., None], "out": decay(end[..., None] - cum, seq == last[..., None])[..., None],
            "over": decay(end, last == 0)[..., None, None], "seq": seq, "beta": _chunks(s["beta"], L)[..., None]}


def _heads(x, c):
    return x.float().repeat_interleave(c["heads"] // c["groups"], 1)


def _walk(s):
    """The chunks in order: the plan, q (scaled), k, v, the inverses, the states before the chunks and after the last, and u."""
    c, L = s["case"], s["case"]["seqlen"]
    m = _plan(s)
    q, k, v = (_tokens(x, L) for x in (_heads(s["q"], c) * s["scale"], _heads(s["k"], c), s["v"].float()))
    X = _inverse((m["beta"] * m["within"] * _mm(k, _T(k))).tril(-1))
    u0, W, ko = _mm(X, m["beta"] * v), _mm(X, m["beta"] * m["in"] * k), _T(m["out"] * k).contiguous()
    S = s["h0"] if c["states"] else torch.zeros((c["batch"], c["heads"], c["dk"], c["dv"]), device="cuda")
    states, us = [S], []
    for i in range(u0.shape[2]):
        us.append(u0[:, :, i] - _mm(W[:, :, i], S))
        S = m["over"][:, :, i] * S + _mm(ko[:, :, i], us[-1])
        states.append(S)
    return m, q, k, v, X, torch.stack(states, 2), torch.stack(us, 2)


def _out(m, q, k, S, u):
    return m["in"] * _mm(q, S[:, :, :-1]) + _mm(_mm(q, _T(k)) * m["within"], u)


def _forward(s):
    m, q, k, _, _, S, u = _walk(s)
    o = _back(_out(m, q, k, S, u), s["case"]["seqlen"]).to(s["v"].dtype).contiguous()
    return (o, S[:, :, -1].contiguous()) if s["case"]["states"] else o


def _backward(s):
    c, L = s["case"], s["case"]["seqlen"]
    m, q, k, v, X, S, u = _walk(s)
    beta, within = m["beta"], m["within"]
    do, XT, qT = _tokens(s["dout"].float(), L), _T(X).contiguous(), _T(q)
    P = _mm(q, _T(k)) * within
    # the gradient of v / beta: X^T of what reaches u, from the outs of the chunk and from the state after it
    r0, Y = _mm(XT, _mm(_T(P), do)), _mm(XT, m["out"] * k)
    D0, kb = _mm(_T(m["in"] * q).contiguous(), do), _T(beta * m["in"] * k).contiguous()
    D = s["dfin"] if c["states"] else torch.zeros_like(S[:, :, 0])
    grads, rs = [D], []
    for i in range(u.shape[2] - 1, -1, -1):
        rs.append(r0[:, :, i] + _mm(Y[:, :, i], D))
        D = m["over"][:, :, i] * D + D0[:, :, i] - _mm(kb[:, :, i], rs[-1])
        grads.append(D)
    D, dr = torch.stack(grads[::-1], 2), torch.stack(rs[::-1], 2)            # D[i]: before chunk i, [i + 1] after it
    S0, ST, DT = S[:, :, :-1], _T(S[:, :, :-1]), _T(D[:, :, 1:])
    dv = beta * dr
    kk, dA = _mm(k, _T(k)) * within, -_mm(dr, _T(u)).tril(-1)
    dP, dK = _mm(do, _T(u)) * within, beta * dA * within
    dq = _mm(dP, k) + m["in"] * _mm(do, ST)
    dk = _mm(_T(dP), q) + _mm(dK, k) + _mm(_T(dK), k) - m["in"] * _mm(dv, ST) + m["out"] * _mm(u, DT)
    dbeta = (dr * (v - m["in"] * _mm(k, S0))).sum(-1) + (dA * kk).sum(-1)
    # the log decays: each passes on what the tokens after it take and what the chunk's last state does
    passing = (_out(m, q, k, S, u) * do).sum(-1) - (v * dv).sum(-1)
    seq, up = m["seq"], torch.ones(CHUNK, CHUNK, dtype=torch.bool, device="cuda").triu()
    over = (S[:, :, 1:] * D[:, :, 1:]).sum((-1, -2))[..., None]
    dg = (((seq[..., :, None] == seq[..., None, :]) & up) * passing[..., None, :]).sum(-1) + (seq == seq[..., -1:]) * over
    dg = torch.where((s["pos"] == 0)[:, None], torch.zeros((), device="cuda"), dg.flatten(2)[..., :L])

    def shared(x):
        return _back(x, L).unflatten(1, (c["groups"], -1)).sum(2)

    out = {"dq": (shared(dq) * s["scale"]).to(s["q"].dtype).contiguous(), "dk": shared(dk).to(s["k"].dtype).contiguous(),
           "dv": _back(dv, L).to(s["v"].dtype).contiguous(), "dbeta": dbeta.flatten(2)[..., :L].contiguous(),
           "ddecay": dg.sum((0, 2), dtype=torch.float64).float() if c["fixed"] else dg.contiguous()}
    if c["states"]:
        out["dinitial_state"] = D[:, :, 0].contiguous()
    return out


def _step(s):
    c = s["case"]
    q, k = _heads(s["q"], c) * s["scale"], _heads(s["k"], c)
    S = s["state"].mul_(torch.exp(s["g"])[..., None, None])
    u = s["beta"][..., None] * (s["v"].float() - (k[..., :, None] * S).sum(-2))
    S.add_(k[..., :, None] * u[..., None, :])
    return (q[..., :, None] * S).sum(-2).to(s["v"].dtype), S


def _rnorm(s):
    return torch.rsqrt(s["x"].float().unflatten(1, (s["case"]["groups"], -1)).square().sum(2) + L2_EPS)


def _l2(s):
    r = _rnorm(s)
    return (s["x"].float().unflatten(1, (s["case"]["groups"], -1)) * r[:, :, None]).flatten(1, 2).to(s["x"].dtype), r


def _l2_backward(s):
    x, g = (s[n].float().unflatten(1, (s["case"]["groups"], -1)) for n in ("x", "dout"))
    r = s["rnorm"][:, :, None]
    return (r * (g - x * r * r * (x * g).sum(2, keepdim=True))).flatten(1, 2).to(s["x"].dtype)


def _moments(s):
    x = s["x"].float()
    mean = x.mean(1)
    return mean, torch.rsqrt((x - mean[:, None]).square().mean(1) + LN_EPS)


def _ln(s):
    mean, r = _moments(s)
    return ((s["x"].float() - mean[:, None]) * r[:, None] * s["w"][:, None] + s["b"][:, None]).to(s["x"].dtype), mean, r


def _ln_backward(s):
    r, g = s["rstd"][:, None], s["dout"].float()
    h = (s["x"].float() - s["mean"][:, None]) * r
    up = g * s["w"][:, None]
    dx = r * (up - up.mean(1, keepdim=True) - h * (up * h).mean(1, keepdim=True))
    if s["dres"] is not None:
        dx = dx + s["dres"].float()
    return {"dx": dx.to(s["x"].dtype), "dweight": (g * h).sum((0, 2)), "dbias": g.sum((0, 2))}


def _own(s, c):
    import paper_2408_03865_amd as P
    if c["kind"] == "fwd":
        return P.delta_rule_fwd(s["q"], s["k"], s["v"], s["beta"], s["g"], s["pos"], scale=s["scale"],
                                initial_state=s["h0"], return_final=c["states"])
    if c["kind"] == "bwd":
        r = P.delta_rule_bwd(s["q"], s["k"], s["v"], s["beta"], s["g"], s["pos"], s["dout"], scale=s["scale"],
                             initial_state=s["h0"], dfinal_state=s["dfin"])
        return {k: v for k, v in r.items() if v is not None}
    if c["kind"] == "step":
        return P.delta_rule_step(s["q"], s["k"], s["v"], s["beta"], s["g"], s["state"], scale=s["scale"]), s["state"]
    if c["kind"] == "l2":
        return P.head_l2norm_fwd(s["x"], groups=c["groups"], eps=L2_EPS)
    if c["kind"] == "l2b":
        return P.head_l2norm_bwd(s["x"], s["rnorm"], s["dout"], groups=c["groups"])
    if c["kind"] == "ln":
        return P.layernorm_fwd(s["x"], s["w"], s["b"], eps=LN_EPS)
    dx, dw, db = P.layernorm_bwd(s["x"], s["w"], s["mean"], s["rstd"], s["dout"], dresidual=s["dres"])
    return {"dx": dx, "dweight": dw, "dbias": db}


def run(state):
    s, c = state, state["case"]
    if own:
        return _own(s, c)
    return {"fwd": _forward, "bwd": _backward, "step": _step, "l2": _l2, "l2b": _l2_backward, "ln": _ln,
            "lnb": _ln_backward}[c["kind"]](s)


# ---------------------------------------------------------------------------------------------
# the same in 64 bits from the definitions: the rule, token by token
# ---------------------------------------------------------------------------------------------

def _exact_norm(c, s):
    x = s["x"].double()
    if c["kind"] in ("l2", "l2b"):
        x = x.view(c["batch"], c["groups"], -1, c["seqlen"])
        if c["kind"] == "l2":
            r = 1 / torch.sqrt((x ** 2).sum(2) + L2_EPS)
            return (x * r[:, :, None]).view(s["x"].shape), r
        g, r = s["dout"].double().view(x.shape), s["rnorm"].double()[:, :, None]
        return (g * r - x * r ** 3 * (x * g).sum(2, keepdim=True)).view(s["x"].shape)
    w = s["w"].double()[:, None]
    if c["kind"] == "ln":
        mean = x.sum(1) / c["dim"]
        r = 1 / torch.sqrt(((x - mean[:, None]) ** 2).sum(1) / c["dim"] + LN_EPS)
        return (x - mean[:, None]) * r[:, None] * w + s["b"].double()[:, None], mean, r
    r, g = s["rstd"].double()[:, None], s["dout"].double()
    h = (x - s["mean"].double()[:, None]) * r
    dx = r * (g * w - (g * w).sum(1, keepdim=True) / c["dim"] - h * (g * w * h).sum(1, keepdim=True) / c["dim"])
    if s["dres"] is not None:
        dx += s["dres"].double()
    return {"dx": dx, "dweight": (g * h).sum((0, 2)), "dbias": g.sum((0, 2))}


def _token(S, a, k, v, beta):
    """One token: the state that it finds (decayed; nothing at a start), its error, and the state after it."""
    found = torch.where(a[..., None, None] == 0, 0.0, S * a[..., None, None])
    e = v - (found * k[..., :, None]).sum(-2)
    return found, e, found + k[..., :, None] * (beta[..., None] * e)[..., None, :]


def exact(case, seed):
    c = case
    if c["kind"] in ("fwd", "bwd"):
        size = c["batch"] * c["heads"] * c["dk"] * c["dv"]
        if c["seqlen"] * (2e-4 + size * 3e-11) * (1 if c["kind"] == "fwd" else 4) > 15:
            return None
    s = prepare(case, seed)
    if c["kind"] in ("l2", "l2b", "ln", "lnb"):
        return _exact_norm(c, s)
    rep = c["heads"] // c["groups"]
    q, k, v, beta = s["q"].double().repeat_interleave(rep, 1), s["k"].double().repeat_interleave(rep, 1), s["v"].double(), s["beta"].double()
    if c["kind"] == "step":
        _, _, S = _token(s["state"].double(), torch.exp(s["g"].double()).expand(beta.shape), k, v, beta)
        return s["scale"] * (S * q[..., :, None]).sum(-2), S
    B, H, L = c["batch"], c["heads"], c["seqlen"]
    g = (s["g"][None, :, None] if c["fixed"] else s["g"]).double().expand(B, H, L)
    a = torch.where((s["pos"] == 0)[:, None], 0.0, torch.exp(g))
    # token-major, so that each step reads whole lines
    q, k, v = (x.permute(3, 0, 1, 2).contiguous() for x in (q, k, v))
    a, beta = (x.permute(2, 0, 1).contiguous() for x in (a, beta))
    S = torch.zeros((B, H, c["dk"], c["dv"]), dtype=torch.float64, device="cuda") if s["h0"] is None else s["h0"].double()
    out, kept = torch.empty_like(v), []
    for t in range(L):
        if t % CHUNK == 0 and c["kind"] == "bwd":
            kept.append(S)
        _, _, S = _token(S, a[t], k[t], v[t], beta[t])
        if c["kind"] == "fwd":
            out[t] = s["scale"] * (S * q[t][..., :, None]).sum(-2)
    if c["kind"] == "fwd":
        out = out.permute(1, 2, 3, 0)
        return (out, S) if c["states"] else out
    do = s["dout"].double().permute(3, 0, 1, 2).contiguous()
    D = torch.zeros_like(S) if s["dfin"] is None else s["dfin"].double()
    dq, dk, dv, dbeta, dg = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v), torch.empty_like(beta), torch.empty_like(a)
    for n in reversed(range(len(kept))):
        first, S, tokens = n * CHUNK, kept.pop(), []
        for t in range(first, min(first + CHUNK, L)):
            found, e, S = _token(S, a[t], k[t], v[t], beta[t])
            tokens.append((found, e, S))
        for t in reversed(range(first, min(first + CHUNK, L))):
            found, e, S = tokens.pop()
            dq[t] = s["scale"] * (S * do[t][..., None, :]).sum(-1)
            D = D + s["scale"] * q[t][..., :, None] * do[t][..., None, :]
            u, du = beta[t][..., None] * e, (D * k[t][..., :, None]).sum(-2)
            dbeta[t], dv[t] = (du * e).sum(-1), beta[t][..., None] * du
            F = D - k[t][..., :, None] * dv[t][..., None, :]            # the gradient of the state that the token finds
            dk[t] = (D * u[..., None, :]).sum(-1) - (found * dv[t][..., None, :]).sum(-1)
            dg[t] = (F * found).sum((-1, -2))
            D = torch.where(a[t][..., None, None] == 0, 0.0, a[t][..., None, None] * F)
    dq, dk, dv = (x.permute(1, 2, 3, 0) for x in (dq, dk, dv))
    dg = dg.permute(1, 2, 0)
    r = {"dq": dq.unflatten(1, (c["groups"], rep)).sum(2), "dk": dk.unflatten(1, (c["groups"], rep)).sum(2), "dv": dv,
         "dbeta": dbeta.permute(1, 2, 0), "ddecay": dg.sum((0, 2)) if c["fixed"] else dg}
    if c["states"]:
        r["dinitial_state"] = D
    return r
