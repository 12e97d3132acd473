"""The operators of a packed linear-attention block: what is measured of them.

Three operators, each in the form that training, prompts or single tokens take:

  fwd    linear attention with a decay for each head over packed rows (linear_attention_fwd): a prompt, or
         the forward pass of training.  States in and out where `states`.
  bwd    its backward pass (linear_attention_bwd): the gradients of q, k, v, the log decays and, where
         `states`, the initial state.
  step   one token of each of `batch` sequences (linear_attention_step), the state updated in place.
  norm   the gated RMSNorm after the mixer, forward (gated_rmsnorm_fwd).
  normb  and backward (gated_rmsnorm_bwd), from what the forward saved.

The recurrence, for every head, at token t of a row (pos: its place in its own sequence):
  S_t = a_t S_{t-1} + k_t v_t^T,  a_t = exp(g_t), 0 where pos is 0;   o_t = scale S_t^T q_t.
Shapes: q, k (batch, groups, dk, seqlen); v, o (batch, heads, dv, seqlen); g (batch, heads, seqlen), or
(heads) where `fixed`; S (batch, heads, dk, dv).
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CHUNK = 64
EPS = 1e-5


def listed():
    return [
        # serving, a chat turn of odd length that continues a conversation: latency
        dict(name="prompt-turn", kind="fwd", batch=1, seqlen=77, heads=8, groups=8, dk=64, dv=64, dtype="bf16",
             fixed=False, states=True, mean=4000.0),
        # serving: two rows of prompts at the 130M width, q and k shared by all heads, an odd total length
        dict(name="prompt-130m", kind="fwd", batch=2, seqlen=3001, heads=24, groups=1, dk=128, dv=64, dtype="bf16",
             fixed=False, states=True, mean=400.0),
        # training forward at the 1.4B width (d_inner 4096), packed rows
        dict(name="fwd-1.4b", kind="fwd", batch=8, seqlen=4096, heads=64, groups=8, dk=128, dv=64, dtype="bf16",
             fixed=False, states=False, mean=646.0),
        # one long row of few sequences, decays fixed for each head
        dict(name="fwd-long-row", kind="fwd", batch=1, seqlen=65536, heads=32, groups=32, dk=64, dv=64, dtype="bf16",
             fixed=True, states=False, mean=20000.0),
        # the smallest training step (the 64-channel configuration), 32-bit, odd head sizes
        dict(name="bwd-tiny", kind="bwd", batch=1, seqlen=256, heads=2, groups=1, dk=24, dv=32, dtype="f32",
             fixed=False, states=True, mean=50.0),
        # training at the 130M width, a head's own q and k
        dict(name="bwd-130m", kind="bwd", batch=4, seqlen=2048, heads=24, groups=24, dk=64, dv=64, dtype="bf16",
             fixed=False, states=False, mean=400.0),
        # training at the 1.4B width, large heads, q and k shared by four heads, short and long sequences
        dict(name="bwd-1.4b", kind="bwd", batch=8, seqlen=4096, heads=32, groups=8, dk=128, dv=128, dtype="bf16",
             fixed=False, states=False, mean=646.0),
        # serving: one conversation's next token, where latency is all
        dict(name="step-one", kind="step", batch=1, heads=24, groups=1, dk=64, dv=64, dtype="bf16", fixed=False),
        # serving: the next tokens of 64 conversations at the 1.4B width
        dict(name="step-1.4b", kind="step", batch=64, heads=64, groups=1, dk=128, dv=64, dtype="bf16", fixed=False),
        # serving: the norm of those tokens, over the whole width
        dict(name="norm-decode", kind="norm", batch=64, seqlen=1, dim=4096, groups=1, dtype="bf16", gate_first=True),
        # training, a norm for each head, rows of odd length, 32-bit
        dict(name="norm-bwd-ragged", kind="normb", batch=2, seqlen=3001, dim=1536, groups=24, dtype="f32",
             gate_first=False),
        # training at the 1.4B width
        dict(name="norm-bwd-1.4b", kind="normb", batch=8, seqlen=4096, dim=4096, groups=8, dtype="bf16",
             gate_first=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _fitting(case):
    """No more work than the largest listed case has: shorter rows where it is."""
    while work(case)["bytes"] > 1.2e9 or case["batch"] * case["seqlen"] * case.get("heads", 1) > (1 << 20):
        case["seqlen"] //= 2
    return case


def draw(rng):
    kind = rng.choice(["fwd", "fwd", "fwd", "bwd", "bwd", "bwd", "step", "step", "norm", "normb"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind in ("norm", "normb"):
        groups = rng.choice([1, 1, 8, 24])
        dim = groups * _log(rng, 8 if groups > 1 else 64, 4096 // groups)
        batch, seqlen = _log(rng, 1, 64), rng.choice([1, _log(rng, 2, 4096)])
        return _fitting(dict(kind=kind, batch=batch, seqlen=seqlen, dim=dim, groups=groups, dtype=dtype,
                             gate_first=rng.random() < 0.5))
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
    if c["kind"] in ("norm", "normb"):
        n, r = c["batch"] * c["seqlen"] * c["dim"], c["batch"] * c["seqlen"] * c["groups"]
        if c["kind"] == "norm":
            return {"bytes": 3 * n * size + 4 * r + 4 * c["dim"], "flops": 10 * n}
        return {"bytes": 5 * n * size + 4 * r + 8 * c["dim"], "flops": 25 * n}
    tok = c["batch"] * c.get("seqlen", 1)
    qk, v = 2 * tok * c["groups"] * c["dk"] * size, tok * c["heads"] * c["dv"] * size
    g = 4 * (c["heads"] if c["fixed"] else tok * c["heads"])
    state = 4 * c["batch"] * c["heads"] * c["dk"] * c["dv"]
    mac = 2 * tok * c["heads"] * c["dk"] * c["dv"]
    if c["kind"] == "step":
        return {"bytes": qk + 2 * v + g + 2 * state, "flops": 2 * mac}
    if c["kind"] == "fwd":
        return {"bytes": qk + 2 * v + g + 4 * tok + (2 * state if c["states"] else 0), "flops": 2 * mac}
    return {"bytes": 2 * qk + 3 * v + 2 * g + 4 * tok + (3 * state if c["states"] else 0), "flops": 5 * mac}


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
    if c["kind"] in ("norm", "normb"):
        D, L = c["dim"], c["seqlen"]
        s = dict(case=c, x=randn(B, D, L), z=randn(B, D, L), w=1 + 0.1 * randn(D, dtype=torch.float32))
        if c["kind"] == "normb":
            s["dout"] = randn(B, D, L)
            s["rstd"] = _rstd(s)
        return s
    H, G, dk, dv = c["heads"], c["groups"], c["dk"], c["dv"]
    s = dict(case=c, scale=dk ** -0.5)
    state = (B, H, dk, dv)
    if c["kind"] == "step":
        s.update(q=randn(B, G, dk), k=randn(B, G, dk), v=randn(B, H, dv), g=_decay(c, (B, H), gen),
                 state=4 * randn(*state, dtype=torch.float32))
        return s
    L = c["seqlen"]
    s.update(q=randn(B, G, dk, L), k=randn(B, G, dk, L), v=randn(B, H, dv, L), g=_decay(c, (B, H, L), gen),
             pos=_positions(c, seed), h0=4 * randn(*state, dtype=torch.float32) if c["states"] else None)
    if c["kind"] == "bwd":
        s.update(dout=randn(B, H, dv, L), dfin=randn(*state, dtype=torch.float32) if c["states"] else None)
    return s


# ---------------------------------------------------------------------------------------------
# the plain forms: 32-bit products and sums over chunks of CHUNK tokens
# ---------------------------------------------------------------------------------------------

def _chunks(x, L):
    """(..., L) -> (..., chunks, CHUNK), padded with zeros."""
    n = -(-L // CHUNK)
    return torch.nn.functional.pad(x, (0, n * CHUNK - L)).unflatten(-1, (n, CHUNK))


def _mm(a, b):
    return torch.matmul(a, b.contiguous())


def _plan(s):
    """What the decays and the sequence starts make: the weights between tokens of a chunk, into and out of
    chunks, and between chunks.  Sums of log decays in 64 bits."""
    c = s["case"]
    B, H, L = c["batch"], c["heads"], c["seqlen"]
    g = (s["g"][None, :, None] if c["fixed"] else s["g"]).double().expand(B, H, L)
    start = (s["pos"] == 0)[:, None]
    g = torch.where(start, torch.zeros_like(g), g)
    cum = _chunks(torch.cumsum(g, -1), L)                                   # the row's running sum
    cum[..., -1, (L - 1) % CHUNK + 1:] = cum[..., -1, (L - 1) % CHUNK, None]
    seq = _chunks(torch.cumsum(start.to(torch.int32), -1), L)               # the sequence of each token
    seq[..., -1, (L - 1) % CHUNK + 1:] = seq[..., -1, (L - 1) % CHUNK, None]
    end, last = cum[..., -1], seq[..., -1]                                  # at each chunk's end
    before = torch.nn.functional.pad(end, (1, 0))                           # at the end of the chunk before, 0 first
    sbefore = torch.nn.functional.pad(last, (1, 0))
    tri = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device="cuda").tril()
    zero = torch.zeros((), dtype=torch.float32, device="cuda")

    def decay(d, keep):
        return torch.where(keep, torch.exp(d).float(), zero)

    m = {"within": decay(cum[..., :, None] - cum[..., None, :], (seq[..., :, None] == seq[..., None, :]) & tri),
         "in": decay(cum - before[..., :-1, None], seq == sbefore[..., :-1, None]),
         "out": decay(end[..., None] - cum, seq == last[..., None])}
    n = end.shape[-1]
    low = torch.ones(n + 1, n + 1, dtype=torch.bool, device="cuda").tril()
    # row: the state after chunk row - 1 (row 0: the initial state), column: what chunk column - 1 added
    m["between"] = decay(before[..., :, None] - before[..., None, :], (sbefore[..., :, None] == sbefore[..., None, :]) & low)
    return m


def _heads(x, c):
    return x.float().repeat_interleave(c["heads"] // c["groups"], 1)


def _states(added, first, between):
    """The state before each chunk and after the last: (..., chunks + 1, a, b)."""
    lead = torch.zeros_like(added[..., :1, :, :]) if first is None else first[..., None, :, :]
    x = torch.cat([lead, added], -3)
    return _mm(between, x.flatten(-2)).unflatten(-1, x.shape[-2:])


def _forward(s):
    c, L = s["case"], s["case"]["seqlen"]
    m = _plan(s)
    q, k, v = (_chunks(x, L).transpose(-3, -2) for x in (_heads(s["q"], c) * s["scale"], _heads(s["k"], c), s["v"].float()))
    S = _states(_mm(k * m["out"][..., None, :], v.transpose(-1, -2)), s["h0"], m["between"])
    qt = q.transpose(-1, -2)
    o = _mm(_mm(qt, k) * m["within"], v.transpose(-1, -2)) + m["in"][..., None] * _mm(qt, S[..., :-1, :, :])
    o = o.flatten(2, 3)[:, :, :L].transpose(-1, -2).to(s["v"].dtype).contiguous()
    return (o, S[..., -1, :, :].contiguous()) if c["states"] else o


def _back(x, L):
    """(batch, heads, chunks, features, CHUNK) -> (batch, heads, features, L)."""
    return x.transpose(2, 3).flatten(3)[..., :L]


def _backward(s):
    c, L = s["case"], s["case"]["seqlen"]
    m = _plan(s)
    q, k, v, do = (_chunks(x, L).transpose(-3, -2) for x in
                   (_heads(s["q"], c) * s["scale"], _heads(s["k"], c), s["v"].float(), s["dout"].float()))
    kt, vt, qt, dot = (x.transpose(-1, -2) for x in (k, v, q, do))
    S = _states(_mm(k * m["out"][..., None, :], vt), s["h0"], m["between"])
    # the gradient of the state after each chunk: the same sum over the chunks that follow
    dS = _states((_mm(q * m["in"][..., None, :], dot)).flip(-3), s["dfin"], m["between"].transpose(-1, -2).flip(-1, -2)).flip(-3)
    P, dP = _mm(qt, k) * m["within"], _mm(dot, v) * m["within"]
    dqi = _mm(S[..., :-1, :, :], do) * m["in"][..., None, :]
    dki = _mm(dS[..., 1:, :, :], v) * m["out"][..., None, :]
    dq = _mm(k, dP.transpose(-1, -2)) + dqi
    dk = _mm(q, dP) + dki
    dv = _mm(do, P) + _mm(dS[..., 1:, :, :].transpose(-1, -2), k) * m["out"][..., None, :]
    # the log decays: what passes over a token, from before it in the row to it or after it
    W = _mm(qt, k) * dP
    passing = W.sum(-1) - W.sum(-2) + (q * dqi).sum(-2) - (k * dki).sum(-2)           # per token of a chunk
    over = (S[..., 1:, :, :] * dS[..., 1:, :, :]).sum((-1, -2))                       # over each chunk's end
    pos = _chunks(s["pos"], L)[:, None]
    tail = torch.arange(pos.shape[-2] * CHUNK, device="cuda").view(pos.shape[-2], CHUNK) >= L
    pos = torch.where(tail, torch.ones_like(pos), pos)
    seq = torch.cumsum((pos == 0).int(), -1)
    same = (seq[..., :, None] == seq[..., None, :]) & torch.ones(CHUNK, CHUNK, dtype=torch.bool, device="cuda").triu()
    dg = (same * passing[..., None, :]).sum(-1) + (seq == seq[..., -1:]) * over[..., None]
    dg = torch.where(pos == 0, torch.zeros_like(dg), dg).flatten(2)[..., :L]

    def shared(x):
        return _back(x, L).unflatten(1, (c["groups"], -1)).sum(2)

    out = {"dq": (shared(dq) * s["scale"]).to(s["q"].dtype), "dk": shared(dk).to(s["k"].dtype),
           "dv": _back(dv, L).to(s["v"].dtype).contiguous(),
           "ddecay": dg.sum((0, 2), dtype=torch.float64).float() if c["fixed"] else dg}
    if c["states"]:
        out["dinitial_state"] = dS[..., 0, :, :].contiguous()
    return out


def _step(s):
    c = s["case"]
    q, k = _heads(s["q"], c) * s["scale"], _heads(s["k"], c)
    a = torch.exp(s["g"])[..., None, None]
    s["state"].mul_(a).add_(k[..., :, None] * s["v"].float()[..., None, :])
    o = (q[..., :, None] * s["state"]).sum(-2)
    return o.to(s["v"].dtype), s["state"]


def _gate(s):
    z = s["z"].float()
    return z * torch.sigmoid(z)


def _rstd(s):
    c = s["case"]
    a = s["x"].float() * _gate(s) if c["gate_first"] else s["x"].float()
    return torch.rsqrt(a.unflatten(1, (c["groups"], -1)).square().mean(2) + EPS)


def _per_channel(r, c):
    return r.repeat_interleave(c["dim"] // c["groups"], 1)


def _norm(s):
    c = s["case"]
    r = _rstd(s)
    out = s["x"].float() * _gate(s) * _per_channel(r, c) * s["w"][:, None]
    return out.to(s["x"].dtype), r


def _norm_backward(s):
    c = s["case"]
    x, z, g, w = s["x"].float(), s["z"].float(), s["dout"].float(), s["w"][:, None]
    r = _per_channel(s["rstd"], c)
    sig = torch.sigmoid(z)
    gate, dgate = z * sig, sig * (1 + z * (1 - sig))
    a = x * gate if c["gate_first"] else x                  # what is normed
    up = g * w if c["gate_first"] else g * gate * w         # the gradient of a rstd
    mean = (up * a).unflatten(1, (c["groups"], -1)).mean(2).repeat_interleave(c["dim"] // c["groups"], 1)
    da = r * (up - a * r * r * mean)
    if c["gate_first"]:
        dx, dz, dw = da * gate, da * x * dgate, g * a * r
    else:
        dx, dz, dw = da, g * w * a * r * dgate, g * gate * a * r
    t = s["x"].dtype
    return {"dx": dx.to(t), "dz": dz.to(t), "dweight": dw.sum((0, 2))}


def run(state):
    s, c = state, state["case"]
    if own:
        import paper_2408_03865_amd as P
        if c["kind"] == "fwd":
            return P.linear_attention_fwd(s["q"], s["k"], s["v"], s["g"], s["pos"], scale=s["scale"],
                                          initial_state=s["h0"], return_final=c["states"])
        if c["kind"] == "bwd":
            r = P.linear_attention_bwd(s["q"], s["k"], s["v"], s["g"], s["pos"], s["dout"], scale=s["scale"],
                                       initial_state=s["h0"], dfinal_state=s["dfin"])
            return {k: v for k, v in r.items() if v is not None}
        if c["kind"] == "step":
            return P.linear_attention_step(s["q"], s["k"], s["v"], s["g"], s["state"], scale=s["scale"]), s["state"]
        if c["kind"] == "norm":
            return P.gated_rmsnorm_fwd(s["x"], s["z"], s["w"], groups=c["groups"], eps=EPS, gate_first=c["gate_first"])
        dx, dz, dw = P.gated_rmsnorm_bwd(s["x"], s["z"], s["w"], s["rstd"], s["dout"], groups=c["groups"],
                                         gate_first=c["gate_first"])
        return {"dx": dx, "dz": dz, "dweight": dw}
    return {"fwd": _forward, "bwd": _backward, "step": _step, "norm": _norm, "normb": _norm_backward}[c["kind"]](s)


# ---------------------------------------------------------------------------------------------
# the same in 64 bits from the definitions: the recurrence, token by token
# ---------------------------------------------------------------------------------------------

def _recurrence(a, k, v, q, first, backwards=False):
    """S_t = a_t S + k_t v_t^T from `first`, out_t = S_t^T q_t, over the tokens in order or from the last;
    the last state is returned too.  k, q (B, H, m, L), v (B, H, n, L), a (B, H, L)."""
    B, H, n, L = v.shape
    S = torch.zeros((B, H, k.shape[2], n), dtype=torch.float64, device=v.device) if first is None else first.double().clone()
    # token-major, so that each step reads whole lines
    k, v, q, a = (x.permute(3, 0, 1, 2).contiguous() if x.dim() == 4 else x.permute(2, 0, 1).contiguous() for x in (k, v, q, a))
    out = torch.empty((L, B, H, n), dtype=torch.float64, device=v.device)
    for t in (range(L - 1, -1, -1) if backwards else range(L)):
        S = torch.where(a[t][..., None, None] == 0, torch.zeros_like(S), S * a[t][..., None, None])
        S += k[t][..., :, None] * v[t][..., None, :]
        out[t] = (S * q[t][..., :, None]).sum(-2)
    return out.permute(1, 2, 3, 0), S


def exact(case, seed):
    c = case
    if c["kind"] in ("fwd", "bwd") and c["seqlen"] * (1e-4 + c["batch"] * c["heads"] * c["dk"] * c["dv"] * 4e-11) * (1 if c["kind"] == "fwd" else 3) > 15:
        return None
    s = prepare(case, seed)
    if c["kind"] in ("norm", "normb"):
        x, z, w = s["x"].double(), s["z"].double(), s["w"].double()[:, None]
        G, per = c["groups"], c["dim"] // c["groups"]
        sig = 1 / (1 + torch.exp(-z))
        a = x * z * sig if c["gate_first"] else x
        if c["kind"] == "norm":
            r = 1 / torch.sqrt((a ** 2).view(c["batch"], G, per, -1).mean(2) + EPS)
            return x * z * sig * w * r[:, :, None].expand(-1, -1, per, -1).reshape(x.shape), r
        g = s["dout"].double()
        r = s["rstd"].double()[:, :, None].expand(-1, -1, per, -1).reshape(x.shape)
        up = g * w * (1 if c["gate_first"] else z * sig)
        inner = (up * a).view(c["batch"], G, per, -1).mean(2, keepdim=True).expand(-1, -1, per, -1).reshape(x.shape)
        da = r * up - r ** 3 * a * inner
        dsilu = sig + z * sig * (1 - sig)
        if c["gate_first"]:
            return {"dx": da * z * sig, "dz": da * x * dsilu, "dweight": (g * a * r).sum((0, 2))}
        return {"dx": da, "dz": g * w * x * r * dsilu, "dweight": (g * x * r * z * sig).sum((0, 2))}
    rep = c["heads"] // c["groups"]
    q, k, v = s["q"].double().repeat_interleave(rep, 1) * s["scale"], s["k"].double().repeat_interleave(rep, 1), s["v"].double()
    if c["kind"] == "step":
        S = s["state"].double() * torch.exp(s["g"].double())[..., None, None] + torch.einsum("bhk,bhv->bhkv", k, v)
        return torch.einsum("bhk,bhkv->bhv", q, S), S
    B, H, L = c["batch"], c["heads"], c["seqlen"]
    g = (s["g"][None, :, None].expand(B, H, L) if c["fixed"] else s["g"]).double()
    start = (s["pos"] == 0)[:, None].expand(B, H, L)
    a = torch.where(start, 0.0, torch.exp(g))
    if c["kind"] == "fwd":
        o, S = _recurrence(a, k, v, q, s["h0"])
        return (o, S) if c["states"] else o
    do = s["dout"].double()
    flip = None if s["h0"] is None else s["h0"].transpose(-1, -2)
    dq, fin = _recurrence(a, v, k, do, flip)                      # S^T in place of S
    after = torch.cat([a[..., 1:], torch.ones_like(a[..., :1])], -1)    # the multiplier of the token that follows
    dk, _ = _recurrence(after, do, q, v, None if s["dfin"] is None else s["dfin"].transpose(-1, -2), backwards=True)
    dv, dS = _recurrence(after, q, do, k, s["dfin"], backwards=True)
    # sum of q dq - k dk from a token to its sequence's end, and what the final state's gradient adds there
    e = (q * dq - k * dk).sum(2)
    total = torch.cumsum(e.flip(-1), -1).flip(-1)
    if s["dfin"] is not None:
        total = total + (fin * s["dfin"].double().transpose(-1, -2)).sum((-1, -2))[..., None]
    seq = torch.cumsum(start.int(), -1)
    starts_after = torch.where(start, torch.arange(L, device="cuda").expand(B, H, L), L)
    nxt = torch.cat([torch.flip(torch.cummin(torch.flip(starts_after, (-1,)), -1)[0], (-1,))[..., 1:],
                     torch.full((B, H, 1), L, device="cuda")], -1)     # where the next sequence starts
    beyond = torch.gather(torch.nn.functional.pad(total, (0, 1)), -1, nxt)
    dg = torch.where(start, 0.0, total - torch.where(seq == seq[..., -1:], torch.zeros_like(beyond), beyond))
    out = {"dq": dq.reshape(B, c["groups"], rep, *dq.shape[2:]).sum(2) * s["scale"],
           "dk": dk.reshape(B, c["groups"], rep, *dk.shape[2:]).sum(2), "dv": dv,
           "ddecay": dg.sum((0, 2)) if c["fixed"] else dg}
    if c["states"]:
        out["dinitial_state"] = dS * a[..., :1, None]
    return out
