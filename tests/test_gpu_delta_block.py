"""GPU: the operators of a packed delta-rule block run together, as a training step (layer norm, projection, conv, the
norm of queries and keys, delta rule, gated norm, and back with a residual) and as generation (a prompt, then token by
token, called and replayed from a graph), in 32 bits against the same composition in 64 bits on the CPU, differentiated
by torch."""
import numpy as np
import pytest

import linear_reference as R
from gpu_common import note

pytestmark = pytest.mark.gpu

B, H, G, DK, DV, L, W, M = 2, 4, 2, 24, 32, 150, 4, 40
D, QK = H * DV, G * DK
F = D + 2 * QK
SCALE = DK ** -0.5
# nine operators in 32 bits, each within some hundred u of its terms; the norms divide by what may be small, and the
# delta rule's state holds what up to forty tokens left of their errors
TOLERANCE = 4000 * 2.0 ** -24


def parameters():
    import torch
    gen = torch.Generator().manual_seed(78)
    r = lambda *s: torch.randn(s, generator=gen)  # noqa: E731
    return dict(x=r(B, M, L), ln_w=1 + 0.1 * r(M), ln_b=0.1 * r(M), proj=r(F, M) * M ** -0.5, w=0.5 * r(F, W), bias=0.1 * r(F),
                beta=torch.rand((B, H, L), generator=gen), decay=-torch.exp(r(B, H, L) - 2), z=r(B, D, L), norm=1 + 0.1 * r(D),
                dout=r(B, D, L), dres=r(B, M, L), pos=torch.from_numpy(R.positions(B, L, 40, np.random.default_rng(9))))


def split(u):
    return u[:, :QK].contiguous(), u[:, QK:2 * QK].contiguous(), u[:, 2 * QK:].reshape(B, H, DV, -1).contiguous()


def reference(p):
    """The block in 64 bits, differentiable: out and the gradients of sum(dout out) + sum(dres x)."""
    import torch
    leaf = {n: p[n].double().requires_grad_() for n in ("x", "ln_w", "ln_b", "proj", "w", "bias", "beta", "decay", "z", "norm")}
    pos = p["pos"].long()
    x = leaf["x"]
    c = x - x.mean(1, keepdim=True)
    h = c * torch.rsqrt(c.square().mean(1, keepdim=True) + 1e-5) * leaf["ln_w"][:, None] + leaf["ln_b"][:, None]
    h = leaf["proj"] @ h
    taps = []
    for k in range(W):                                       # weight[:, W-1-k] times the token k back, of the same sequence
        back = torch.nn.functional.pad(h, (k, 0))[..., :L]
        taps.append(torch.where((pos >= k)[:, None], back, torch.zeros_like(back)) * leaf["w"][:, W - 1 - k, None])
    q, k, v = split(torch.nn.functional.silu(sum(taps) + leaf["bias"][:, None]))
    unit = lambda t: (t * torch.rsqrt(t.square().sum(2, keepdim=True) + 1e-6)).repeat_interleave(H // G, 1)  # noqa: E731
    q, k = unit(q.reshape(B, G, DK, L)), unit(k.reshape(B, G, DK, L))
    a = torch.where((pos == 0)[:, None], torch.zeros_like(leaf["decay"]), torch.exp(leaf["decay"]))
    S, outs = torch.zeros(B, H, DK, DV, dtype=torch.float64), []
    for t in range(L):
        S = a[:, :, t, None, None] * S
        u = leaf["beta"][:, :, t, None] * (v[..., t] - (S * k[..., t, None]).sum(-2))
        S = S + k[..., t, None] * u[..., None, :]
        outs.append((S * q[..., t, None]).sum(-2) * SCALE)
    g = torch.stack(outs, -1).reshape(B, D, L) * torch.nn.functional.silu(leaf["z"])
    n = g.reshape(B, H, DV, L)
    y = (n * torch.rsqrt(n.square().mean(2, keepdim=True) + 1e-5)).reshape(B, D, L) * leaf["norm"][:, None]
    ((y * p["dout"].double()).sum() + (x * p["dres"].double()).sum()).backward()
    return y.detach(), {n: t.grad for n, t in leaf.items()}


def test_training_step():
    import torch
    import paper_2408_03865_amd as P
    p = parameters()
    y, grads = reference(p)
    c = {n: t.cuda() for n, t in p.items()}
    h, mean, rstd = P.layernorm_fwd(c["x"], c["ln_w"], c["ln_b"])
    u = (c["proj"] @ h).contiguous()
    s = P.causal_conv1d_fwd(u, c["w"], c["bias"], c["pos"])
    q0, k0, v = split(s)
    q, qn = P.head_l2norm_fwd(q0, groups=G)
    k, kn = P.head_l2norm_fwd(k0, groups=G)
    q, k = q.reshape(B, G, DK, L), k.reshape(B, G, DK, L)
    o = P.delta_rule_fwd(q, k, v, c["beta"], c["decay"], c["pos"], scale=SCALE).reshape(B, D, L)
    got, gr = P.gated_rmsnorm_fwd(o, c["z"], c["norm"], groups=H)

    do, dz, dn = P.gated_rmsnorm_bwd(o, c["z"], c["norm"], gr, c["dout"], groups=H)
    a = P.delta_rule_bwd(q, k, v, c["beta"], c["decay"], c["pos"], do.reshape(B, H, DV, L), scale=SCALE)
    dq = P.head_l2norm_bwd(q0, qn, a["dq"].reshape(B, QK, L), groups=G)
    dk = P.head_l2norm_bwd(k0, kn, a["dk"].reshape(B, QK, L), groups=G)
    du, dw, db = P.causal_conv1d_bwd(u, c["w"], c["bias"], c["pos"], torch.cat([dq, dk, a["dv"].reshape(B, D, L)], 1))
    dproj = sum(du[b] @ h[b].t().contiguous() for b in range(B))
    dh = (c["proj"].t().contiguous() @ du).contiguous()
    dx, dlw, dlb = P.layernorm_bwd(c["x"], c["ln_w"], mean, rstd, dh, dresidual=c["dres"])
    for name, g, r in [("out", got, y), ("z", dz, grads["z"]), ("norm", dn, grads["norm"]), ("beta", a["dbeta"], grads["beta"]),
                       ("decay", a["ddecay"], grads["decay"]), ("w", dw, grads["w"]), ("bias", db, grads["bias"]),
                       ("proj", dproj, grads["proj"]), ("ln_w", dlw, grads["ln_w"]), ("ln_b", dlb, grads["ln_b"]), ("x", dx, grads["x"])]:
        rel = ((g.double().cpu() - r).norm() / r.norm()).item()
        note(f"block {name}: {rel:.2g} off")
        assert rel <= TOLERANCE, name


def prompt(P, c, n):
    """The first n tokens of the rows: the states that they leave."""
    t = {k: (v[..., :n].contiguous() if k in ("x", "beta", "decay", "pos") else v) for k, v in c.items()}
    h, _, _ = P.layernorm_fwd(t["x"], t["ln_w"], t["ln_b"])
    s, conv = P.causal_conv1d_fwd((c["proj"] @ h).contiguous(), c["w"], c["bias"], t["pos"], return_final=True)
    q, k, v = split(s)
    q, k = (P.head_l2norm_fwd(x, groups=G)[0].reshape(B, G, DK, n) for x in (q, k))
    return P.delta_rule_fwd(q, k, v, t["beta"], t["decay"], t["pos"], scale=SCALE, return_final=True)[1], conv


def token(P, c, t, state, conv):
    """One token of each row: its out and the conv's state."""
    h, _, _ = P.layernorm_fwd(t["x"], c["ln_w"], c["ln_b"])
    s, conv = P.causal_conv1d_fwd((c["proj"] @ h).contiguous(), c["w"], c["bias"], t["pos"], initial_x=conv, return_final=True)
    q, k, v = split(s)
    q, k = (P.head_l2norm_fwd(x, groups=G)[0].reshape(B, G, DK) for x in (q, k))
    o = P.delta_rule_step(q, k, v[..., 0].contiguous(), t["beta"][..., 0].contiguous(), t["decay"][..., 0].contiguous(), state,
                          t["pos"][:, 0].contiguous(), scale=SCALE)
    return P.gated_rmsnorm_fwd(o.reshape(B, D, 1), t["z"], c["norm"], groups=H)[0], conv


def at(c, t):
    return {k: c[k][..., t:t + 1].contiguous() for k in ("x", "beta", "decay", "pos", "z")}


def test_generation():
    """A prompt, then token by token from the states it left: every output as the whole row's."""
    import torch
    import paper_2408_03865_amd as P
    p, n = parameters(), 20
    p["pos"] = (torch.arange(L, dtype=torch.int32) % 100).expand(B, L).contiguous()
    y, _ = reference(p)
    c = {k: t.cuda() for k, t in p.items()}
    state, conv = prompt(P, c, L - n)
    for t in range(L - n, L):
        got, conv = token(P, c, at(c, t), state, conv)
        r = y[..., t:t + 1]
        assert ((got.double().cpu() - r).norm() / r.norm()).item() <= TOLERANCE, t


def test_generation_replayed():
    """A token's norms and its step in a graph, replayed over other inputs in the same buffers, with eager work and
    synchronizations between: every out and state as the eager calls give it, to the bit.  A second graph of the same
    buffers runs in between."""
    import torch
    import paper_2408_03865_amd as P
    gen = torch.Generator().manual_seed(5)
    r = lambda *s: torch.randn(s, generator=gen).cuda()  # noqa: E731
    x, beta, decay, z = r(B, F, 1), torch.rand((B, H), generator=gen).cuda(), -torch.exp(r(B, H)), r(B, D, 1)
    pos, ln_w, norm = torch.zeros(B, dtype=torch.int32).cuda(), 1 + 0.1 * r(F), 1 + 0.1 * r(D)
    state = torch.zeros(B, H, DK, DV).cuda()

    def one(state):
        h, _, _ = P.layernorm_fwd(x, ln_w)
        q, k, v = split(h)
        q, k = (P.head_l2norm_fwd(t, groups=G)[0].reshape(B, G, DK) for t in (q, k))
        o = P.delta_rule_step(q, k, v[..., 0].contiguous(), beta, decay, state, pos, scale=SCALE)
        return P.gated_rmsnorm_fwd(o.reshape(B, D, 1), z, norm, groups=H)[0]

    one(state.clone())
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(one(state))
        graphs.append(g)
    eager = torch.zeros_like(state)
    state.zero_()
    for t in range(6):
        for dst, src in ((x, r(B, F, 1)), (beta, torch.rand((B, H), generator=gen).cuda()), (decay, -torch.exp(r(B, H))), (z, r(B, D, 1)),
                         (pos, torch.tensor([t, (t + 1) % 3], dtype=torch.int32).cuda())):
            dst.copy_(src)
        want = one(eager)
        torch.cuda.synchronize()
        graphs[t % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[t % 2], want) and torch.equal(state, eager), t


def test_another_stream():
    """The training calls on a stream of their own, with a workspace of the caller's: to the bit what the default stream
    gives."""
    import torch
    import paper_2408_03865_amd as P
    c = {n: t.cuda() for n, t in parameters().items()}
    g = torch.Generator().manual_seed(6)
    q, k = (torch.nn.functional.normalize(torch.randn(B, G, DK, L, generator=g), dim=2).cuda() for _ in range(2))
    v, do = (torch.randn(B, H, DV, L, generator=g).cuda() for _ in range(2))

    def run(**ws):
        o = P.delta_rule_fwd(q, k, v, c["beta"], c["decay"], c["pos"], scale=SCALE, **ws)
        a = P.delta_rule_bwd(q, k, v, c["beta"], c["decay"], c["pos"], do, scale=SCALE, **ws)
        n, m, s = P.layernorm_fwd(c["x"], c["ln_w"], c["ln_b"])
        return [o, n, m, s, *P.layernorm_bwd(c["x"], c["ln_w"], m, s, n, **ws), *(t for t in a.values() if t is not None)]

    want = run()
    need = max(P.load().packmamba_delta_rule_bwd_workspace_size(B, H, G, DK, DV, L, 0),
               P.load().packmamba_layernorm_bwd_workspace_size(B, M, L, 0))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        got = run(workspace=ws)
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want, strict=True))
