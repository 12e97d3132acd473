"""GPU: the operators of a packed linear-attention block run together, as a training step (conv, linear attention,
gated norm, and back) and as generation (a prompt, then token by token), in 32 bits against the same composition
in 64 bits on the CPU, differentiated by torch."""
import numpy as np
import pytest

import linear_reference as R
from gpu_common import note

pytestmark = pytest.mark.gpu

B, H, G, DK, DV, L, W = 2, 4, 2, 24, 32, 150, 4
D = H * DV


def parameters():
    import torch
    gen = torch.Generator().manual_seed(77)
    r = lambda *s: torch.randn(s, generator=gen)  # noqa: E731
    return dict(x=r(B, D + 2 * G * DK, L), z=r(B, D, L), decay=-torch.exp(r(B, H, L) - 2), w=0.5 * r(D + 2 * G * DK, W),
                bias=0.1 * r(D + 2 * G * DK), norm=1 + 0.1 * r(D), dout=r(B, D, L),
                pos=torch.from_numpy(R.positions(B, L, 40, np.random.default_rng(8))))


def split(u):
    return (u[:, :G * DK].reshape(B, G, DK, -1).contiguous(), u[:, G * DK:2 * G * DK].reshape(B, G, DK, -1).contiguous(),
            u[:, 2 * G * DK:].reshape(B, H, DV, -1).contiguous())


def reference(p, scale):
    """The block in 64 bits, differentiable: out and the gradients of sum(dout out)."""
    import torch
    leaf = {n: p[n].double().requires_grad_() for n in ("x", "z", "decay", "w", "bias", "norm")}
    pos = p["pos"].long()
    taps = []
    for k in range(W):                                       # weight[:, W-1-k] times the token k back, of the same sequence
        back = torch.nn.functional.pad(leaf["x"], (k, 0))[..., :L]
        taps.append(torch.where((pos >= k)[:, None], back, torch.zeros_like(back)) * leaf["w"][:, W - 1 - k, None])
    u = torch.nn.functional.silu(sum(taps) + leaf["bias"][:, None])
    q, k, v = (t.repeat_interleave(H // G, 1) if i < 2 else t for i, t in enumerate(split(u)))
    a = torch.where((pos == 0)[:, None], torch.zeros_like(leaf["decay"]), torch.exp(leaf["decay"]))
    S, outs = torch.zeros(B, H, DK, DV, dtype=torch.float64), []
    for t in range(L):
        S = a[:, :, t, None, None] * S + k[..., t, None] * v[..., None, :, t]
        outs.append((S * q[..., t, None]).sum(-2) * scale)
    o = torch.stack(outs, -1).reshape(B, D, L)
    g = o * torch.nn.functional.silu(leaf["z"])
    n = g.reshape(B, H, DV, L)
    y = (n * torch.rsqrt(n.square().mean(2, keepdim=True) + 1e-5)).reshape(B, D, L) * leaf["norm"][:, None]
    (y * p["dout"].double()).sum().backward()
    return y.detach(), {n: t.grad for n, t in leaf.items()}


def test_training_step():
    import torch
    import paper_2408_03865_amd as P
    p, scale = parameters(), DK ** -0.5
    y, grads = reference(p, scale)
    c = {n: t.cuda() for n, t in p.items()}
    u = P.causal_conv1d_fwd(c["x"], c["w"], c["bias"], c["pos"])
    q, k, v = split(u)
    o = P.linear_attention_fwd(q, k, v, c["decay"], c["pos"], scale=scale).reshape(B, D, L)
    got, rstd = P.gated_rmsnorm_fwd(o, c["z"], c["norm"], groups=H)
    do, dz, dn = P.gated_rmsnorm_bwd(o, c["z"], c["norm"], rstd, c["dout"], groups=H)
    a = P.linear_attention_bwd(q, k, v, c["decay"], c["pos"], do.reshape(B, H, DV, L), scale=scale)
    du = torch.cat([a["dq"].reshape(B, G * DK, L), a["dk"].reshape(B, G * DK, L), a["dv"].reshape(B, D, L)], 1)
    dx, dw, db = P.causal_conv1d_bwd(c["x"], c["w"], c["bias"], c["pos"], du)
    # six operators, each within some hundred u of its terms; the norm divides by what may be small
    for name, g, r in [("out", got, y), ("z", dz, grads["z"]), ("norm", dn, grads["norm"]), ("decay", a["ddecay"], grads["decay"]),
                       ("x", dx, grads["x"]), ("w", dw, grads["w"]), ("bias", db, grads["bias"])]:
        g = g.double().cpu()
        rel = ((g - r).norm() / r.norm()).item()
        note(f"block {name}: {rel:.2g} off")
        assert rel <= 2000 * 2.0 ** -24, name


def test_generation():
    """A prompt, then token by token from the states it left: every output as the whole row's."""
    import torch
    import paper_2408_03865_amd as P
    p, scale, n = parameters(), DK ** -0.5, 20
    p["pos"] = (torch.arange(L, dtype=torch.int32) % 100).expand(B, L).contiguous()
    y, _ = reference(p, scale)
    c = {k: t.cuda() for k, t in p.items()}

    def tokens(s):
        return {k: (t[..., s].contiguous() if k in ("x", "z", "decay", "pos") else t) for k, t in c.items()}

    head = tokens(slice(0, L - n))
    u, conv = P.causal_conv1d_fwd(head["x"], c["w"], c["bias"], head["pos"], return_final=True)
    _, state = P.linear_attention_fwd(*split(u), head["decay"], head["pos"], scale=scale, return_final=True)
    for t in range(L - n, L):
        one = tokens(slice(t, t + 1))
        u, conv = P.causal_conv1d_fwd(one["x"], c["w"], c["bias"], one["pos"], initial_x=conv, return_final=True)
        q, k, v = (s[..., 0].contiguous() for s in split(u))
        o = P.linear_attention_step(q, k, v, one["decay"][..., 0].contiguous(), state, one["pos"][:, 0].contiguous(), scale=scale)
        got, _ = P.gated_rmsnorm_fwd(o.reshape(B, D, 1), one["z"], c["norm"], groups=H)
        r = y[..., t:t + 1]
        assert ((got.double().cpu() - r).norm() / r.norm()).item() <= 2000 * 2.0 ** -24, t
