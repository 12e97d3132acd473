"""GPU: one token of the gated delta rule for each sequence, the state updated in place, against 64 bits.

With u = 2^-24 and M the sums over the terms' absolute values: S' is off by 3 u M (the exponential, 1 u and its argument's
rounding, a product), its product with k by dk u more, u_t by 3 u; the state by (dk + 16) u M with M = |S'| + |k| beta
(|v| + |S'|^T |k|), out by (2 dk + 16) u |q| M and, in bf16, its rounding, 2^-8 |out|."""
import numpy as np
import pytest

import linear_reference as R
from gpu_common import note

pytestmark = pytest.mark.gpu

U, HALF = 2.0 ** -24, 2.0 ** -8


def make(B, H, G, dk, dv, dtype, kind, seed):
    import torch
    gen = torch.Generator().manual_seed(seed)
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    rnd = lambda *s: torch.randn(s, generator=gen)  # noqa: E731
    unit = lambda *s: (lambda x: x / x.norm(dim=-1, keepdim=True).clamp(min=1e-3))(rnd(*s))  # noqa: E731
    decay = {"token": lambda: -torch.exp(rnd(B, H) - 2), "head": lambda: -torch.exp(rnd(H) - 2), "none": lambda: None}[kind]()
    return dict(q=unit(B, G, dk).to(t), k=unit(B, G, dk).to(t), v=rnd(B, H, dv).to(t), beta=torch.sigmoid(rnd(B, H)), decay=decay,
                state=rnd(B, H, dk, dv) * 3)


def reference(d, pos, scale):
    """(out, state) and what bounds their errors."""
    import torch
    H, G = d["v"].shape[1], d["q"].shape[1]
    q, k = (d[n].double().repeat_interleave(H // G, 1) for n in "qk")
    B, dk = q.shape[0], q.shape[2]
    v, beta, S = d["v"].double(), d["beta"].double(), d["state"].double()
    g = torch.zeros(B, H, dtype=torch.float64) if d["decay"] is None else d["decay"].double().expand(B, H)
    cut = (g <= R.CUT) if pos is None else (pos == 0)[:, None] | (g <= R.CUT)
    a = torch.where(cut, torch.zeros_like(g), torch.exp(g))
    found = torch.where(a[..., None, None] == 0, torch.zeros_like(S), a[..., None, None] * S)
    u = beta[..., None] * (v - (found * k[..., None]).sum(-2))
    new = found + k[..., None] * u[..., None, :]
    um = beta[..., None] * (v.abs() + (found.abs() * k.abs()[..., None]).sum(-2))
    mag = found.abs() + k.abs()[..., None] * um[..., None, :]
    out = (q[..., None] * new).sum(-2) * scale
    om = abs(scale) * (q.abs()[..., None] * found.abs()).sum(-2) + abs(scale) * (q.abs() * k.abs()).sum(-1, keepdim=True) * um
    if pos is not None:
        idle = (pos < 0)[:, None, None]
        new = torch.where(idle[..., None], S, new)
        out = torch.where(idle, torch.zeros_like(out), out)
    return out, new, (2 * dk + 16) * U * om + 1e-30, (dk + 16) * U * mag + 1e-30


SHAPES = [(1, 1, 1, 1, 1), (3, 4, 2, 24, 32), (2, 3, 1, 128, 128), (5, 6, 6, 65, 7), (2, 3, 3, 100, 126),
          (64, 8, 1, 64, 64), (70, 4, 4, 128, 128), (300, 2, 1, 17, 33), (40, 8, 2, 128, 100)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["token", "head", "none"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_delta_step(shape, kind, dtype):
    import torch
    import paper_2408_03865_amd as P
    B = shape[0]
    d = make(*shape, dtype, kind, sum(shape))
    note(f"delta rule step {shape} {kind} {dtype}")
    for pos in (None, torch.from_numpy(np.random.default_rng(B).integers(-1, 3, B).astype(np.int32))):
        out_ref, state_ref, out_tol, state_tol = reference(d, pos, 0.3)
        g = {n: None if t is None else t.cuda() for n, t in d.items()}
        out = P.delta_rule_step(g["q"], g["k"], g["v"], g["beta"], g["decay"], g["state"], None if pos is None else pos.cuda(), scale=0.3)
        assert out.dtype == d["q"].dtype
        assert bool(((g["state"].double().cpu() - state_ref).abs() <= state_tol).all())
        assert bool(((out.double().cpu() - out_ref).abs() <= out_tol + (HALF * out_ref.abs() if dtype == "bf16" else 0)).all())
        if pos is not None:
            idle = pos < 0
            assert torch.equal(g["state"].cpu()[idle], d["state"][idle]) and not bool(out.cpu()[idle].any())


def test_step_nonfinite():
    """A start takes nothing of its state, a sequence nothing of another's."""
    import torch
    import paper_2408_03865_amd as P
    d = make(4, 2, 2, 40, 36, "f32", "token", 9)
    d["state"][0] = float("nan")
    d["state"][1, 0, 3, 5] = float("inf")
    d["v"][2, 1, 7] = float("nan")
    pos = torch.tensor([0, 5, 0, 3], dtype=torch.int32)
    clean = {n: t.clone() for n, t in d.items()}
    clean["state"][0], clean["state"][1, 0, 3, 5], clean["v"][2, 1, 7] = 0, 0, 0
    got = []
    for e in (d, clean):
        g = {n: t.cuda() for n, t in e.items()}
        out = P.delta_rule_step(g["q"], g["k"], g["v"], g["beta"], g["decay"], g["state"], pos.cuda())
        got.append((out.cpu(), g["state"].cpu()))
    keep = torch.ones(4, 2, 36, dtype=torch.bool)
    keep[1, 0, 5] = keep[2, 1, 7] = False
    assert torch.equal(got[0][0][keep], got[1][0][keep]) and not bool(got[0][0][~keep].isfinite().any())
    keep = keep[:, :, None].expand(4, 2, 40, 36)
    assert torch.equal(got[0][1][keep], got[1][1][keep])


def test_steps_continue_a_prompt():
    """A prompt through the chunks, then token by token: every output, and the last state, as the whole row through the
    chunks gives them (32-bit: both within the forward's bound of the reference)."""
    import torch
    import paper_2408_03865_amd as P
    import test_gpu_delta as T
    shape = B, H, G, dk, dv, L = 3, 4, 2, 48, 64, 140
    n = 9
    d = T.make(shape, "f32", "token", False, 5, mean=60)
    ref, mag = T.reference(d, back=False)
    g = T.cuda(d)
    cut = {k: v[..., :L - n].contiguous() if isinstance(v, torch.Tensor) and v.shape[-1] == L else v for k, v in g.items()}
    out, state = T.forward(cut)
    outs = [out]
    for t in range(L - n, L):
        one = lambda x: x[..., t].contiguous()  # noqa: E731
        outs.append(P.delta_rule_step(one(g["q"]), one(g["k"]), one(g["v"]), one(g["beta"]), one(g["decay"]), state,
                                      g["pos"][:, t].contiguous(), scale=d["scale"])[..., None])
    T.check(torch.cat(outs, -1), ref["out"], mag["out"], shape, "out", False)
    T.check(state, ref["final_state"], mag["final_state"], shape, "final_state", False)
