"""GPU: one token of linear attention for each sequence, the state updated in place, against 64 bits.

With u = 2^-24 and M the sums over the terms' absolute values: the state is off by 4 u M (the exponential,
1 u and its argument's rounding, a product and a fused sum), out by (dk + 4) u M besides the state's and,
in bf16, its rounding, 2^-8 |out|."""
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
    decay = {"token": lambda: -torch.exp(rnd(B, H) - 2), "head": lambda: -torch.exp(rnd(H) - 2), "none": lambda: None}[kind]()
    return dict(q=rnd(B, G, dk).to(t), k=rnd(B, G, dk).to(t), v=rnd(B, H, dv).to(t), decay=decay, state=rnd(B, H, dk, dv) * 3)


def reference(d, pos, scale, absolute=False):
    import torch
    f = (lambda x: x.double().abs()) if absolute else (lambda x: x.double())
    H, G = d["v"].shape[1], d["q"].shape[1]
    q, k = (f(d[n]).repeat_interleave(H // G, 1) for n in "qk")
    B = q.shape[0]
    g = torch.zeros(B, H, dtype=torch.float64) if d["decay"] is None else d["decay"].double().expand(B, H)
    cut = (g <= R.CUT) if pos is None else (pos == 0)[:, None] | (g <= R.CUT)
    a = torch.where(cut, torch.zeros_like(g), torch.exp(g))
    S = f(d["state"])
    new = torch.where(a[..., None, None] == 0, torch.zeros_like(S), a[..., None, None] * S) + k[..., None] * f(d["v"])[..., None, :]
    if pos is not None:
        new = torch.where((pos < 0)[:, None, None, None], S, new)
    out = (q[..., None] * new).sum(-2) * (abs(scale) if absolute else scale)
    if pos is not None:
        out = torch.where((pos < 0)[:, None, None], torch.zeros_like(out), out)
    return out, new


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["token", "head", "none"])
@pytest.mark.parametrize("shape", [(1, 1, 1, 1, 1), (3, 4, 2, 24, 32), (2, 3, 1, 128, 128), (5, 6, 6, 65, 7), (2, 3, 3, 100, 126),
                                   (64, 8, 1, 64, 64), (70, 4, 4, 128, 128), (300, 2, 1, 17, 33), (40, 8, 2, 128, 100)],
                         ids=lambda s: "x".join(map(str, s)))
def test_linear_step(shape, kind, dtype):
    import torch
    import paper_2408_03865_amd as P
    B = shape[0]
    d = make(*shape, dtype, kind, sum(shape))
    note(f"linear attention step {shape} {kind} {dtype}")
    for pos in (None, torch.from_numpy(np.random.default_rng(B).integers(-1, 3, B).astype(np.int32))):
        ref, mag = reference(d, pos, 0.3), reference(d, pos, 0.3, absolute=True)
        g = {n: None if t is None else t.cuda() for n, t in d.items()}
        out = P.linear_attention_step(g["q"], g["k"], g["v"], g["decay"], g["state"], None if pos is None else pos.cuda(), scale=0.3)
        n = 4 * U
        assert bool(((g["state"].double().cpu() - ref[1]).abs() <= n * mag[1] + 1e-30).all())
        bound = (shape[3] + 8) * U * mag[0] + (HALF * ref[0].abs() if dtype == "bf16" else 0) + 1e-30
        assert bool(((out.double().cpu() - ref[0]).abs() <= bound).all())
        if pos is not None:
            idle = pos < 0
            assert torch.equal(g["state"].cpu()[idle], d["state"][idle])


def test_steps_continue_a_prompt():
    """A prompt through the chunks, then token by token: every state and output as the whole row through the
    chunks gives them (32-bit: twice the forward's bound)."""
    import torch
    import paper_2408_03865_amd as P
    B, H, G, dk, dv, L, n = 3, 4, 2, 48, 64, 140, 9
    gen = torch.Generator().manual_seed(5)
    q, k, v = (torch.randn(s, generator=gen).cuda() for s in ((B, G, dk, L), (B, G, dk, L), (B, H, dv, L)))
    decay = -torch.exp(torch.randn((B, H, L), generator=gen) - 2).cuda()
    pos = torch.from_numpy(R.positions(B, L, 60, np.random.default_rng(3))).cuda()
    out, fin = P.linear_attention_fwd(q, k, v, decay, pos, return_final=True)
    cut = lambda t: t[..., :L - n].contiguous()  # noqa: E731
    _, state = P.linear_attention_fwd(cut(q), cut(k), cut(v), cut(decay), cut(pos), return_final=True)
    ref = R.reference(*(t.cpu() for t in (q, k, v, decay, pos)), 1.0, absolute=True)
    bound = 2 * 2 * (dk + dv + 128 + 6 + 2) * U
    for t in range(L - n, L):
        one = lambda x: x[..., t].contiguous()  # noqa: E731
        o = P.linear_attention_step(one(q), one(k), one(v), one(decay), state, pos[:, t].contiguous())
        assert bool(((o - out[..., t]).cpu().double().abs() <= bound * ref["out"][..., t]).all()), t
    assert bool(((state - fin).cpu().double().abs() <= bound * ref["final_state"]).all())
