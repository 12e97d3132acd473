"""GPU: the packed linear attention against the recurrence in 64 bits, token by token.

Tolerances, element by element, with M the same sum over the terms' absolute values and u = 2^-24:
  32-bit results   n u M.  A term passes at most dk + dv products and sums inside a chunk's product, 64 over
                   its tokens, 2 for each chunk that carries the state, the exponentials (1 u each, and
                   ln 2 |x| 2 u for an argument x; e^-|x| |x| < 0.4) and the sums over heads and tokens.
                   n = 2 (dk + dv + 64 + 2 chunks + 64), for ddecay n (terms + 512 tokens) on its own M.
  bf16 results     besides: the weighted products and the copy of the state rounded to bf16 once, 2^-8 M, the
                   state's weighted operands in 16 bits, 2^-15 M, and the result's own rounding, 2^-8 |out|.
"""
import numpy as np
import pytest

import linear_reference as R
from gpu_common import note

pytestmark = pytest.mark.gpu

U, HALF = 2.0 ** -24, 2.0 ** -8


def make(shape, dtype, kind, states, seed, mean=40, scale=None):
    import torch
    B, H, G, dk, dv, L = shape
    gen = torch.Generator().manual_seed(seed)
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    rnd = lambda *s: torch.randn(s, generator=gen)  # noqa: E731
    decay = {"token": lambda: -torch.exp(2 * rnd(B, H, L) - 3), "head": lambda: -torch.exp(rnd(H) - 3), "none": lambda: None}[kind]()
    pos = torch.from_numpy(R.positions(B, L, mean, np.random.default_rng(seed), states))
    d = dict(q=rnd(B, G, dk, L).to(t), k=rnd(B, G, dk, L).to(t), v=rnd(B, H, dv, L).to(t), decay=decay, pos=pos,
             dout=rnd(B, H, dv, L).to(t), initial=rnd(B, H, dk, dv) * 2 if states else None,
             dfinal=rnd(B, H, dk, dv) if states else None, scale=dk ** -0.5 if scale is None else scale)
    return d


def cuda(d):
    import torch
    return {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in d.items()}


def forward(g, **kw):
    import paper_2408_03865_amd as P
    return P.linear_attention_fwd(g["q"], g["k"], g["v"], g["decay"], g["pos"], scale=g["scale"],
                                  initial_state=g["initial"], return_final=True, **kw)


def backward(g, **kw):
    import paper_2408_03865_amd as P
    return P.linear_attention_bwd(g["q"], g["k"], g["v"], g["decay"], g["pos"], g["dout"], scale=g["scale"],
                                  initial_state=g["initial"], dfinal_state=g["dfinal"], **kw)


def check(got, ref, mag, shape, name, rounded):
    B, H, G, dk, dv, L = shape
    got = got.double().cpu()
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    assert bool(got.isfinite().all()), name
    n = 2 * (dk + dv + 128 + 2 * (-(-L // 64)) + H // G)
    if name == "ddecay":
        n += 2 * 512
    bound = n * U * mag + 1e-30
    if rounded:
        bound = bound + (HALF + 2.0 ** -15) * mag + HALF * ref.abs()
    over = ((got - ref).abs() / bound).max().item()
    assert over <= 1, f"{name}: error {over:.2f} of its bound"
    return over, ((got - ref).norm() / ref.norm().clamp(min=1e-300)).item()


# rows of one token, of a chunk, around a chunk's end, split and whole, odd head sizes, shared heads
SHAPES = [(1, 1, 1, 1, 1, 1), (2, 3, 3, 16, 16, 1), (1, 2, 1, 24, 32, 63), (2, 4, 2, 64, 64, 64), (1, 4, 4, 33, 47, 65),
          (3, 2, 1, 128, 64, 130), (1, 3, 3, 64, 128, 257), (1, 6, 2, 128, 128, 300), (2, 5, 1, 7, 100, 515),
          (1, 2, 2, 65, 127, 1101), (1, 3, 1, 128, 64, 523),
          (24, 11, 11, 16, 16, 150)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind,states", [("token", True), ("head", False), ("none", True)])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_linear_forward(shape, kind, states, dtype):
    d = make(shape, dtype, kind, states, 11 + sum(shape))
    note(f"linear attention forward {shape} {kind} states={states} {dtype}")
    ref, mag = (R.reference(d["q"], d["k"], d["v"], d["decay"], d["pos"], d["scale"], d["initial"], absolute=m) for m in (False, True))
    out, fin = forward(cuda(d))
    assert out.dtype == d["q"].dtype
    w = check(out, ref["out"], mag["out"], shape, "out", dtype == "bf16")
    note(f"  out {w[0]:.2g} of its bound, {w[1]:.2g} off")
    w = check(fin, ref["final_state"], mag["final_state"], shape, "final_state", False)
    note(f"  final_state {w[0]:.2g} of its bound, {w[1]:.2g} off")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind,states", [("token", True), ("head", False), ("none", True), ("token", False)])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_linear_backward(shape, kind, states, dtype):
    d = make(shape, dtype, kind, states, 12 + sum(shape))
    note(f"linear attention backward {shape} {kind} states={states} {dtype}")
    args = (d["q"], d["k"], d["v"], d["decay"], d["pos"], d["scale"], d["initial"], d["dout"], d["dfinal"])
    ref, mag = (R.reference(*args, absolute=m) for m in (False, True))
    got = backward(cuda(d))
    assert (got["ddecay"] is None) == (kind == "none") and (got["dinitial_state"] is None) == (not states)
    for name in ("dq", "dk", "dv", "ddecay", "dinitial_state"):
        if got[name] is not None:
            w = check(got[name], ref[name], mag[name], shape, name, dtype == "bf16" and name in ("dq", "dk", "dv"))
            note(f"  {name} {w[0]:.2g} of its bound, {w[1]:.2g} off")
            # the 512 summed parts and the two states' product are off by some u of their size each, at random:
            # sqrt(512) 4 u = 5e-6 of it, and they are a few times what is left of them
            assert name != "ddecay" or w[1] <= 2e-5
