"""GPU: the packed gated delta rule against the rule in 64 bits, token by token.

Tolerances, element by element, with M the budgets of delta_reference and u = 2^-24:
  32-bit results   n u M.  A term passes at most dk + dv products and sums inside a chunk's products, 64 over its tokens
                   twice (P or the update, and H, whose own entries pass as many), 2 for each chunk that carries the state,
                   the exponentials (1 u each, and ln 2 |x| 2 u for an argument x; e^-|x| |x| < 0.4) and the sums over
                   heads; n = 4 (dk + dv + 256 + 2 chunks + heads / groups), for ddecay 1024 more for the sums over tokens.
  bf16 results     besides: P or a pair's weight, u or dv and the copy of the state rounded to bf16 once each, 3 2^-8 M, and
                   the result's own rounding, 2^-8 |out|.
The budgets are sums of norms, far above most elements, so results of 1000 elements and more are held in the 2-norm as well:
roundings to bf16 (four at most, each of at most 2^-8 and spread over it evenly: 2^-8 / sqrt 3 of the norm) 2 2^-8 / sqrt 3,
32-bit ones 2e-5.  That is a mean over elements: a single one can be the small difference of two rounded terms (0.13 of
2.4, with one token and one feature), where the element's bound alone says something.  So is ddecay where decays are strong: it is
what sums of out . dout and v . dv leave, of the size of a token's multiplier; at e^-7 of those sums their 1e-6 is 1e-3 of it.
"""
import numpy as np
import pytest

import delta_reference as DR
import linear_reference as R
from gpu_common import note

pytestmark = pytest.mark.gpu

U, HALF = 2.0 ** -24, 2.0 ** -8
NAMES = ("dq", "dk", "dv", "dbeta", "ddecay", "dinitial_state")


def make(shape, dtype, kind, states, seed, mean=40, scale=None):
    import torch
    B, H, G, dk, dv, L = shape
    gen = torch.Generator().manual_seed(seed)
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    rnd = lambda *s: torch.randn(s, generator=gen)  # noqa: E731
    unit = lambda *s: (lambda x: x / x.norm(dim=2, keepdim=True).clamp(min=1e-3) * 0.99)(rnd(*s))  # noqa: E731
    decay = {"token": lambda: -torch.exp(2 * rnd(B, H, L) - 3), "head": lambda: -torch.exp(rnd(H) - 3), "none": lambda: None}[kind]()
    pos = torch.from_numpy(R.positions(B, L, mean, np.random.default_rng(seed), states))
    return dict(q=unit(B, G, dk, L).to(t), k=unit(B, G, dk, L).to(t), v=rnd(B, H, dv, L).to(t), beta=torch.sigmoid(2 * rnd(B, H, L)),
                decay=decay, pos=pos, dout=rnd(B, H, dv, L).to(t), initial=rnd(B, H, dk, dv) * 0.5 if states else None,
                dfinal=rnd(B, H, dk, dv) if states else None, scale=dk ** -0.5 if scale is None else scale)


def cuda(d):
    import torch
    return {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in d.items()}


def forward(g, **kw):
    import paper_2408_03865_amd as P
    kw.setdefault("return_final", True)
    return P.delta_rule_fwd(g["q"], g["k"], g["v"], g["beta"], g["decay"], g["pos"], scale=g["scale"],
                            initial_state=g["initial"], **kw)


def backward(g, **kw):
    import paper_2408_03865_amd as P
    return P.delta_rule_bwd(g["q"], g["k"], g["v"], g["beta"], g["decay"], g["pos"], g["dout"], scale=g["scale"],
                            initial_state=g["initial"], dfinal_state=g["dfinal"], **kw)


def reference(d, back=True):
    return DR.reference(d["q"], d["k"], d["v"], d["beta"], d["decay"], d["pos"], d["scale"], d["initial"],
                        d["dout"] if back else None, d["dfinal"] if back else None)


def bound_of(ref, mag, shape, name, rounded):
    B, H, G, dk, dv, L = shape
    n = 4 * (dk + dv + 256 + 2 * (-(-L // 64)) + H // G) + (1024 if name == "ddecay" else 0)
    bound = n * U * mag + 1e-30
    return bound + 3 * HALF * mag + HALF * ref.abs() if rounded else bound


def check(got, ref, mag, shape, name, rounded, norm=1.0):
    got = got.double().cpu()
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    assert bool(got.isfinite().all()), name
    over = ((got - ref).abs() / bound_of(ref, mag, shape, name, rounded)).max().item()
    rel = ((got - ref).norm() / ref.norm().clamp(min=1e-300)).item()
    note(f"  {name} {over:.2g} of its bound, {rel:.2g} off")
    assert over <= 1, f"{name}: error {over:.2f} of its bound"
    if norm and ref.numel() >= 1000 and ref.norm() > 0:
        assert rel <= norm * (2 * HALF / 3 ** 0.5 if rounded else 2e-5), f"{name}: {rel:.2g} off"


def rounded_name(name, dtype):
    return dtype == "bf16" and name in ("out", "dq", "dk", "dv")


# rows of one token, of a chunk, around a chunk's end, split and whole, odd head sizes, shared heads
SHAPES = [(1, 1, 1, 1, 1, 1), (2, 3, 3, 16, 16, 1), (1, 2, 1, 24, 32, 63), (2, 4, 2, 64, 64, 64), (1, 4, 4, 33, 47, 65),
          (3, 2, 1, 128, 64, 130), (1, 3, 3, 64, 128, 257), (1, 6, 2, 128, 128, 300), (2, 5, 1, 7, 100, 515),
          (1, 2, 2, 65, 127, 1101), (1, 3, 1, 128, 64, 1023), (24, 11, 11, 16, 16, 150)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind,states", [("token", True), ("head", False), ("none", True)])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_delta_forward(shape, kind, states, dtype):
    d = make(shape, dtype, kind, states, 11 + sum(shape))
    note(f"delta rule forward {shape} {kind} states={states} {dtype}")
    ref, mag = reference(d, back=False)
    g = cuda(d)
    out, fin = forward(g)
    assert out.dtype == d["q"].dtype
    check(out, ref["out"], mag["out"], shape, "out", dtype == "bf16")
    check(fin, ref["final_state"], mag["final_state"], shape, "final_state", False)
    check(forward(g, return_final=False), ref["out"], mag["out"], shape, "out", dtype == "bf16")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind,states", [("token", True), ("head", False), ("none", True), ("token", False)])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_delta_backward(shape, kind, states, dtype):
    d = make(shape, dtype, kind, states, 12 + sum(shape))
    note(f"delta rule backward {shape} {kind} states={states} {dtype}")
    ref, mag = reference(d)
    got = backward(cuda(d))
    assert (got["ddecay"] is None) == (kind == "none") and (got["dinitial_state"] is None) == (not states)
    for name in NAMES:
        if got[name] is not None:
            check(got[name], ref[name], mag[name], shape, name, rounded_name(name, dtype))
