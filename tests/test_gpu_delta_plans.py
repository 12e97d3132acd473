"""GPU: the gated delta rule in calls large enough that a block takes several heads of a group and the decays' boundaries lie two and
four chunks apart in fp32, against the rule in 64 bits.  Small heads keep the reference cheap.  What the rules of delta_api.cpp give:
heads a block of the preparation and of the gradients of q and k, chunks between boundaries.  Bounds as in test_gpu_delta; results
in bf16 are held to one rounding, 2^-8 / sqrt 3 in the 2-norm."""
import numpy as np
import pytest

import linear_reference as R
from gpu_common import note
from test_gpu_delta import NAMES, backward, bound_of, check, cuda, forward, make, reference, rounded_name

pytestmark = pytest.mark.gpu

# (batch, heads, groups, dk, dv, tokens), starts              preparation, gradients, fp32's boundaries
SHAPES = [((4, 40, 8, 8, 12, 320), 0),                      # 1, 3 of 5 (two parts), 1
          ((9, 40, 8, 8, 12, 257), 128),                    # 2 of 5 (three parts), 5, 2
          ((16, 40, 8, 8, 12, 127), 0),                     # 1, 5, 2
          ((16, 40, 8, 8, 12, 128), 64),                    # 1, 5, 2
          ((16, 40, 8, 8, 12, 129), 128),                   # 2, 5, 2
          ((26, 40, 8, 5, 9, 255), 192),                    # 3 of 5 (two parts), 5, 4
          ((26, 40, 8, 5, 9, 256), 128),                    # 3 of 5 (two parts), 5, 4
          ((26, 40, 8, 5, 9, 257), 256),                    # 5, 5, 4
          ((16, 40, 8, 8, 12, 513), 256),                   # 5, 5, 4
          ((8, 44, 4, 70, 66, 400), 256)]                   # 2 of 11 (six parts), 11, 2: both halves of large heads


def packed(shape, dtype, kind, states, starts_at, seed):
    """Sequences of all lengths; with starts_at rows of odd index have starts at every multiple of it and nowhere else."""
    import torch
    d = make(shape, dtype, kind, states, seed, mean=90)
    if starts_at:
        for b in range(1, shape[0], 2):
            d["pos"][b] = torch.arange(shape[-1], dtype=torch.int32) % starts_at
            if states and b % 4 == 1:
                d["pos"][b, :starts_at] += 3                # the first sequence goes on
    return d


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind,states", [("token", True), ("head", False)])
@pytest.mark.parametrize("shape,starts_at", SHAPES, ids=lambda s: str(s).replace(", ", "x"))
def test_plans(shape, starts_at, kind, states, dtype):
    import torch
    d = packed(shape, dtype, kind, states, starts_at, 51 + sum(shape))
    note(f"delta rule plan of {shape} {kind} states={states} {dtype}")
    ref, mag = reference(d)
    g = cuda(d)
    out, fin = forward(g)
    one = 0.5 if dtype == "bf16" else 1.0
    check(out, ref["out"], mag["out"], shape, "out", dtype == "bf16", one)
    check(fin, ref["final_state"], mag["final_state"], shape, "final_state", False)
    assert torch.equal(forward(g, return_final=False), out)
    got = backward(g)
    for name in NAMES:
        if got[name] is not None:
            check(got[name], ref[name], mag[name], shape, name, rounded_name(name, dtype), one if rounded_name(name, dtype) else 1.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("which", ["q", "k", "v", "dout"])
def test_a_bad_value_among_shared_heads(which, dtype):
    """An infinity in a block of five heads: pairs are summed one by one there, and other sequences and groups are as without it."""
    import torch
    shape = B, H, G, dk, dv, L = (16, 40, 8, 8, 12, 257)
    d = packed(shape, dtype, "token", True, 0, 77)
    ref, mag = reference(d)
    b, head, t = 5, 13, 150
    e = dict(d, **{which: d[which].clone()})
    groups = which in ("q", "k")
    e[which][b, head // 5 if groups else head, 3, t] = float("inf")
    seq = torch.cumsum((d["pos"] == 0).int(), 1)
    hit = torch.zeros(B, H, L, dtype=torch.bool)
    heads = slice(head // 5 * 5, head // 5 * 5 + 5) if groups else slice(head, head + 1)
    hit[b, heads] = seq[b] == seq[b, t]
    note(f"delta rule, infinite {which} in {shape} {dtype}")
    g = cuda(e)
    got = dict(backward(g), out=forward(g)[0])
    late = hit & (torch.arange(L) >= t)
    for name in ("out", "dq", "dk", "dv", "dbeta", "ddecay"):
        r, m = ref[name], mag[name]
        reach = late if name == "out" else hit
        if name == "out" and which in ("q", "dout"):
            reach = reach & (torch.arange(L) == t) if which == "q" else torch.zeros_like(hit)
        if name in ("dq", "dk"):
            reach = reach.view(B, G, H // G, L).any(2)
        keep = ~reach[:, :, None, :].expand_as(r) if r.dim() == 4 else ~reach
        x = got[name].double().cpu()
        tol = bound_of(r, m, shape, name, rounded_name(name, dtype))
        near = bool(((x - r).abs() <= tol)[keep].all())
        assert near, name
    if which != "dout":
        bad = got["out"][b, heads, :, t].isfinite().all()
        assert not bool(bad)
