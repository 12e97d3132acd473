"""GPU: the gated delta rule with log decays above 0, where the state is bounded by what its tokens replace, in rows that are
walked whole and in rows that are split, against 64 bits.

Tolerances, in the 2-norm, with g the decay and u = 2^-24: a chunk's sums hold terms up to e^(64 g) times the state, and H comes of
weights up to e^(64 g); each is off by as much more, in both at worst: e^(128 g) times what sums without growth are off by, 4e-6
(sqrt(320) u and three sums, as in test_gpu_delta_large).  A decay's gradient is left of sums over up to 256 tokens: 256 times
that.  bf16 results are rounded once besides, 2^-8 / sqrt 3."""
import math

import pytest

from gpu_common import note
from test_gpu_delta import NAMES, backward, cuda, forward, make, reference, rounded_name

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8


def growing(shape, dtype, g, states, seed=6):
    """Decays of g and up to a tenth less, no starts, keys replaced whole."""
    import torch
    d = make(shape, dtype, "token", states, seed)
    gen = torch.Generator().manual_seed(seed)
    d["decay"] = g * (1 - 0.1 * torch.rand(d["decay"].shape, generator=gen))
    d["beta"].fill_(1.0)
    d["pos"].copy_(torch.arange(shape[-1], dtype=torch.int32) + 1)
    return d


def near(got, ref, name, g, dtype):
    got = got.double().cpu()
    tol = 4e-6 * math.exp(128 * g) * (256 if name == "ddecay" else 1) + (HALF / 3 ** 0.5 if rounded_name(name, dtype) else 0)
    rel = ((got - ref).norm() / ref.norm()).item()
    note(f"  {name} {rel:.2g} off of {tol:.2g}")
    finite = bool(got.isfinite().all())
    assert finite, name
    assert rel <= tol, f"{name}: {rel:.2g} off, {tol:.2g} allowed"


# the last one in segments of 36 chunks, over each of which the decays sum to more than what 32 bits hold, e^88.7
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,g,states", [((2, 3, 1, 7, 16, 333), 0.03, False), ((1, 2, 2, 65, 70, 200), 0.01, True),
                                            ((1, 2, 1, 3, 5, 1500), 0.05, True), ((1, 128, 32, 3, 8, 9200), 0.042, True)], ids=lambda s: str(s))
def test_decays_above_zero(shape, g, states, dtype):
    note(f"delta rule, decays of {g}, {shape} states={states} {dtype}")
    d = growing(shape, dtype, g, states)
    ref, _ = reference(d)
    c = cuda(d)
    out, fin = forward(c)
    near(out, ref["out"], "out", g, dtype)
    near(fin, ref["final_state"], "final_state", g, dtype)
    got = backward(c)
    for name in NAMES:
        if got[name] is not None:
            near(got[name], ref[name], name, g, dtype)


LONG = (1, 128, 32, 3, 8, 9200)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nothing_grows_to_nothing(dtype):
    """States of 0 that are only decayed, by more than 32 bits hold over a segment, stay 0: a row whose first 5000 tokens write
    nothing, and heads that write and ask for nothing at all."""
    g, quiet = 0.042, 5000
    note(f"delta rule, decays of {g} over empty states, {dtype}")
    d = growing(LONG, dtype, g, False)
    d["beta"][..., :quiet] = 0.0
    ref, _ = reference(d, back=False)
    out, fin = forward(cuda(d))
    near(out, ref["out"], "out", g, dtype)
    near(fin, ref["final_state"], "final_state", g, dtype)
    assert not bool(out[..., :quiet].any())
    d = growing(LONG, dtype, g, False)
    d["beta"][:, :8] = 0.0
    d["dout"][:, :8] = 0.0
    ref, _ = reference(d)
    c = cuda(d)
    out, _ = forward(c)
    near(out, ref["out"], "out", g, dtype)
    got = backward(c)
    for name in ("dq", "dk", "dv", "dbeta", "ddecay"):
        near(got[name], ref[name], name, g, dtype)
        quiet_part = got[name][:, :8 // (4 if name in ("dq", "dk") else 1)]
        assert not bool(quiet_part.any()), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_features_of_zeros(dtype):
    """Heads filled up with features that no key and no query has: what they would hold is only decayed, and stays 0."""
    import torch
    g, shape = 0.042, (1, 128, 32, 5, 8, 9200)
    note(f"delta rule, decays of {g} over empty features, {dtype}")
    d = growing(shape, dtype, g, False)
    three = growing(LONG, dtype, g, False)
    for n in "qk":
        d[n] = torch.cat([three[n], torch.zeros_like(three[n][:, :, :2])], 2).contiguous()
    ref, _ = reference(d)
    c = cuda(d)
    out, fin = forward(c)
    near(out, ref["out"], "out", g, dtype)
    near(fin, ref["final_state"], "final_state", g, dtype)
    got = backward(c)
    for name in ("dq", "dk", "dv", "dbeta", "ddecay"):
        near(got[name], ref[name], name, g, dtype)
