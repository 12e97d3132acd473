"""GPU: the gated delta rule where what a state holds is far larger than what it answers: a value a thousand times the others,
which the next token of the same key replaces.  Its terms cancel in the outs and gradients of the tokens behind it, so that
what is rounded of them shows there, and not what is rounded of the results.

Tolerances, in the 2-norm over those tokens.  With C the largest token's result over the compared ones' (by length): a sum
of up to dk + 192 terms, each rounded to 32 bits by at most u = 2^-24 and apart from each other, is off by about sqrt(320) u of its
terms, 1.1e-6; e comes of two such sums and a result of one more: 4e-6 C.  bf16 results are rounded once: 2^-8 of themselves at
most, spread evenly, 2^-8 / sqrt 3."""
import pytest

from gpu_common import note
from test_gpu_delta import cuda, forward, make, reference

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8
SHAPES = [(1, 2, 2, 64, 64, 300), (1, 2, 1, 128, 128, 200), (2, 4, 2, 24, 40, 200), (1, 1, 1, 65, 64, 1400), (1, 2, 1, 64, 128, 300)]


def same_keys(shape, dtype, seed=3):
    """One key, written whole by every token, asked for by every query, nothing forgotten."""
    import torch
    d = make(shape, dtype, "none", False, seed)
    d["pos"].copy_(torch.arange(shape[-1], dtype=torch.int32) + 1)
    d["k"].copy_(d["k"][..., :1].float().div(0.99).to(d["k"].dtype).expand_as(d["k"]))
    d["q"].copy_(d["k"])
    d["beta"].copy_(1 / d["k"].float().square().sum(2).repeat_interleave(shape[1] // shape[2], 1))
    return d


def near(got, ref, tokens, rounded, name):
    got = got.double().cpu()
    length = ref.square().sum(2).sqrt()
    rms = length[..., tokens].square().mean().sqrt()
    C = (length.max() / rms).item()
    rel = ((got - ref)[..., tokens].norm() / ref[..., tokens].norm()).item()
    tol = 4e-6 * C + (HALF / 3 ** 0.5 if rounded else 0)
    note(f"  {name} {rel:.2g} off of {tol:.2g}, the largest {C:.2g} of these")
    assert got.isfinite().all() and rel <= tol, f"{name}: {rel:.2g} off, {tol:.2g} allowed"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("at,times", [(0, 30), (0, 1000), (63, 30), (63, 1000), (140, 1000)])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_outs_behind_a_large_value(shape, at, times, dtype):
    import torch
    d = same_keys(shape, dtype)
    d["v"][..., at] *= times
    note(f"delta rule, value {at} times {times}, {shape} {dtype}")
    ref, _ = reference(d, back=False)
    g = cuda(d)
    tokens = slice(at + 3, (at + 3) // 64 * 64 + 64)
    out, _ = forward(g)
    near(out, ref["out"], tokens, dtype == "bf16", "out")
    assert torch.equal(forward(g, return_final=False), out)
    if dtype == "bf16":
        near(forward(g, out_f32=True)[0], ref["out"], tokens, False, "out in 32 bits")
