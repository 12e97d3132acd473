"""GPU: the gated delta rule where what a state holds is far larger than what it answers: a value a thousand times the others,
which the next token of the same key replaces.  Its terms cancel in the outs and gradients of the tokens behind it, so that
what is rounded of them shows there, and not what is rounded of the results.

Tolerances, in the 2-norm over those tokens. With C the size of the terms that cancel over the compared results' (by length): a
sum of up to dk + 192 terms, each rounded to 32 bits by at most u = 2^-24 and apart from each other, is off by about sqrt(320) u
of its terms, 1.1e-6; e comes of two such sums and a result of one more: 4e-6 C. But k.k is one sum for all pairs of tokens,
whose error, at most dk u, is the same in all of them: e sums to x / (1 + dk u) where it should to x, which shows as dk u C. The
terms' size follows from beta |k|^2 = 1 with one key and no decay: S_t holds v_t along the key and D_t what makes dv_t, so that
with |q| = |k| = 1 the terms of out are as large as the largest |v|, of dq (S dout, dout's elements of size 1) scale |v|, of dv
|dv|, of dk (S dv and D u, whose sums over v's features have random signs) |v| |dv| / sqrt(dv) and |dv| |u| / sqrt(dv), the
largest of the row times the compared tokens'. The result's own length is no measure: that of the large token alone is a product
of two vectors that may be small by chance. bf16 results are rounded once: 2^-8 of themselves at most, spread evenly, 2^-8 /
sqrt 3."""
import pytest

from gpu_common import note
from test_gpu_delta import backward, cuda, forward, make, reference

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


def rms(x, tokens=slice(None)):
    return x[..., tokens].square().sum(2).mean().sqrt().item()


def largest(x):
    return x.square().sum(2).max().sqrt().item()


def near(got, ref, tokens, size, dk, rounded, name):
    got = got.double().cpu()
    C = size / rms(ref, tokens)
    rel = ((got - ref)[..., tokens].norm() / ref[..., tokens].norm()).item()
    tol = (4e-6 + dk * 2.0 ** -24) * max(C, 1) + (HALF / 3 ** 0.5 if rounded else 0)
    note(f"  {name} {rel:.2g} off of {tol:.2g}, terms {C:.2g} times the results")
    finite = bool(got.isfinite().all())
    assert finite and rel <= tol, f"{name}: {rel:.2g} off, {tol:.2g} allowed"


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
    size = largest(d["v"].double())
    near(out, ref["out"], tokens, size, shape[3], dtype == "bf16", "out")
    assert torch.equal(forward(g, return_final=False), out)
    if dtype == "bf16":
        near(forward(g, out_f32=True)[0], ref["out"], tokens, size, shape[3], False, "out in 32 bits")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("where,times", [(0, 1000), (63, 30), (63, 1000), (140, 1000), ("final", 30), ("final", 1000)])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_gradients_beside_a_large_value(shape, where, times, dtype):
    """dq, dk and dv of the tokens behind a large value, or before the last ones where the final state's gradient is large and its
    part along the key ends with them."""
    import torch
    d = same_keys(shape, dtype, 4)
    note(f"delta rule gradients, {where} times {times}, {shape} {dtype}")
    B, H, G, dk, dv, L = shape
    if where == "final":
        key = d["k"][..., :1].float().repeat_interleave(H // G, 1)
        d["dfinal"] = times * key * torch.randn((B, H, 1, dv), generator=torch.Generator().manual_seed(5))
        tokens = slice((L - 4) // 64 * 64, L - 3)
    else:
        d["v"][..., where] *= times
        tokens = slice(where + 3, (where + 3) // 64 * 64 + 64)
    ref, _ = reference(d)
    v, gv = d["v"].double(), ref["dv"]
    u = torch.diff(v, dim=-1, prepend=torch.zeros_like(v[..., :1]))
    sizes = {"dq": d["scale"] * largest(v), "dv": largest(gv),
             "dk": (largest(v) * rms(gv, tokens) + largest(gv) * rms(u, tokens)) / dv ** 0.5}
    g = cuda(d)
    for wide in (False, True)[:1 + (dtype == "bf16")]:
        got = backward(g, out_f32=wide)
        for name in ("dq", "dk", "dv"):
            near(got[name], ref[name], tokens, sizes[name], dk, dtype == "bf16" and not wide, name + " in 32 bits" * wide)
