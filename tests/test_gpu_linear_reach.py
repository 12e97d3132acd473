"""GPU: how far an infinity or a NaN reaches in linear attention: the outputs whose sums hold it, and no other.
References and bounds as in test_gpu_linear."""
import pytest

import linear_reference as R
from gpu_common import note
from test_gpu_linear import HALF, U, backward, cuda, forward, make

pytestmark = pytest.mark.gpu

# a value at token t: the tokens of its sequence whose results hold it
REACH = {"q": {"out": "t", "dq": "", "dk": "early", "dv": "early"},
         "k": {"out": "late", "dq": "late", "dk": "", "dv": "t"},
         "v": {"out": "late", "dq": "late", "dk": "t", "dv": ""},
         "dout": {"out": "", "dq": "t", "dk": "early", "dv": "early"},
         # the multiplier of t is between t - 1 and t
         "decay": {"out": "late", "dq": "late", "dk": "before", "dv": "before"}}
BAD = {"nan": 0x7fc00000, "negative nan": 0xffc00000 - (1 << 32), "inf": 0x7f800000}


# rows of a few chunks, split rows, and rows so many that a walk takes its form for them; t in a chunk's inside, its
# first and its last token
SHAPES = [(2, 2, 1, 32, 64, 200), (1, 2, 2, 128, 128, 700), (1, 3, 1, 16, 20, 61), (97, 8, 1, 16, 20, 130)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("place", ["inside", "first", "last"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_reach(shape, place, dtype):
    import torch
    B, H, G, dk, dv, L = shape
    if B > 90 and dtype == "f32":
        pytest.skip("the form of many rows is bf16's")
    d = make(shape, dtype, "token", True, 22, mean=30)
    b = B - 1
    chunk = (L // 2) // 64
    t = chunk * 64 + {"inside": 29, "first": 0, "last": 63}[place]
    t = min(t, L - 2)
    # t inside of a sequence that begins in its chunk or the one before (or before the row) and ends after it, another
    # one behind
    start, end = max(0, t - 40), min(L - 1, t + 25)
    d["pos"][b, start:end] = torch.arange(end - start, dtype=torch.int32) + (3 if start == 0 else 0)
    d["pos"][b, end:] = torch.arange(L - end, dtype=torch.int32)
    ref, mag = (R.reference(d["q"], d["k"], d["v"], d["decay"], d["pos"], d["scale"], d["initial"], d["dout"], d["dfinal"],
                            absolute=m) for m in (False, True))
    seq = torch.cumsum((d["pos"] == 0).int(), 1)
    same = torch.zeros(B, L, dtype=torch.bool)
    same[b] = seq[b] == seq[b, t]
    at = torch.arange(L)
    reach = {"": same & False, "t": same & (at == t), "late": same & (at >= t), "early": same & (at <= t), "before": same & (at < t)}
    n = 2 * (dk + dv + 128 + 2 * (-(-L // 64)) + H)

    def near(got, name, reached, rounded):
        got, r, m = got.double().cpu(), ref[name], mag[name]
        keep = (~reached)[:, None, None, :].expand_as(r) if r.dim() == 4 else (~reached)[:, None].expand_as(r)
        bound = (n + (1024 if name == "ddecay" else 0)) * U * m + 1e-30
        if rounded:
            bound = bound + (HALF + 2.0 ** -15) * m + HALF * r.abs()
        assert bool(((got - r).abs() <= bound)[keep].all()), name

    for which, tokens in REACH.items():
        for kind, bits in BAD.items():
            e = dict(d, **{which: d[which].clone()})
            bad = torch.tensor(bits, dtype=torch.int32).view(torch.float32)
            if which == "decay":
                e["decay"][b, :, t] = bad
            else:
                e[which][b, :, 0, t] = bad.to(d[which].dtype)
            note(f"linear attention reach of {which} {kind} at {t} {shape} {dtype}")
            g = cuda(e)
            out, fin = forward(g)
            got = dict(backward(g), out=out)
            for name, tok in tokens.items():
                near(got[name], name, reach[tok], dtype == "bf16")
                # and it does reach those
                hit = got[name].cpu()[b][..., reach[tok][b]]
                assert not tok or bool((~hit.isfinite()).any(1).any(0).all()), (which, name)
            near(got["ddecay"], "ddecay", same, False)
            # the row's last sequence is another one
            assert bool(fin.isfinite().all())
            other = torch.ones(B, dtype=torch.bool)
            other[b] = bool(seq[b, t] > 0)
            assert bool(got["dinitial_state"].cpu()[other].isfinite().all())
