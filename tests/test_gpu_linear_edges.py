"""GPU: linear attention where it can go wrong: infinities and NaN in other sequences, later tokens and padding,
decays of the lowest values, rows of starts only or of none, states cut and passed on, in place, on other
streams, captured, beyond 32-bit offsets.  References and bounds as in test_gpu_linear."""
import numpy as np
import pytest

import linear_reference as R
from gpu_common import note
from test_gpu_linear import HALF, U, backward, check, cuda, forward, make

pytestmark = pytest.mark.gpu

NAMES = ("dq", "dk", "dv", "ddecay", "dinitial_state")


def compare(d, shape, dtype, skip=()):
    """Forward and backward against the recurrence."""
    args = (d["q"], d["k"], d["v"], d["decay"], d["pos"], d["scale"], d["initial"], d["dout"], d["dfinal"])
    ref, mag = (R.reference(*args, absolute=m) for m in (False, True))
    g = cuda(d)
    out, fin = forward(g)
    check(out, ref["out"], mag["out"], shape, "out", dtype == "bf16")
    check(fin, ref["final_state"], mag["final_state"], shape, "final_state", False)
    got = backward(g)
    for n in NAMES:
        if got[n] is not None and n not in skip:
            check(got[n], ref[n], mag[n], shape, n, dtype == "bf16" and n in ("dq", "dk", "dv"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L", [2, 3, 4, 5, 7, 8, 9, 12, 127, 128, 192, 193])
def test_lengths(L, dtype):
    """Rows shorter than a vector, of odd lengths, and ends inside and at a chunk."""
    shape = (3, 4, 2, 20, 33, L)
    note(f"linear attention length {L} {dtype}")
    compare(make(shape, dtype, "token", True, 100 + L, mean=max(1, L // 3)), shape, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", ["starts", "none", "lowest", "cuts", "strong", "growth", "zero scale", "negative scale"])
def test_decays_and_starts(case, dtype):
    import torch
    shape = (2, 3, 1, 40, 64, 333)
    d = make(shape, dtype, "token", True, 7)
    note(f"linear attention {case} {dtype}")
    if case == "starts":
        d["pos"].zero_()                                    # every token a sequence of its own
    elif case == "none":
        d["pos"].copy_(torch.arange(333, dtype=torch.int32) + 5)
    elif case == "lowest":
        d["decay"][:, :, ::5] = float("-inf")
        d["decay"][:, :, 2::7] = torch.finfo(torch.float32).min
    elif case == "cuts":
        d["decay"][:, :, ::3] = -104.0                      # at and just above the value that cuts
        d["decay"][:, :, 1::9] = -100.0
    elif case == "strong":
        d["decay"].fill_(-7.0)
    elif case == "growth":
        d["decay"].copy_(0.02 * torch.rand(d["decay"].shape))
        d["pos"] = torch.from_numpy(R.positions(2, 333, 20, np.random.default_rng(5), True))
    elif case == "zero scale":
        d["scale"] = 0.0
    elif case == "negative scale":
        d["scale"] = -1.5
    compare(d, shape, dtype)


SHAPES = [(2, 2, 1, 32, 64, 200), (1, 2, 2, 128, 128, 700), (1, 3, 1, 16, 20, 61)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_nonfinite_stays(shape, dtype):
    """A bad value reaches its own sequence alone, and there no earlier (in the backward, no later) token.  What it
    does not reach is as near the reference as without it."""
    import torch
    B, H, G, dk, dv, L = shape
    d = make(shape, dtype, "token", True, 21, mean=30)
    args = lambda e: (e["q"], e["k"], e["v"], e["decay"], e["pos"], e["scale"], e["initial"], e["dout"], e["dfinal"])  # noqa: E731
    ref, mag = (R.reference(*args(d), absolute=m) for m in (False, True))
    seq = torch.cumsum((d["pos"] == 0).int(), 1)
    b, t = B - 1, (2 * L) // 3
    same = torch.zeros(B, L, dtype=torch.bool)
    same[b] = seq[b] == seq[b, t]
    late = same & (torch.arange(L) >= t)
    early = same & (torch.arange(L) <= t)
    n = 2 * (dk + dv + 128 + 2 * (-(-L // 64)) + H)

    def near(got, name, reached, rounded):
        got, r, m = got.double().cpu(), ref[name], mag[name]
        keep = (~reached)[:, None, None, :].expand_as(r) if r.dim() == 4 else (~reached)[:, None].expand_as(r)
        bound = (n + (1024 if name == "ddecay" else 0)) * U * m + 1e-30
        if rounded:
            bound = bound + (HALF + 2.0 ** -15) * m + HALF * r.abs()
        assert bool(((got - r).abs() <= bound)[keep].all()), name

    bf = dtype == "bf16"
    for which in ("q", "k", "v", "dout", "decay"):
        for bad in (float("nan"), float("inf")):
            e = dict(d, **{which: d[which].clone()})
            if which == "decay":
                e["decay"][b, :, t] = float("nan")
            else:
                e[which][b, :, 0, t] = bad
            note(f"linear attention {which} {bad} {shape} {dtype}")
            g = cuda(e)
            out, fin = forward(g)
            got = backward(g)
            reach = {"q": (same & (torch.arange(L) == t)), "dout": torch.zeros_like(same)}.get(which, late)
            near(out, "out", reach, bf)
            if which in ("q", "k", "v") and reach[b, t]:
                assert not bool(out[b, :, :, t].isfinite().all())
            ended = bool((seq[b, t] != seq[b, -1]) or which in ("q", "dout"))
            keep = torch.ones(B, dtype=torch.bool)
            keep[b] = ended
            assert bool(fin.cpu()[keep].isfinite().all())
            reach = {"q": {"dq": same & False, "dk": early, "dv": early}, "k": {"dq": late, "dk": same & False, "dv": same},
                     "v": {"dq": late, "dk": same, "dv": same & False}, "dout": {"dq": same, "dk": early, "dv": early},
                     "decay": {"dq": late, "dk": same, "dv": same}}[which]
            for name in ("dq", "dk", "dv"):
                near(got[name], name, reach[name], bf)
            near(got["ddecay"], "ddecay", same, False)
            lead = torch.ones(B, dtype=torch.bool)
            lead[b] = bool(seq[b, t] > 0)
            assert bool(got["dinitial_state"].cpu()[lead].isfinite().all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L,cut", [(150, 64), (150, 37), (600, 333), (90, 1)])
def test_cut_rows_equal_the_whole(L, cut, dtype):
    """A row cut in two, states and their gradients passed on, against the uncut reference."""
    import torch
    import paper_2408_03865_amd as P
    shape = (2, 4, 2, 32, 48, L)
    d = make(shape, dtype, "token", True, 33, mean=70)
    args = (d["q"], d["k"], d["v"], d["decay"], d["pos"], d["scale"], d["initial"], d["dout"], d["dfinal"])
    ref, mag = (R.reference(*args, absolute=m) for m in (False, True))
    g = cuda(d)
    part = [{k: v[..., s].contiguous() for k, v in g.items() if k in ("q", "k", "v", "decay", "pos", "dout")}
            for s in (slice(0, cut), slice(cut, L))]
    call = lambda p, **kw: P.linear_attention_fwd(p["q"], p["k"], p["v"], p["decay"], p["pos"], scale=g["scale"],  # noqa: E731
                                                  return_final=True, **kw)
    o1, mid = call(part[0], initial_state=g["initial"])
    o2, fin = call(part[1], initial_state=mid)
    bf = dtype == "bf16"
    check(torch.cat([o1, o2], -1), ref["out"], mag["out"], shape, "out", bf)
    check(fin, ref["final_state"], mag["final_state"], shape, "final_state", False)
    back = lambda p, **kw: P.linear_attention_bwd(p["q"], p["k"], p["v"], p["decay"], p["pos"], p["dout"],  # noqa: E731
                                                  scale=g["scale"], **kw)
    g2 = back(part[1], initial_state=mid, dfinal_state=g["dfinal"])
    g1 = back(part[0], initial_state=g["initial"], dfinal_state=g2["dinitial_state"])
    for n in ("dq", "dk", "dv", "ddecay"):
        check(torch.cat([g1[n], g2[n]], -1), ref[n], mag[n], shape, n, bf and n != "ddecay")
    check(g1["dinitial_state"], ref["dinitial_state"], mag["dinitial_state"], shape, "dinitial_state", False)


def test_same_results_again_in_place_and_elsewhere():
    """Bit for bit: the same call again, states updated in place, another stream, captured and replayed, with
    the caller's workspace; bf16 results are the rounded 32-bit ones."""
    import torch
    import paper_2408_03865_amd as P
    for shape, dtype in (((1, 6, 2, 64, 64, 700), "bf16"), ((2, 2, 2, 128, 40, 90), "f32")):
        note(f"linear attention again {shape} {dtype}")
        g = cuda(make(shape, dtype, "token", True, 44))
        out, fin = forward(g)
        grads = backward(g)

        def same(o, f, gr):
            assert torch.equal(o, out) and torch.equal(f, fin)
            for n in NAMES:
                assert torch.equal(gr[n], grads[n]), n

        same(*forward(g), backward(g))
        if dtype == "bf16":
            o32, f32 = forward(g, out_f32=True)
            g32 = backward(g, out_f32=True)
            assert torch.equal(o32.bfloat16(), out) and torch.equal(f32, fin)
            for n in NAMES:
                assert torch.equal(g32[n].to(grads[n].dtype), grads[n]), n
        # in place, through the C ABI: the final state over the initial, the initial state's gradient over the final's
        from paper_2408_03865_amd import _lib
        lib, p = _lib.load(), lambda t: t.data_ptr()
        B, H, G, dk, dv, L = shape
        code = _lib.BF16 if dtype == "bf16" else _lib.F32
        state, o = g["initial"].clone(), torch.empty_like(out)
        dims = (B, H, G, dk, dv, L)
        need = lib.packmamba_linear_attention_fwd_workspace_size(*dims)
        ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
        stream = torch.cuda.current_stream().cuda_stream
        st = lib.packmamba_linear_attention_fwd(p(g["q"]), p(g["k"]), p(g["v"]), p(g["decay"]), p(g["pos"]), p(state), g["scale"],
                                                p(o), p(state), p(ws), need, *dims, 1, code, stream)
        assert st == 0 and torch.equal(o, out) and torch.equal(state, fin)
        need = lib.packmamba_linear_attention_bwd_workspace_size(*dims)
        ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")       # NaN: everything read is written first
        r = {n: torch.empty_like(v) for n, v in grads.items()}
        dstate = g["dfinal"].clone()
        st = lib.packmamba_linear_attention_bwd(p(g["q"]), p(g["k"]), p(g["v"]), p(g["decay"]), p(g["pos"]), p(g["initial"]),
                                                g["scale"], p(g["dout"]), p(dstate), p(r["dq"]), p(r["dk"]), p(r["dv"]),
                                                p(r["ddecay"]), p(dstate), p(ws), need, *dims, 1, code, stream)
        r["dinitial_state"] = dstate
        assert st == 0
        same(o, state, r)
        # without the decay's gradient: the plain walks, whose results are within the bounds, not the same bits
        assert P.linear_attention_bwd(g["q"], g["k"], g["v"], g["decay"], g["pos"], g["dout"], decay_grad=False)["ddecay"] is None
        # another stream
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            res = (*forward(g), backward(g))
            graph = torch.cuda.CUDAGraph()
            side.synchronize()
            with torch.cuda.graph(graph, stream=side):
                go, gf = forward(g)
                gg = backward(g)
        torch.cuda.synchronize()
        same(*res)
        for _ in range(3):
            for v in (go, gf, *[gg[n] for n in NAMES]):
                v.fill_(float("nan"))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            same(go, gf, gg)


def test_step_and_norm_captured():
    import torch
    import paper_2408_03865_amd as P
    gen = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    q, k, v, z, w = r(5, 2, 64).bfloat16(), r(5, 2, 64).bfloat16(), r(5, 4, 64).bfloat16(), r(5, 256, 1).bfloat16(), r(256)
    decay, state0 = -torch.rand(4, device="cuda"), r(5, 4, 64, 64)
    pos = torch.tensor([0, 3, -1, 7, 0], dtype=torch.int32, device="cuda")

    def run(state):
        o = P.linear_attention_step(q, k, v, decay, state, pos, scale=0.125)
        y, rstd = P.gated_rmsnorm_fwd(o.reshape(5, 256, 1), z, w, groups=4)
        return (o, y, rstd) + P.gated_rmsnorm_bwd(o.reshape(5, 256, 1), z, w, rstd, y, groups=4)

    ref_state = state0.clone()
    ref = [run(ref_state) for _ in range(3)]
    state, side, graph = state0.clone(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            got = run(state)
    torch.cuda.synchronize()
    for want in ref:
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
    assert torch.equal(state, ref_state)
    assert torch.equal(state[2], state0[2]) and not bool(got[0][2].any())


def test_offsets_beyond_32_bits():
    """v and out of more than 2^32 elements: the last row as it is by itself."""
    import torch
    import paper_2408_03865_amd as P
    B, H, dk, dv, L = 9, 64, 16, 128, 65536
    note("linear attention with 4.8e9 elements")
    v = torch.empty((B, H, dv, L), dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    v[-1] = torch.randn((H, dv, L), generator=gen, device="cuda", dtype=torch.bfloat16)
    q, k = (torch.randn((B, 1, dk, L), generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    decay = -0.1 - torch.rand(H, generator=gen, device="cuda")
    pos = (torch.arange(L, device="cuda", dtype=torch.int32) % 5000).expand(B, L).contiguous()
    out = P.linear_attention_fwd(q, k, v, decay, pos)
    # two heads of it by themselves (copies: a view need not be 16-byte aligned), few enough to be split: within both results' bounds of each other
    one = P.linear_attention_fwd(q[-1:].contiguous(), k[-1:].contiguous(), v[-1:, -2:].contiguous(), decay[-2:].clone(), pos[-1:].clone())
    mag = P.linear_attention_fwd(q[-1:].abs(), k[-1:].abs(), v[-1:, -2:].abs(), decay[-2:].clone(), pos[-1:].clone(), out_f32=True)
    assert bool(((out[-1:, -2:].float() - one.float()).abs() <= 2 * (HALF * 1.02) * mag + 2 * HALF * one.float().abs()).all())
