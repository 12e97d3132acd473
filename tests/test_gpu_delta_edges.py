"""GPU: the gated delta rule where it can go wrong: infinities and NaN in other sequences, later tokens and padding, decays of
the lowest values, strengths of 0 and 2, repeated keys, rows of starts only or of none, states cut and passed on, in place,
on other streams, captured, beyond 32-bit offsets.  References and bounds as in test_gpu_delta."""
import numpy as np
import pytest

import linear_reference as R
from gpu_common import note
from test_gpu_delta import NAMES, backward, bound_of, check, cuda, forward, make, reference, rounded_name

pytestmark = pytest.mark.gpu


def compare(d, shape, dtype, case=""):
    """Forward and backward against the rule.  Where decays are e^-7 and less, ddecay is held by its elements' bounds alone
    (test_gpu_delta).  With keys all the same, beta 1 and no decay u_s is v_s - v_{s-1}, and S_t holds v_t as the sum of
    them: a chunk's 64 roundings of errors of length sqrt 2 |v| to bf16 add up as a random walk in dq and dk, to
    sqrt(64) sqrt 2 times one."""
    ref, mag = reference(d)
    g = cuda(d)
    out, fin = forward(g)
    check(out, ref["out"], mag["out"], shape, "out", dtype == "bf16")
    check(fin, ref["final_state"], mag["final_state"], shape, "final_state", False)
    got = backward(g)
    for n in NAMES:
        if got[n] is not None:
            norm = 0.0 if case in ("strong", "lowest", "cuts") and n == "ddecay" else 8 * 2 ** 0.5 if case == "same keys" and n in ("dq", "dk") else 1.0
            check(got[n], ref[n], mag[n], shape, n, rounded_name(n, dtype), norm=norm)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L", [2, 3, 4, 5, 7, 8, 9, 12, 127, 128, 192, 193, 255, 256, 257, 511, 512, 513, 769])
def test_lengths(L, dtype):
    """Rows shorter than a vector, of odd lengths, and ends inside and at a chunk, and at a boundary of the decays' sums."""
    shape = (3, 4, 2, 20, 33, L)
    note(f"delta rule length {L} {dtype}")
    compare(make(shape, dtype, "token", True, 100 + L, mean=max(1, L // 3)), shape, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1, 1, 128, 1, 70), (2, 2, 1, 1, 128, 70), (1, 2, 2, 3, 5, 200), (5, 8, 1, 96, 80, 130), (1, 24, 1, 64, 64, 100),
                                   (1, 1, 1, 64, 64, 3000), (2, 1, 1, 128, 128, 2000)], ids=lambda s: "x".join(map(str, s)))
def test_shapes(shape, dtype):
    """Heads of one feature, one group of many heads, one head of a long row (its sums in segments)."""
    note(f"delta rule {shape} {dtype}")
    compare(make(shape, dtype, "token", True, sum(shape), mean=700), shape, dtype)


CASES = ["starts", "none", "lowest", "cuts", "strong", "zero beta", "beta 2", "same keys", "zero keys", "zero scale", "negative scale", "segments of one"]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES)
def test_decays_strengths_and_starts(case, dtype):
    import torch
    shape = (2, 3, 1, 40, 64, 333)
    d = make(shape, dtype, "token", True, 7)
    note(f"delta rule {case} {dtype}")
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
    elif case == "zero beta":
        d["beta"][:, :, ::2] = 0.0
        d["beta"][:, 1] = 0.0
    elif case == "beta 2":
        d["beta"].fill_(2.0)                                # keys a little shorter than 1: reflections
        d["decay"].fill_(0.0)
    elif case == "same keys":
        d["k"].copy_(d["k"][..., :1].expand_as(d["k"]))     # the inverse's terms grow with the tokens, the errors vanish
        d["beta"].fill_(1.0)
        d["decay"].fill_(0.0)
        d["pos"].copy_(torch.arange(333, dtype=torch.int32) + 1)
    elif case == "zero keys":
        d["k"][..., ::2] = 0.0
        d["q"][..., 1::3] = 0.0
    elif case == "zero scale":
        d["scale"] = 0.0
    elif case == "negative scale":
        d["scale"] = -1.5
    elif case == "segments of one":
        d["pos"] = torch.from_numpy(R.positions(2, 333, 1, np.random.default_rng(5), True))
    compare(d, shape, dtype, case)


SHAPES = [(2, 2, 1, 32, 64, 200), (1, 2, 2, 128, 128, 700), (1, 3, 1, 16, 20, 61)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_nonfinite_stays(shape, dtype):
    """A bad value reaches its own sequence alone, and in the forward there no earlier token.  What it does not reach is as
    near the reference as without it."""
    import torch
    B, H, G, dk, dv, L = shape
    d = make(shape, dtype, "token", True, 21, mean=30)
    ref, mag = reference(d)
    seq = torch.cumsum((d["pos"] == 0).int(), 1)
    b = B - 1
    for t in ((2 * L) // 3, 64 if L > 70 else 5, 0):
        same = torch.zeros(B, L, dtype=torch.bool)
        same[b] = seq[b] == seq[b, t]
        late = same & (torch.arange(L) >= t)
        for which in ("q", "k", "v", "beta", "dout", "decay", "initial"):
            for bad in (float("nan"), float("inf")):
                e = dict(d, **{which: d[which].clone()})
                reach = late
                if which == "decay":
                    if d["pos"][b, t] == 0:
                        continue                             # a start takes nothing of it
                    e[which][b, :, t] = float("nan")
                elif which == "beta":
                    e[which][b, :, t] = bad
                elif which == "initial":
                    if t:
                        continue
                    e[which][b, :, 0, 0] = bad
                    reach = same if d["pos"][b, 0] else torch.zeros_like(same)
                else:
                    e[which][b, :, 0, t] = bad
                if which == "q":
                    reach = same & (torch.arange(L) == t)
                elif which == "dout":
                    reach = torch.zeros_like(same)
                note(f"delta rule {which} {bad} at {t} {shape} {dtype}")
                g = cuda(e)
                out, fin = forward(g)
                got = backward(g)

                def near(x, name, reached, rounded):
                    x, r, m = x.double().cpu(), ref[name], mag[name]
                    keep = (~reached)[:, None, None, :].expand_as(r) if r.dim() == 4 else (~reached)[:, None].expand_as(r)
                    assert bool(((x - r).abs() <= bound_of(r, m, shape, name, rounded))[keep].all()), name

                near(out, "out", reach, dtype == "bf16")
                if which in ("q", "k", "v"):
                    assert not bool(out[b, :, :, t].isfinite().all())
                ended = bool((seq[b, t] != seq[b, -1]) or which in ("q", "dout") or not bool(reach.any()))
                keep = torch.ones(B, dtype=torch.bool)
                keep[b] = ended
                assert bool(fin.cpu()[keep].isfinite().all())
                for name in ("dq", "dk", "dv", "dbeta", "ddecay"):
                    near(got[name], name, same, rounded_name(name, dtype))
                lead = torch.ones(B, dtype=torch.bool)
                lead[b] = bool(seq[b, t] > 0)
                assert bool(got["dinitial_state"].cpu()[lead].isfinite().all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nonfinite_state_ends_with_its_sequence(dtype):
    """A split row whose first sequence is spoiled: what follows its end is not, across segments."""
    import torch
    shape = (1, 1, 1, 64, 64, 1500)
    d = make(shape, dtype, "token", True, 3, mean=10 ** 6)
    d["pos"].copy_(torch.arange(1500, dtype=torch.int32) + 9)
    d["pos"][0, 700:] = torch.arange(800, dtype=torch.int32)
    ref, mag = reference(d)
    e = dict(d, initial=d["initial"].clone())
    e["initial"][0, 0, 3, 5] = float("nan")
    out, fin = forward(cuda(e))
    late = slice(700, None)
    tol = bound_of(ref["out"], mag["out"], shape, "out", dtype == "bf16")
    assert bool(((out.double().cpu() - ref["out"]).abs() <= tol)[..., late].all()) and bool(out[0, 0, 5, :700].isnan().all())
    check(fin, ref["final_state"], mag["final_state"], shape, "final_state", False)
    got = backward(cuda(e))
    for n in ("dq", "dk", "dv", "dbeta", "ddecay"):
        tol = bound_of(ref[n], mag[n], shape, n, rounded_name(n, dtype))
        assert bool(((got[n].double().cpu() - ref[n]).abs() <= tol)[..., late].all()), n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L,cut", [(150, 64), (150, 37), (600, 333), (90, 1), (1400, 700)])
def test_cut_rows_equal_the_whole(L, cut, dtype):
    """A row cut in two, states and their gradients passed on, against the uncut reference."""
    import torch
    import paper_2408_03865_amd as P
    shape = (2, 4, 2, 32, 48, L)
    d = make(shape, dtype, "token", True, 33, mean=70)
    ref, mag = reference(d)
    g = cuda(d)
    part = [{k: v[..., s].contiguous() for k, v in g.items() if k in ("q", "k", "v", "beta", "decay", "pos", "dout")}
            for s in (slice(0, cut), slice(cut, L))]
    ins = lambda p: (p["q"], p["k"], p["v"], p["beta"], p["decay"], p["pos"])  # noqa: E731
    o1, mid = P.delta_rule_fwd(*ins(part[0]), scale=g["scale"], return_final=True, initial_state=g["initial"])
    o2, fin = P.delta_rule_fwd(*ins(part[1]), scale=g["scale"], return_final=True, initial_state=mid)
    check(torch.cat([o1, o2], -1), ref["out"], mag["out"], shape, "out", dtype == "bf16")
    check(fin, ref["final_state"], mag["final_state"], shape, "final_state", False)
    g2 = P.delta_rule_bwd(*ins(part[1]), part[1]["dout"], scale=g["scale"], initial_state=mid, dfinal_state=g["dfinal"])
    g1 = P.delta_rule_bwd(*ins(part[0]), part[0]["dout"], scale=g["scale"], initial_state=g["initial"],
                          dfinal_state=g2["dinitial_state"])
    for n in ("dq", "dk", "dv", "dbeta", "ddecay"):
        check(torch.cat([g1[n], g2[n]], -1), ref[n], mag[n], shape, n, rounded_name(n, dtype))
    check(g1["dinitial_state"], ref["dinitial_state"], mag["dinitial_state"], shape, "dinitial_state", False)


def test_gradients_are_differences():
    """The gradients against differences of the kernel's own forward, 32-bit: a step of 2^-6 in one input moves the loss by the
    gradient times it, up to the third order (2^-12 of the loss' scale here) and the sum's rounding."""
    import torch
    shape = (1, 2, 1, 8, 8, 40)
    d = make(shape, "f32", "token", True, 5, mean=15)
    g = cuda(d)
    grads = backward(g)

    def loss(h):
        out, fin = forward(h)
        return ((out.double() * g["dout"].double()).sum() + (fin.double() * g["dfinal"].double()).sum()).item()

    h = 2.0 ** -6
    gen = torch.Generator().manual_seed(1)
    for name, grad in (("q", "dq"), ("k", "dk"), ("v", "dv"), ("beta", "dbeta"), ("decay", "ddecay"), ("initial", "dinitial_state")):
        for _ in range(6):
            i = int(torch.randint(g[name].numel(), (1,), generator=gen))
            vals = []
            for s in (h, -h):
                x = g[name].clone()
                x.view(-1)[i] += s
                vals.append(loss(dict(g, **{name: x})))
            want = 0.0 if name == "decay" and int(d["pos"][0, i % 40]) == 0 else (vals[0] - vals[1]) / (2 * h)
            got = float(grads[grad].reshape(-1)[i])
            assert abs(got - want) <= 2.0 ** -9 * (abs(want) + 4), (name, i, got, want)


def test_same_results_again_in_place_and_elsewhere():
    """Bit for bit: the same call again, states updated in place, another stream, captured and replayed, with
    the caller's workspace; bf16 results are the rounded 32-bit ones."""
    import torch
    for shape, dtype in (((1, 6, 2, 64, 64, 1400), "bf16"), ((2, 2, 2, 128, 40, 90), "f32"), ((1, 2, 1, 128, 128, 1100), "bf16")):
        note(f"delta rule again {shape} {dtype}")
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
        B, H, G, dk, dv, L = dims = shape
        code = _lib.BF16 if dtype == "bf16" else _lib.F32
        state, o = g["initial"].clone(), torch.empty_like(out)
        need = lib.packmamba_delta_rule_fwd_workspace_size(*dims)
        ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")       # NaN: everything read is written first
        stream = torch.cuda.current_stream().cuda_stream
        st = lib.packmamba_delta_rule_fwd(p(g["q"]), p(g["k"]), p(g["v"]), p(g["beta"]), p(g["decay"]), p(g["pos"]), p(state),
                                          g["scale"], p(o), p(state), p(ws), need, *dims, 1, code, stream)
        assert st == 0 and torch.equal(o, out) and torch.equal(state, fin)
        need = lib.packmamba_delta_rule_bwd_workspace_size(*dims, code)
        ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
        r = {n: torch.empty_like(v) for n, v in grads.items()}
        dstate = g["dfinal"].clone()
        st = lib.packmamba_delta_rule_bwd(p(g["q"]), p(g["k"]), p(g["v"]), p(g["beta"]), p(g["decay"]), p(g["pos"]), p(g["initial"]),
                                          g["scale"], p(g["dout"]), p(dstate), p(r["dq"]), p(r["dk"]), p(r["dv"]), p(r["dbeta"]),
                                          p(r["ddecay"]), p(dstate), p(ws), need, *dims, 1, code, stream)
        r["dinitial_state"] = dstate
        assert st == 0
        same(o, state, r)
        assert backward(g, decay_grad=False)["ddecay"] is None
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


def test_what_lies_beside_stays():
    """Nothing is written before or after the outputs and the workspace, and nothing of the inputs."""
    import torch
    from paper_2408_03865_amd import _lib
    lib = _lib.load()
    for dtype in ("bf16", "f32"):
        for shape in ((2, 3, 1, 33, 47, 77), (1, 2, 2, 128, 65, 1029)):
            note(f"delta rule guards {shape} {dtype}")
            B, H, G, dk, dv, L = shape
            g = cuda(make(shape, dtype, "token", True, 9))
            keep = {n: t.clone() for n, t in g.items() if isinstance(t, torch.Tensor)}
            code = _lib.BF16 if dtype == "bf16" else _lib.F32
            held = []

            def out(like, nbytes=None):
                n = like.numel() * like.element_size() if nbytes is None else nbytes
                whole = torch.full((n + 512,), 0xa5, dtype=torch.uint8, device="cuda")
                held.append((whole, n))
                return whole.data_ptr() + 256

            p = lambda t: t.data_ptr()  # noqa: E731
            ins = [p(g[n]) for n in ("q", "k", "v", "beta", "decay", "pos", "initial")]
            need = lib.packmamba_delta_rule_fwd_workspace_size(*shape)
            st = lib.packmamba_delta_rule_fwd(*ins, g["scale"], out(g["v"]), out(g["initial"]), out(None, need), need, *shape, 1, code,
                                              torch.cuda.current_stream().cuda_stream)
            assert st == 0
            need = lib.packmamba_delta_rule_bwd_workspace_size(*shape, code)
            st = lib.packmamba_delta_rule_bwd(*ins, g["scale"], p(g["dout"]), p(g["dfinal"]), out(g["q"]), out(g["k"]), out(g["v"]),
                                              out(g["beta"]), out(g["decay"]), out(g["initial"]), out(None, need), need, *shape, 1, code,
                                              torch.cuda.current_stream().cuda_stream)
            assert st == 0
            torch.cuda.synchronize()
            for whole, n in held:
                assert bool((whole[:256] == 0xa5).all()) and bool((whole[256 + n:] == 0xa5).all())
            for n, t in keep.items():
                assert torch.equal(t, g[n]), n


def test_offsets_beyond_32_bits():
    """v and out of more than 2^32 elements: the last row as it is by itself."""
    import torch
    import paper_2408_03865_amd as P
    B, H, dk, dv, L = 9, 64, 16, 128, 65536
    note("delta rule with 4.8e9 elements")
    v = torch.empty((B, H, dv, L), dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    v[-1] = torch.randn((H, dv, L), generator=gen, device="cuda", dtype=torch.bfloat16)
    q, k = (torch.randn((B, 1, dk, L), generator=gen, device="cuda", dtype=torch.bfloat16) * 0.2 for _ in range(2))
    beta = torch.rand((B, H, L), generator=gen, device="cuda")
    decay = -0.1 - torch.rand(H, generator=gen, device="cuda")
    pos = (torch.arange(L, device="cuda", dtype=torch.int32) % 5000).expand(B, L).contiguous()
    out = P.delta_rule_fwd(q, k, v, beta, decay, pos)
    # two heads of it by themselves, few enough to be split: apart by both results' roundings to bf16, four of at most 2^-8 each
    # of the budget of norms |q| (|v| + |S|), here below 8 times the largest out
    one = P.delta_rule_fwd(q[-1:].contiguous(), k[-1:].contiguous(), v[-1:, -2:].contiguous(), beta[-1:, -2:].contiguous(), decay[-2:].clone(),
                           pos[-1:].clone())
    a, b = out[-1:, -2:].float(), one.float()
    assert bool(b.any()) and bool(((a - b).abs() <= 8 * 2.0 ** -8 * 8 * b.abs().max()).all())
    assert float((a - b).norm() / b.norm()) <= 2.0 ** -7
