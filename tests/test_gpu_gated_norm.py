"""GPU: the gated RMSNorm, forward and backward, against 64 bits.

With u = 2^-24 and every term by its absolute value: the gate is off by 12 u (|z| 2 u through the exponential,
which e^-|z| |z| < 0.4 bounds where it counts; a sum, a reciprocal of 1 u and a product), a group's sum of n terms by
(n + 30) u, its root by half of that.  Values below are held to 2 (n + 40) u of their magnitude M (dweight:
with the number of tokens in place of n), and in bf16 to their own rounding, 2^-8 |value|, besides."""
import pytest

from gpu_common import note

pytestmark = pytest.mark.gpu

U, HALF, EPS = 2.0 ** -24, 2.0 ** -8, 1e-5


def reference(x, z, w, dout, groups, first, rstd=None):
    """Values and the sums over absolute terms, in doubles."""
    import torch
    x, z, w, g = x.double(), z.double(), w.double()[:, None], dout.double()
    B, D, L = x.shape
    per = D // groups
    mean = lambda t: t.view(B, groups, per, L).mean(2)  # noqa: E731
    up = lambda t: t[:, :, None].expand(B, groups, per, L).reshape(B, D, L)  # noqa: E731
    sig = torch.sigmoid(z)
    gate, dgate = z * sig, sig * (1 + z * (1 - sig))
    mdg = sig * (1 + z.abs() * (1 - sig))
    a = x * gate if first else x
    r = 1 / torch.sqrt(mean(a * a) + EPS)
    out = a * up(r) * w * (1 if first else gate)
    if rstd is not None:
        r = rstd.double()
    R = up(r)
    d = g * w if first else g * w * gate
    s, ms = up(mean(d * a)), up(mean((d * a).abs()))
    da, mda = R * (d - a * R * R * s), R * (d.abs() + a.abs() * R * R * ms)
    if first:
        dx, mdx, dz, mdz, dw = da * gate, mda * gate.abs(), da * x * dgate, mda * x.abs() * mdg, g * a * R
    else:
        dx, mdx, dz, mdz, dw = da, mda, g * w * a * R * dgate, (g * w * a * R).abs() * mdg, g * gate * a * R
    return {"out": (out, out.abs()), "rstd": (r, r), "dx": (dx, mdx), "dz": (dz, mdz),
            "dweight": (dw.sum((0, 2)), dw.abs().sum((0, 2)))}


def held(name, got, ref, n, rounded):
    got = got.double().cpu()
    assert got.shape == ref[0].shape and bool(got.isfinite().all()), name
    bound = 2 * (n + 40) * U * ref[1] + (HALF * ref[0].abs() if rounded else 0) + 1e-37
    over = ((got - ref[0]).abs() / bound).max().item()
    note(f"  {name} {over:.2g} of its bound")
    assert over <= 1, name


# one token, tiles of whole and of partial vectors, odd lengths, groups of one feature, of few and of more than is kept
SHAPES = [(1, 1, 1, 1), (5, 96, 1, 1), (3, 4096, 1, 1), (2, 70, 33, 1), (2, 48, 64, 6), (3, 24, 130, 24), (1, 640, 100, 5),
          (2, 1100, 72, 1), (1, 2600, 129, 2), (1, 5000, 40, 1), (70, 64, 7, 2),
          # tiles of 64 tokens: more than 64 of them, groups for each number of threads; then 64, of 16 tokens each
          (3, 36, 130, 12), (33, 200, 70, 1), (70, 300, 9, 1), (33, 1100, 72, 1), (34, 1040, 64, 2), (66, 4200, 33, 1),
          (1, 40, 4160, 1), (1, 40, 4096, 1), (4, 1040, 1016, 1), (1, 128, 16, 64)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("first", [True, False])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_gated_norm(shape, first, dtype):
    import torch
    import paper_2408_03865_amd as P
    B, D, L, groups = shape
    gen = torch.Generator().manual_seed(sum(shape))
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    x, z, dout = (2 * torch.randn((B, D, L), generator=gen).to(t) for _ in range(3))
    w = torch.randn(D, generator=gen)
    note(f"gated norm {shape} first={first} {dtype}")
    bf = dtype == "bf16"
    X, Z, Wt, G = x.cuda(), z.cuda(), w.cuda(), dout.cuda()
    out, rstd = P.gated_rmsnorm_fwd(X, Z, Wt, groups=groups, gate_first=first)
    dx, dz, dw = P.gated_rmsnorm_bwd(X, Z, Wt, rstd, G, groups=groups, gate_first=first)
    assert out.dtype == dx.dtype == dz.dtype == t
    ref = reference(x, z, w, dout, groups, first)
    per = D // groups
    held("out", out, ref["out"], per, bf)
    held("rstd", rstd, ref["rstd"], per, False)
    ref = reference(x, z, w, dout, groups, first, rstd.cpu())
    held("dx", dx, ref["dx"], per, bf)
    held("dz", dz, ref["dz"], per, bf)
    held("dweight", dw, ref["dweight"], B * L, False)
    if bf:                                  # the same before the last rounding
        o32, r32 = P.gated_rmsnorm_fwd(X, Z, Wt, groups=groups, gate_first=first, out_f32=True)
        d32 = P.gated_rmsnorm_bwd(X, Z, Wt, rstd, G, groups=groups, gate_first=first, out_f32=True)
        assert torch.equal(o32.to(t), out) and torch.equal(r32, rstd)
        assert torch.equal(d32[0].to(t), dx) and torch.equal(d32[1].to(t), dz) and torch.equal(d32[2], dw)


@pytest.mark.parametrize("first", [True, False])
def test_gated_norm_differences(first):
    """dx, dz and dweight against central differences of the forward, 32-bit."""
    import torch
    import paper_2408_03865_amd as P
    gen = torch.Generator().manual_seed(9)
    x, z, dout = (torch.randn((1, 12, 9), generator=gen).cuda() for _ in range(3))
    w = torch.randn(12, generator=gen).cuda()
    out, rstd = P.gated_rmsnorm_fwd(x, z, w, groups=3, gate_first=first)
    got = P.gated_rmsnorm_bwd(x, z, w, rstd, dout, groups=3, gate_first=first)
    # step h: the third derivative's h^2 / 6, and 32-bit sums of 108 terms of up to about 10 over 2 h
    h = 2.0 ** -6
    for t, g in zip((x, z, w), got):
        for i in range(0, t.numel(), 5):
            old = t.view(-1)[i].item()
            vals = []
            for s in (h, -h):
                t.view(-1)[i] = old + s
                vals.append((P.gated_rmsnorm_fwd(x, z, w, groups=3, gate_first=first)[0].double() * dout.double()).sum().item())
            t.view(-1)[i] = old
            num = (vals[0] - vals[1]) / (2 * h)
            assert abs(num - g.view(-1)[i].item()) <= 50 * h * h + 108 * 10 * 8 * U / (2 * h), (i, num, g.view(-1)[i].item())
