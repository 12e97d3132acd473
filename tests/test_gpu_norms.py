"""GPU: the layer norm and the norm by a head's length against 64 bits.

With u = 2^-24, n features and t tokens.  Length: the sum of squares is off by (n + 1) u of itself (its terms are all
positive), rnorm by half of that and 4 u (root, quotient); out adds 1 u.  Its backward: the sum of x g by (n + 2) u sum |x g|.
Layer norm: the mean is off by (n + 4) u mean|x| =: m; (x - mean) by m + u |x - mean|; the variance by the squares' sum
2 n u var, by the threads' differences from their own first feature, at most 2 n u (max - min)^2 of one thread's share, and by
m^2 + 2 m std; out adds 4 u of its terms.  Sums over tokens: t u of the terms' absolute values besides the terms' own errors.
bf16 results are rounded once more: 2^-8 of themselves."""
import numpy as np
import pytest

from gpu_common import note

pytestmark = pytest.mark.gpu

U, HALF = 2.0 ** -24, 2.0 ** -8


def within(got, ref, tol, name):
    got = got.double().cpu()
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    over = ((got - ref).abs() / (tol + 1e-30)).max().item()
    note(f"  {name} {over:.2g} of its bound")
    assert over <= 1, f"{name}: {over:.2f} of its bound"


def data(shape, dtype, seed, kind="plain"):
    import torch
    gen = torch.Generator().manual_seed(seed)
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    x = torch.randn(shape, generator=gen)
    if kind == "offset":
        x = x + 30.0
    elif kind == "first":                     # one feature far from the others
        x[:, 0] += 1000.0
    elif kind == "constant":
        x = torch.full(shape, 3.0)
    elif kind == "zero":
        x = torch.zeros(shape)
    g, r = (torch.randn(shape, generator=gen).to(t) for _ in range(2))
    return x.to(t), g, r, 1 + 0.2 * torch.randn(shape[1], generator=gen), torch.randn(shape[1], generator=gen)


def rounding(ref, dtype):
    return HALF * ref.abs() if dtype == "bf16" else 0 * ref


LAYER = [(1, 1, 1), (3, 7, 1), (5, 2048, 1), (2, 2050, 1), (70, 300, 1), (2, 33, 5), (1, 64, 8), (3, 100, 17), (2, 700, 130), (1, 2048, 512),
         (4, 1000, 1001), (17, 2560, 576), (40, 96, 333), (9, 256, 2051), (2, 1024, 4096), (1, 9000, 64)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", LAYER, ids=lambda s: "x".join(map(str, s)))
def test_layernorm(shape, dtype):
    kinds = ["plain"] if shape[0] * shape[1] * shape[2] > 1 << 20 else ["plain", "offset", "first", "constant", "zero"]
    for kind in kinds:
        layer(shape, dtype, kind)


def layer(shape, dtype, kind):
    import torch
    import paper_2408_03865_amd as P
    B, n, L = shape
    eps = 1e-5
    x, g, res, w, b = data(shape, dtype, sum(shape), kind)
    note(f"layer norm {shape} {dtype} {kind}")
    xd, wd, bd = x.double(), w.double()[:, None], b.double()[:, None]
    mean = xd.mean(1)
    c = xd - mean[:, None]
    var = c.square().mean(1)
    r = (var + eps).rsqrt()
    m = (n + 4) * U * xd.abs().mean(1)
    spread = (xd.amax(1) - xd.amin(1)).square()
    # the share of the sum that one thread's first feature can spoil: its own difference, met by at most n / 64 others
    dvar = 2 * (n + 8) * U * var + m.square() + 2 * m * var.sqrt() + 8 * U * spread * (n / 64 + 1) / n
    dr = r * (0.5 * dvar * r.square() + 4 * U)
    rows = lambda t: t[:, None]  # noqa: E731
    gx = [t.cuda() for t in (x, w, b)]
    out, gm, gr = P.layernorm_fwd(*gx, eps=eps)
    assert out.dtype == x.dtype
    within(gm, mean, m, "mean")
    within(gr, r, dr, "rstd")
    ref = c * rows(r) * wd + bd
    tol = (rows(m) * rows(r) + c.abs() * rows(dr) + 4 * U * (c.abs() * rows(r))) * wd.abs() + 2 * U * (ref.abs() + bd.abs())
    within(out, ref, tol + rounding(ref, dtype), "out")
    if dtype == "bf16":
        assert torch.equal(P.layernorm_fwd(*gx, eps=eps, out_f32=True)[0].bfloat16(), out)
    nob = P.layernorm_fwd(gx[0], gx[1], eps=eps)[0]
    within(nob, ref - bd, tol + rounding(ref - bd, dtype), "out without bias")
    # backward, from moments of 32 bits that are given
    mf, rf = mean.float(), r.float()
    c, r = xd - rows(mf.double()), rows(rf.double())
    h, gd = c * r, g.double()
    up = gd * wd
    s1, s2 = up.mean(1, keepdim=True), (up * h).mean(1, keepdim=True)
    a1, a2 = up.abs().mean(1, keepdim=True), (up * h).abs().mean(1, keepdim=True)
    dh = 3 * U * h.abs() + U * rows(mf.double().abs()) * r
    for with_res in (False, True):
        dx, dw, db = P.layernorm_bwd(gx[0], gx[1], mf.cuda(), rf.cuda(), g.cuda(), dresidual=res.cuda() if with_res else None)
        ref = r * (up - s1 - h * s2) + (res.double() if with_res else 0)
        tol = r * ((n + 4) * U * (a1 + h.abs() * a2) + dh * s2.abs() + h.abs() * (up.abs() * dh).mean(1, keepdim=True)
                   + 6 * U * (up.abs() + s1.abs() + (h * s2).abs())) + 2 * U * ref.abs()
        within(dx, ref, tol + rounding(ref, dtype), f"dx {with_res}")
        t = B * L
        within(dw, (gd * h).sum((0, 2)), (t * U * (gd * h).abs() + gd.abs() * dh).sum((0, 2)), "dweight")
        within(db, gd.sum((0, 2)), (t * U * gd.abs()).sum((0, 2)), "dbias")
    dx2, dw2, none = P.layernorm_bwd(gx[0], gx[1], mf.cuda(), rf.cuda(), g.cuda(), dresidual=res.cuda(), bias_grad=False)
    assert none is None and torch.equal(dx2, dx) and torch.equal(dw2, dw)


HEADS = [(1, 1, 1, 1), (3, 4, 32, 1), (2, 3, 600, 1), (2, 3, 7, 5), (2, 8, 64, 16), (3, 5, 33, 17), (2, 24, 64, 301), (1, 16, 128, 4096),
         (2, 3, 256, 130), (1, 2, 300, 77), (1, 1, 1000, 100), (40, 6, 8, 65)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", HEADS, ids=lambda s: "x".join(map(str, s)))
def test_head_l2norm(shape, dtype):
    import torch
    import paper_2408_03865_amd as P
    B, G, n, L = shape
    for kind in ("plain", "zero"):
        x, g, _, _, _ = data((B, G * n, L), dtype, sum(shape), kind)
        note(f"head l2 norm {shape} {dtype} {kind}")
        eps = 1e-6
        xd, gd = x.double().view(B, G, n, L), g.double().view(B, G, n, L)
        r = (xd.square().sum(2) + eps).rsqrt()
        dr = ((n + 3) / 2 + 4) * U
        out, gr = P.head_l2norm_fwd(x.cuda(), groups=G, eps=eps)
        assert out.dtype == x.dtype
        within(gr, r, dr * r, "rnorm")
        ref = (xd * r[:, :, None]).view(x.shape)
        within(out, ref, (dr + 2 * U) * ref.abs() + rounding(ref, dtype), "out")
        rf = r.float()
        r = rf.double()[:, :, None]
        s, sa = (xd * gd).sum(2, keepdim=True), (xd * gd).abs().sum(2, keepdim=True)
        ref = (r * (gd - xd * r * r * s)).view(x.shape)
        tol = r * (4 * U * gd.abs() + (n + 8) * U * (xd.abs() * r * r * sa))
        dx = P.head_l2norm_bwd(x.cuda(), rf.cuda(), g.cuda(), groups=G)
        within(dx, ref, tol.view(x.shape) + rounding(ref, dtype), "dx")
        if dtype == "bf16":
            assert torch.equal(P.head_l2norm_bwd(x.cuda(), rf.cuda(), g.cuda(), groups=G, out_f32=True).bfloat16(), dx)


def test_nonfinite_stays_with_its_token():
    import torch
    import paper_2408_03865_amd as P
    for L in (1, 5, 65, 300):
        x, g, _, w, b = data((3, 64, L), "f32", L)
        t = L // 2
        y = x.clone()
        y[1, 5, t] = float("nan")
        y[2, 9, t] = float("inf")
        for a, c in ((P.layernorm_fwd(x.cuda(), w.cuda(), b.cuda())[0], P.layernorm_fwd(y.cuda(), w.cuda(), b.cuda())[0]),
                     (P.head_l2norm_fwd(x.cuda(), groups=2)[0], P.head_l2norm_fwd(y.cuda(), groups=2)[0])):
            keep = torch.ones(3, L, dtype=torch.bool, device="cuda")
            keep[1:, t] = False
            keep = keep[:, None].expand(3, 64, L)
            assert torch.equal(a[keep], c[keep])
            assert not bool(c[1, 5, t].isfinite()) and not bool(c[2, 9, t].isfinite())
