"""GPU: the norms where they could go wrong beside their sums: what lies next to their outputs, offsets beyond 32 bits, the
same call again."""
import pytest

from gpu_common import note

pytestmark = pytest.mark.gpu

U, HALF = 2.0 ** -24, 2.0 ** -8


def test_what_lies_beside_stays():
    """Nothing is written before or after the outputs and the workspace, and nothing of the inputs."""
    import torch
    from paper_2408_03865_amd import _lib
    lib = _lib.load()
    s = torch.cuda.current_stream().cuda_stream
    for dtype, code in ((torch.float32, _lib.F32), (torch.bfloat16, _lib.BF16)):
        for B, D, L, G in ((1, 1, 1, 1), (3, 70, 1, 7), (2, 33, 5, 3), (2, 96, 77, 6), (5, 600, 1031, 4), (40, 64, 333, 2), (9, 2050, 290, 1)):
            note(f"norms' guards {B}x{D}x{L} {dtype}")
            gen = torch.Generator(device="cuda").manual_seed(D + L)
            r = lambda *n: torch.randn(n, generator=gen, device="cuda")  # noqa: E731
            x, g, res = (r(B, D, L).to(dtype) for _ in range(3))
            w, b, mean, rstd, rnorm = r(D), r(D), r(B, L), r(B, L).abs(), r(B, G, L).abs()
            ins = [x, g, res, w, b, mean, rstd, rnorm]
            keep = [t.clone() for t in ins]
            held = []

            def out(like, nbytes=None):
                n = like.numel() * like.element_size() if nbytes is None else nbytes
                whole = torch.full(((n + 15) // 16 * 16 + 512,), 0xa5, dtype=torch.uint8, device="cuda")
                held.append((whole, n))
                return whole.data_ptr() + 256

            p = lambda t: t.data_ptr()  # noqa: E731
            need = lib.packmamba_layernorm_bwd_workspace_size(B, D, L, code)
            st = [lib.packmamba_head_l2norm_fwd(p(x), 1e-6, out(x), out(rnorm), B, D, L, G, code, s),
                  lib.packmamba_head_l2norm_bwd(p(x), p(rnorm), p(g), out(x), B, D, L, G, code, s),
                  lib.packmamba_layernorm_fwd(p(x), p(w), p(b), 1e-5, out(x), out(mean), out(rstd), B, D, L, code, s),
                  lib.packmamba_layernorm_bwd(p(x), p(w), p(mean), p(rstd), p(g), p(res), out(x), out(w), out(w), out(None, need), need,
                                              B, D, L, code, s)]
            assert st == [0] * 4
            torch.cuda.synchronize()
            for whole, n in held:
                assert bool((whole[:256] == 0xa5).all()) and bool((whole[256 + n:] == 0xa5).all())
            assert all(torch.equal(a, c) for a, c in zip(ins, keep))


def test_same_results_again():
    """Two calls at once, on two streams, and a call after them: the same bits."""
    import torch
    import paper_2408_03865_amd as P
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, g = (torch.randn((5, 768, 2051), generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    w, b = torch.randn(768, generator=gen, device="cuda"), torch.randn(768, generator=gen, device="cuda")

    def run():
        o, m, s = P.layernorm_fwd(x, w, b)
        h, r = P.head_l2norm_fwd(x, groups=12)
        return [o, m, s, h, r, *P.layernorm_bwd(x, w, m, s, g), P.head_l2norm_bwd(x, r, g, groups=12)]

    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for s in streams:
        with torch.cuda.stream(s):
            got.append(run())
    torch.cuda.synchronize()
    want = run()
    assert all(torch.equal(t, c) for one in got for t, c in zip(one, want, strict=True))


def test_offsets_beyond_32_bits():
    """Rows of more than 2^32 elements: their end as it is by itself."""
    import torch
    import paper_2408_03865_amd as P
    D, L, n = 4100, (1 << 20) + 8, 1032
    note(f"norms of {D} x {L}")
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, g = (torch.randn((1, D, L), generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    w, b = 1 + 0.2 * torch.randn(D, generator=gen, device="cuda"), torch.randn(D, generator=gen, device="cuda")
    out, mean, rstd = P.layernorm_fwd(x, w, b)
    dx, dw, db = P.layernorm_bwd(x, w, mean, rstd, g)
    X, Gd = (t[..., -n:].contiguous() for t in (x, g))
    o1, m1, r1 = P.layernorm_fwd(X, w, b)
    dx1, _, _ = P.layernorm_bwd(X, w, m1, r1, Gd)
    # sums of D terms in 32 bits, in any two orders: apart by c = 4 (D + 40) u of their terms' sizes, which are those of x about
    # its mean and, backwards, up = |g w| and its means with h; bf16 rounds both, by half a step of values that differ by as much
    c = 4 * (D + 40) * U
    xf, up = X.float(), (Gd.float() * w[:, None]).abs()
    h = ((xf - m1[:, None]) * r1[:, None]).abs()
    assert bool(((mean[..., -n:] - m1).abs() <= c * xf.abs().mean(1)).all()) and bool(((rstd[..., -n:] - r1).abs() <= c * r1).all())
    mo = (h + xf.abs().mean(1, keepdim=True) * r1[:, None]) * w[:, None].abs() + b[:, None].abs()
    md = r1[:, None] * (up + up.mean(1, keepdim=True) + h * (up * h).mean(1, keepdim=True) + 2 * (up * h).mean(1, keepdim=True))
    for name, big, one, m in (("out", out, o1, mo), ("dx", dx, dx1, md)):
        one = one.float()
        assert bool(((big[..., -n:].float() - one).abs() <= c * 1.02 * m + 2 * HALF * (one.abs() * 1.01 + c * m) + 1e-37).all()), name
    # dweight and dbias: the whole row's sums, by 64-bit sums over pieces of it
    ref, mag, rb, mb = (torch.zeros(D, dtype=torch.float64, device="cuda") for _ in range(4))
    for t in range(0, L, 1 << 15):
        s = slice(t, min(L, t + (1 << 15)))
        gd = g[0, :, s].double()
        term = gd * (x[0, :, s].double() - mean[0, s].double()) * rstd[0, s].double()
        ref += term.sum(1)
        mag += term.abs().sum(1)
        rb += gd.sum(1)
        mb += gd.abs().sum(1)
    # a tile's products (four roundings each), then the tiles in order: fewer than L / 64 + 64 + 40 roundings of what they sum
    assert bool(((dw.double() - ref).abs() <= 2 * (L / 64 + 104) * U * mag).all())
    assert bool(((db.double() - rb).abs() <= 2 * (L / 64 + 104) * U * mb).all())
    # each head's length, in two groups
    del out, dx
    y, rn = P.head_l2norm_fwd(x, groups=2)
    dy = P.head_l2norm_bwd(x, rn, g, groups=2)
    y1, rn1 = P.head_l2norm_fwd(X, groups=2)
    dy1 = P.head_l2norm_bwd(X, rn1, Gd, groups=2)
    assert bool(((rn[..., -n:] - rn1).abs() <= c * rn1).all())
    rr = rn1.repeat_interleave(D // 2, 1)
    a = xf.abs() * rr
    md = rr * (Gd.float().abs() + a * rr * (xf * Gd.float()).abs().view(1, 2, D // 2, n).sum(2).repeat_interleave(D // 2, 1))
    for name, big, one, m in (("y", y, y1, a), ("dy", dy, dy1, md)):
        one = one.float()
        assert bool(((big[..., -n:].float() - one).abs() <= c * 1.02 * m + 2 * HALF * (one.abs() * 1.01 + c * m) + 1e-37).all()), name
