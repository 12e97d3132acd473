"""GPU: the gated RMSNorm of a group of more than 2^32 elements: the row's end as it is by itself, and dweight."""
import pytest

from gpu_common import note

pytestmark = pytest.mark.gpu

U, HALF = 2.0 ** -24, 2.0 ** -8


@pytest.mark.parametrize("first", [True, False])
def test_more_than_32_bits(first):
    import torch
    import paper_2408_03865_amd as P
    D, L, n = 1040, (1 << 22) + 8, 8200
    assert D * L > 1 << 32
    note(f"gated norm of {D} x {L}, first={first}")
    gen = torch.Generator(device="cuda").manual_seed(5)
    x, z, dout = (torch.empty((1, D, L), device="cuda", dtype=torch.bfloat16) for _ in range(3))
    for t in (x, z, dout):
        for f in range(0, D, 16):
            t[:, f:f + 16] = torch.randn((1, 16, L), generator=gen, device="cuda")
    w = torch.randn(D, generator=gen, device="cuda")
    out, rstd = P.gated_rmsnorm_fwd(x, z, w, gate_first=first)
    dx, dz, dw = P.gated_rmsnorm_bwd(x, z, w, rstd, dout, gate_first=first)
    for a, b in ((0, n), (L - n, L)):
        X, Z, G = (t[..., a:b].contiguous() for t in (x, z, dout))
        o1, r1 = P.gated_rmsnorm_fwd(X, Z, w, gate_first=first)
        dx1, dz1, _ = P.gated_rmsnorm_bwd(X, Z, w, r1, G, gate_first=first)
        # each of the two is off by the bounds of test_gpu_gated_norm: 2 (D + 40) u of the terms' size M and a bf16 rounding
        v, g = X.float(), G.float()
        gate, mdg = Z.float() * torch.sigmoid(Z.float()), torch.sigmoid(Z.float()) * (1 + Z.float().abs())
        v, d = (v * gate, g * w[:, None]) if first else (v, g * w[:, None] * gate)
        da = r1 * (d.abs() + v.abs() * r1 * r1 * (d * v).abs().mean(1, keepdim=True))
        mdx = da * gate.abs() if first else da
        mdz = (da * X.float().abs() if first else (g * w[:, None] * v * r1).abs()) * mdg
        c = 4 * (D + 40) * U
        assert bool(((rstd[..., a:b] - r1).abs() <= c * r1).all())
        for name, big, one, m in (("out", out, o1, o1.float().abs()), ("dx", dx, dx1, mdx), ("dz", dz, dz1, mdz)):
            one = one.float()
            # half a step of a value that differs by c M, twice
            assert bool(((big[..., a:b].float() - one).abs() <= c * 1.02 * m + 2 * HALF * (one.abs() * 1.01 + c * m) + 1e-37).all()), name
    # dweight: 64-bit sums over pieces of the row; a tile's 64 products, then the tiles' in order: fewer than
    # L / 64 + 64 + 40 roundings of what they sum
    ref, mag = torch.zeros(D, dtype=torch.float64, device="cuda"), torch.zeros(D, dtype=torch.float64, device="cuda")
    for t in range(0, L, 1 << 17):
        s = slice(t, min(L, t + (1 << 17)))
        term = dout[0, :, s].double() * x[0, :, s].double() * torch.nn.functional.silu(z[0, :, s].double()) * rstd[0, :, s].double()
        ref += term.sum(1)
        mag += term.abs().sum(1)
    assert bool(((dw.double() - ref).abs() <= 2 * (L / 64 + 104) * U * mag).all())
