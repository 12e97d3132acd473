"""GPU: the norms of more features than a block keeps in registers, and their results in 32 bits of bf16 inputs.  Bounds as in
test_gpu_norms."""
import pytest

from gpu_common import note
from test_gpu_norms import data, layer, within

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 4097, 1), (2, 8192, 1), (2, 8193, 1), (5, 12001, 1), (1, 20000, 1), (2, 4099, 9), (1, 8200, 70)],
                         ids=lambda s: "x".join(map(str, s)))
def test_layernorm_of_many_features(shape, dtype):
    """One token: from 4096 features on in 32 bits and 8192 in bf16 the rest is read again."""
    for kind in ("plain", "offset", "first", "constant", "zero"):
        layer(shape, dtype, kind)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(2, 1, 4097, 1), (2, 3, 8193, 1), (1, 1, 20000, 1), (1, 2, 4100, 3), (1, 1, 9000, 66)],
                         ids=lambda s: "x".join(map(str, s)))
def test_length_of_many_features(shape, dtype):
    import torch
    import paper_2408_03865_amd as P
    B, G, n, L = shape
    x, g, _, _, _ = data((B, G * n, L), dtype, sum(shape))
    note(f"length of {shape} {dtype}")
    xd, gd = x.double().view(B, G, n, L), g.double().view(B, G, n, L)
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    r = (xd.square().sum(2) + 1e-6).rsqrt()
    dr = ((n + 3) / 2 + 4) * U
    out, gr = P.head_l2norm_fwd(x.cuda(), groups=G)
    within(gr, r, dr * r, "rnorm")
    ref = (xd * r[:, :, None]).view(x.shape)
    within(out, ref, (dr + 2 * U + half) * ref.abs(), "out")
    rf = r.float()
    r = rf.double()[:, :, None]
    s, sa = (xd * gd).sum(2, keepdim=True), (xd * gd).abs().sum(2, keepdim=True)
    ref = (r * (gd - xd * r * r * s)).view(x.shape)
    tol = (r * (4 * U * gd.abs() + (n + 8) * U * (xd.abs() * r * r * sa))).view(x.shape)
    within(P.head_l2norm_bwd(x.cuda(), rf.cuda(), g.cuda(), groups=G), ref, tol + half * ref.abs(), "dx")


@pytest.mark.parametrize("shape", [(3, 70, 1), (2, 64, 5), (2, 700, 130), (4, 1000, 1001), (9, 256, 2051)], ids=lambda s: "x".join(map(str, s)))
def test_results_in_32_bits(shape):
    """out_f32: what the bf16 results are rounded from, to the bit, and its own sums the same."""
    import torch
    import paper_2408_03865_amd as P
    x, g, res, w, b = (t.cuda() for t in data(shape, "bf16", sum(shape)))
    note(f"norms in 32 bits of {shape}")
    y, r = P.head_l2norm_fwd(x, groups=2)
    y32, r32 = P.head_l2norm_fwd(x, groups=2, out_f32=True)
    assert y32.dtype == torch.float32 and torch.equal(y32.bfloat16(), y) and torch.equal(r32, r)
    _, mean, rstd = P.layernorm_fwd(x, w, b)
    for dres in (None, res):
        narrow = P.layernorm_bwd(x, w, mean, rstd, g, dresidual=dres)
        wide = P.layernorm_bwd(x, w, mean, rstd, g, dresidual=dres, out_f32=True)
        assert wide[0].dtype == torch.float32 and torch.equal(wide[0].bfloat16(), narrow[0])
        assert torch.equal(wide[1], narrow[1]) and torch.equal(wide[2], narrow[2])
