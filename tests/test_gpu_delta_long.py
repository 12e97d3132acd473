"""GPU: the gated delta rule over the longest rows that it takes, against the same rows in two pieces."""
import pytest

from gpu_common import note

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_longest_rows(dtype):
    """2^22 tokens of 128 x 128, cut at a boundary of the decay's sums: outs, states and gradients of the whole row as of its
    pieces, the states and their gradients passed on.  In 32 bits each is off by less than 2e-5 in the 2-norm (what the tests
    against 64 bits hold it to); bf16 results by two roundings of half a step each, at most 2^-8 of themselves, of the result and
    three operands."""
    import torch
    import paper_2408_03865_amd as P
    L, cut, n = 1 << 22, (1 << 21) + 256 * 3, 128
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    note(f"delta rule of {L} tokens, {dtype}")
    gen = torch.Generator(device="cuda").manual_seed(8)

    def unit():
        x = torch.randn((1, 1, n, L), generator=gen, device="cuda")
        return x.mul_(x.square().sum(2, keepdim=True).add_(1e-6).rsqrt_()).to(t)

    q, k = unit(), unit()
    v, do = (torch.randn((1, 1, n, L), generator=gen, device="cuda", dtype=t) for _ in range(2))
    beta = torch.rand((1, 1, L), generator=gen, device="cuda")
    decay = -0.05 * torch.rand((1, 1, L), generator=gen, device="cuda")
    pos = (torch.arange(L, device="cuda", dtype=torch.int32) % 1000003 + 1)[None]
    init, dfin = (torch.randn((1, 1, n, n), generator=gen, device="cuda") for _ in range(2))
    a = (q, k, v, beta, decay, pos)
    out, fin = P.delta_rule_fwd(*a, scale=0.1, initial_state=init, return_final=True)
    g = P.delta_rule_bwd(*a, do, scale=0.1, initial_state=init, dfinal_state=dfin)
    one, two = ([x[..., s].contiguous() for x in (*a, do)] for s in (slice(0, cut), slice(cut, L)))
    o1, mid = P.delta_rule_fwd(*one[:6], scale=0.1, initial_state=init, return_final=True)
    o2, last = P.delta_rule_fwd(*two[:6], scale=0.1, initial_state=mid, return_final=True)
    g2 = P.delta_rule_bwd(*two, scale=0.1, initial_state=mid, dfinal_state=dfin)
    g1 = P.delta_rule_bwd(*one, scale=0.1, initial_state=init, dfinal_state=g2["dinitial_state"])
    exact, rounded = 4e-5, 4e-5 if dtype == "f32" else 2 * 2 * 2.0 ** -8

    def close(x, y, tol, name):
        d, r = (x.float() - y.float()).norm(dtype=torch.float64), y.float().norm(dtype=torch.float64)
        note(f"  {name} {float(d / r):.2g} apart")
        assert bool(y.isfinite().all()) and float(r) > 0 and float(d) <= tol * float(r), name

    close(out[..., :cut], o1, rounded, "out")
    close(out[..., cut:], o2, rounded, "out")
    close(fin, last, exact, "final_state")
    close(g["dinitial_state"], g1["dinitial_state"], exact, "dinitial_state")
    for name in ("dq", "dk", "dv", "dbeta", "ddecay"):
        tol = rounded if name in ("dq", "dk", "dv") else exact
        close(g[name][..., :cut], g1[name], tol, name)
        close(g[name][..., cut:], g2[name], tol, name)
