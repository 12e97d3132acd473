"""The 64-bit reference of the gated delta rule (delta_reference.py) on the CPU: its gradients against central
differences, its packing against separate rows, its outputs against closed forms."""
import numpy as np
import torch

import delta_reference as R
from linear_reference import positions


def inputs(B, H, G, dk, dv, L, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    k = r(B, G, dk, L)
    return (r(B, G, dk, L), k / k.norm(dim=2, keepdim=True), r(B, H, dv, L), torch.rand((B, H, L), generator=g, dtype=torch.float64) * 2,
            -torch.exp(r(B, H, L)), r(B, H, dv, L), r(B, H, dk, dv), r(B, H, dk, dv))


def test_gradients_against_differences():
    q, k, v, beta, decay, do, init, dfin = inputs(2, 4, 2, 3, 2, 7, 0)
    pos = torch.from_numpy(positions(2, 7, 3, np.random.default_rng(1), True))
    for dec in (decay, decay[0, :, 0].clone()):
        ref, _ = R.reference(q, k, v, beta, dec, pos, 0.7, init, do, dfin)

        def loss():
            r, _ = R.reference(q, k, v, beta, dec, pos, 0.7, init)
            return ((r["out"] * do).sum() + (r["final_state"] * dfin).sum()).item()

        for name, t in (("dq", q), ("dk", k), ("dv", v), ("dbeta", beta), ("ddecay", dec), ("dinitial_state", init)):
            flat = t.view(-1)
            for i in range(0, flat.numel(), 3):
                old = flat[i].item()
                vals = []
                for s in (1e-5, -1e-5):
                    flat[i] = old + s
                    vals.append(loss())
                flat[i] = old
                assert abs((vals[0] - vals[1]) / 2e-5 - ref[name].reshape(-1)[i].item()) < 1e-6, (name, i)


def test_packed_rows_equal_separate_ones():
    q, k, v, beta, decay, do, _, _ = inputs(1, 2, 1, 4, 3, 20, 2)
    lengths = [1, 7, 3, 9]
    pos = torch.cat([torch.arange(n, dtype=torch.int32) for n in lengths])[None]
    (whole, _), t = R.reference(q, k, v, beta, decay, pos, 1.0, dout=do), 0
    for n in lengths:
        s = slice(t, t + n)
        one, _ = R.reference(q[..., s], k[..., s], v[..., s], beta[..., s], decay[..., s], pos[:, s], 1.0, dout=do[..., s])
        for name in ("out", "dq", "dk", "dv", "dbeta", "ddecay"):
            assert torch.allclose(whole[name][..., s], one[name], atol=1e-12), name
        t += n


def test_closed_forms():
    """With beta = 1 and keys of length 1 a state answers its last key with its last value; with one feature and constant
    inputs it nears v / k by the factor 1 - beta k^2 a token."""
    q, k, v, _, _, _, _, _ = inputs(1, 2, 2, 4, 3, 9, 5)
    pos = torch.arange(9, dtype=torch.int32)[None]
    r, _ = R.reference(k, k, v, torch.ones(1, 2, 9, dtype=torch.float64), None, pos, 1.0)
    assert torch.allclose(r["out"], v, atol=1e-12)
    one = torch.ones(1, 1, 1, 9, dtype=torch.float64)
    r, _ = R.reference(one, one * 0.5, one * 3, one[:, :, 0] * 0.8, None, pos, 1.0)
    assert torch.allclose(r["out"][0, 0, 0], 6 * (1 - (1 - 0.8 * 0.25) ** torch.arange(1, 10, dtype=torch.float64)), rtol=1e-12)
