"""The 64-bit reference of linear attention (linear_reference.py) on the CPU: its gradients against central
differences, its packing against separate rows, its outputs against a closed form."""
import numpy as np
import torch

import linear_reference as R


def inputs(B, H, G, dk, dv, L, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    return r(B, G, dk, L), r(B, G, dk, L), r(B, H, dv, L), -torch.exp(r(B, H, L)), r(B, H, dv, L), r(B, H, dk, dv), r(B, H, dk, dv)


def test_gradients_against_differences():
    q, k, v, decay, do, init, dfin = inputs(2, 4, 2, 3, 2, 7, 0)
    pos = torch.from_numpy(R.positions(2, 7, 3, np.random.default_rng(1), True))
    for dec in (decay, decay[0, :, 0].clone()):
        ref = R.reference(q, k, v, dec, pos, 0.7, init, do, dfin)

        def loss():
            r = R.reference(q, k, v, dec, pos, 0.7, init)
            return ((r["out"] * do).sum() + (r["final_state"] * dfin).sum()).item()

        for name, t in (("dq", q), ("dk", k), ("dv", v), ("ddecay", dec), ("dinitial_state", init)):
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
    q, k, v, decay, do, _, _ = inputs(1, 2, 1, 4, 3, 20, 2)
    lengths = [1, 7, 3, 9]
    pos = torch.cat([torch.arange(n, dtype=torch.int32) for n in lengths])[None]
    whole, t = R.reference(q, k, v, decay, pos, 1.0, dout=do), 0
    for n in lengths:
        s = slice(t, t + n)
        one = R.reference(q[..., s], k[..., s], v[..., s], decay[..., s], pos[:, s], 1.0, dout=do[..., s])
        for name in ("out", "dq", "dk", "dv", "ddecay"):
            assert torch.allclose(whole[name][..., s], one[name], atol=1e-12), name
        t += n


def test_closed_form():
    """Constant q, k, v and decay: a geometric sum."""
    L, a = 12, 0.8
    one = torch.ones(1, 1, 1, L, dtype=torch.float64)
    r = R.reference(one * 2, one * 3, one * 5, torch.full((1,), float(np.log(a)), dtype=torch.float64), torch.arange(L, dtype=torch.int32)[None], 0.5)
    want = 15 * (1 - a ** torch.arange(1, L + 1, dtype=torch.float64)) / (1 - a)
    assert torch.allclose(r["out"][0, 0, 0], want, rtol=1e-12)
