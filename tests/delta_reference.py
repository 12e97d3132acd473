"""The gated delta rule, token by token in 64 bits on the CPU, with its backward pass, and the budgets that rounding
errors are bounded by.

Where beta |k|^2 is in [0, 2] and the decay is no growth, a token's map of the state, a (I - beta k k^T), lengthens no
column, and so does its transpose to the gradient.  What is rounded at a token then stays at most as large as it was, in
the norm of a column, and shrinks by the decays: with s_t = |S'| + (|v| + |e|) |k| what a token adds to its column's
products, the error of the column is at most (some u) times E_t = a_t E_{t-1} + s_t.  The same holds for the
gradient's columns with G_t = a_{t+1} G_{t+1} + |D| + (|dout| |q| + |du| |k|).  In chunks, e = x - H (beta x) has
|H_ts| = |k_t^T (the maps between) k_s| <= |k_t| |k_s| D_ts, so that its sums are inside the same budgets."""
from __future__ import annotations

import torch

from linear_reference import multipliers


def _norm(x):
    return x.square().sum(-2).sqrt()


def reference(q, k, v, beta, decay, pos, scale, initial=None, dout=None, dfinal=None):
    """({out, final_state, and with dout dq, dk, dv, dbeta, ddecay, dinitial_state}, budgets of the same names); the tensors
    as the framework takes them, on the CPU."""
    H, G = v.shape[1], q.shape[1]
    B, L = pos.shape
    dk, dv = q.shape[2], v.shape[2]
    rep = H // G
    qh, kh = (x.double().repeat_interleave(rep, 1).permute(3, 0, 1, 2) for x in (q, k))
    vh, bh = v.double().permute(3, 0, 1, 2), beta.double().permute(2, 0, 1)
    a, cut = multipliers(decay, pos, H)
    a = a.permute(2, 0, 1)
    sc = abs(scale)

    def through(m, S):
        m = m.reshape(m.shape + (1,) * (S.dim() - m.dim()))
        return torch.where(m == 0, torch.zeros_like(S), m * S)

    S = torch.zeros(B, H, dk, dv, dtype=torch.float64) if initial is None else initial.double()
    E = _norm(S)
    out, ob = torch.zeros(L, B, H, dv, dtype=torch.float64), torch.zeros(L, B, H, dv, dtype=torch.float64)
    kept = []
    for t in range(L):
        found = through(a[t], S)
        e = vh[t] - (found * kh[t][..., :, None]).sum(-2)
        u = bh[t][..., None] * e
        S = found + kh[t][..., :, None] * u[..., None, :]
        kn, qn = kh[t].norm(dim=-1)[..., None], qh[t].norm(dim=-1)[..., None]
        E = through(a[t], E) + _norm(found) + (vh[t].abs() + e.abs()) * kn
        out[t] = scale * (S * qh[t][..., :, None]).sum(-2)
        ob[t] = sc * qn * E
        kept.append((found, e, u, S, E))
    perm = lambda x: x.permute(1, 2, 3, 0)  # noqa: E731
    r = {"out": perm(out), "final_state": S}
    m = {"out": perm(ob), "final_state": E[..., None, :].expand_as(S)}
    if dout is None:
        return r, m
    do = dout.double().permute(3, 0, 1, 2)
    D = torch.zeros_like(S) if dfinal is None else dfinal.double()
    N = _norm(D)
    z = lambda n: torch.zeros((L, B, H) + ((n,) if n else ()), dtype=torch.float64)  # noqa: E731
    g = dict(dq=z(dk), dk=z(dk), dv=z(dv), dbeta=z(0), ddecay=z(0))
    gm = {n: torch.zeros_like(x) for n, x in g.items()}
    tail = (kept[-1][3].abs() * D.abs()).sum((-1, -2))
    for t in reversed(range(L)):
        found, e, u, S, E = kept[t]
        kn, qn = kh[t].norm(dim=-1)[..., None], qh[t].norm(dim=-1)[..., None]
        g["dq"][t] = scale * (S * do[t][..., None, :]).sum(-1)
        gm["dq"][t] = (sc * (E * do[t].abs()).sum(-1))[..., None]
        D = D + scale * qh[t][..., :, None] * do[t][..., None, :]
        du = (D * kh[t][..., :, None]).sum(-2)
        N = N + _norm(D) + sc * do[t].abs() * qn + du.abs() * kn
        b1 = bh[t][..., None].abs()
        g["dbeta"][t], gm["dbeta"][t] = (du * e).sum(-1), ((N * e.abs() + du.abs() * E) * kn).sum(-1)
        g["dv"][t], gm["dv"][t] = bh[t][..., None] * du, b1 * N * kn
        F = D - kh[t][..., :, None] * g["dv"][t][..., None, :]
        g["dk"][t] = (D * u[..., None, :]).sum(-1) - (found * g["dv"][t][..., None, :]).sum(-1)
        # u and dv are off by their budgets, and meet D and S
        gm["dk"][t] = ((N * u.abs() + b1 * E * _norm(D)) + (E * g["dv"][t].abs() + _norm(found) * b1 * N * kn)).sum(-1)[..., None]
        g["ddecay"][t] = (F * found).sum((-1, -2))
        # summed from out . dout and v . dv of the tokens that follow, and the states' product
        tail = tail + sc * (E * qn * do[t].abs()).sum(-1) + (vh[t].abs() * b1 * N * kn).sum(-1)
        gm["ddecay"][t] = tail + (E * N).sum(-1)
        tail = torch.where(cut[..., t], torch.zeros_like(tail), tail)
        D, N = through(a[t], F), through(a[t], N)
    group = lambda x: perm(x).unflatten(1, (G, rep)).sum(2)  # noqa: E731
    for src, to in ((g, r), (gm, m)):
        to.update(dq=group(src["dq"]), dk=group(src["dk"]), dv=perm(src["dv"]), dbeta=src["dbeta"].permute(1, 2, 0))
        if decay is not None:
            dg = torch.where(cut, torch.zeros((), dtype=torch.float64), src["ddecay"].permute(1, 2, 0))
            to["ddecay"] = dg.sum((0, 2)) if decay.dim() == 1 else dg
    r["dinitial_state"], m["dinitial_state"] = D, N[..., None, :].expand_as(D)
    return r, m
