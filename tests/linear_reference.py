"""Linear attention with a decay for each head, token by token in 64 bits on the CPU, with its backward
pass, and the same sums over the terms' absolute values, which rounding errors are bounded by."""
from __future__ import annotations

import numpy as np
import torch

CUT = -104.0


def positions(batch, seqlen, mean, rng, continued=False):
    """Packed rows of sequences of about `mean` tokens, lengths of 1 among them."""
    pos = np.zeros((batch, seqlen), np.int32)
    for b in range(batch):
        t, first = 0, continued
        while t < seqlen:
            n = min(seqlen - t, 1 if rng.random() < 0.1 else int(rng.integers(1, 2 * mean + 1)))
            pos[b, t:t + n] = np.arange(n) + (7 if first else 0)
            t, first = t + n, False
    return pos


def multipliers(decay, pos, heads):
    """(batch, heads, seqlen) doubles: exp(decay), 0 at a start."""
    B, L = pos.shape
    g = torch.zeros(B, heads, L, dtype=torch.float64) if decay is None else \
        (decay[None, :, None] if decay.dim() == 1 else decay).double().expand(B, heads, L)
    cut = (pos == 0)[:, None].expand(B, heads, L) | (g <= CUT)
    return torch.where(cut, torch.zeros_like(g), torch.exp(g)), cut


def walk(a, x, y, z, entry, rev=False):
    """S = a_t S + y_t z_t^T, out_t = S^T x_t from `entry`: (out, the last state)."""
    B, H, L = a.shape
    S = torch.zeros(B, H, y.shape[2], z.shape[2], dtype=torch.float64) if entry is None else entry.double().clone()
    out = torch.empty(B, H, z.shape[2], L, dtype=torch.float64)
    for t in (reversed(range(L)) if rev else range(L)):
        m = a[:, :, t, None, None]
        S = torch.where(m == 0, torch.zeros_like(S), m * S) + y[..., t, None] * z[..., None, :, t]
        out[..., t] = (S * x[..., t, None]).sum(-2)
    return out, S


def reference(q, k, v, decay, pos, scale, initial=None, dout=None, dfinal=None, absolute=False):
    """{out, final_state}, with dout also {dq, dk, dv, ddecay, dinitial_state}; the tensors as the
    framework takes them, on the CPU.  absolute: every term by its absolute value."""
    f = (lambda t: None if t is None else t.double().abs()) if absolute else (lambda t: None if t is None else t.double())
    H, G = v.shape[1], q.shape[1]
    s = abs(scale) if absolute else scale
    qh, kh = f(q).repeat_interleave(H // G, 1) * s, f(k).repeat_interleave(H // G, 1)
    vh, init, do, dfin = f(v), f(initial), f(dout), f(dfinal)
    a, cut = multipliers(decay, pos, H)
    out, fin = walk(a, qh, kh, vh, init)
    r = {"out": out, "final_state": fin}
    if dout is None:
        return r
    T = lambda t: None if t is None else t.transpose(-1, -2)  # noqa: E731
    dq, _ = walk(a, do, vh, kh, T(init))
    nxt = torch.cat([a[..., 1:], torch.ones_like(a[..., :1])], -1)
    dk, _ = walk(nxt, vh, do, qh, T(dfin), rev=True)
    dv, dS = walk(nxt, kh, qh, do, dfin, rev=True)
    group = lambda t: t.unflatten(1, (G, H // G)).sum(2)  # noqa: E731
    r.update(dq=group(dq) * s, dk=group(dk), dv=dv, dinitial_state=dS * a[..., :1, None])
    if decay is not None:
        # a_t <dS_t, S_{t-1}>, by the definition
        B, L = pos.shape
        states, S = [], torch.zeros_like(fin) if init is None else init.clone()
        for t in range(L):
            states.append(S)
            m = a[:, :, t, None, None]
            S = torch.where(m == 0, torch.zeros_like(S), m * S) + kh[..., t, None] * vh[..., None, :, t]
        dg = torch.zeros(B, H, L, dtype=torch.float64)
        D = torch.zeros_like(fin) if dfin is None else dfin.clone()
        for t in reversed(range(L)):
            m = nxt[:, :, t, None, None]
            D = torch.where(m == 0, torch.zeros_like(D), m * D) + qh[..., t, None] * do[..., None, :, t]
            dg[..., t] = a[..., t] * (D * states[t]).sum((-1, -2))
        if absolute:
            # the kernels sum q dq + k dk over the tokens that follow in the sequence
            e = (qh * dq).sum(2) + (kh * dk).sum(2)
            tail = torch.zeros(B, H, dtype=torch.float64) if dfin is None else (fin * dfin).sum((-1, -2))
            for t in reversed(range(L)):
                tail = tail + e[..., t]
                dg[..., t] = tail
                tail = torch.where(cut[..., t], torch.zeros_like(tail), tail)
        dg = torch.where(cut, torch.zeros_like(dg), dg)
        r["ddecay"] = dg.sum((0, 2)) if decay.dim() == 1 else dg
    return r
