"""Torch wrappers of include/packmamba_delta.h: the packed gated delta rule (in chunks, and token by token).

    out, state = delta_rule_fwd(q, k, v, beta, decay, position_indices, scale=s, return_final=True)
    grads = delta_rule_bwd(q, k, v, beta, decay, position_indices, dout, scale=s)
    out = delta_rule_step(q, k, v, beta, decay, state, scale=s)          # one token, state in place

With S' = exp(decay_t) S_{t-1} (nothing of S_{t-1} where position_indices is 0), u_t = beta_t (v_t - S'^T k_t):
S_t = S' + k_t u_t^T and out_t = scale S_t^T q_t, per batch row and head; q and k are shared by heads / groups
heads.  Tensors are contiguous, on one GPU; what does not fit raises TypeError, ValueError or, from the library's
own checks (alignment, limits, the workspace's size), PackMambaError before anything is launched.
"""
from __future__ import annotations

from typing import Dict

from . import _code, _empty_out, _p, _size, _stream, _torch, load
from .linear import _bytes, _call, _check, _decay_shape, _dims, _on_gpu, _workspace


def _inputs(q, k, v, beta, decay, position_indices, initial_state):
    torch = _torch()
    Nb, H, G, dk, dv, L = _dims(q, v, 4)
    device = _on_gpu("q", q)
    shape, per_token = _decay_shape(decay, Nb, H, L)
    _check(device, [("q", q, (Nb, G, dk, L), q.dtype), ("k", k, (Nb, G, dk, L), q.dtype), ("v", v, (Nb, H, dv, L), q.dtype),
                    ("beta", beta, (Nb, H, L), torch.float32), ("decay", decay, shape, torch.float32),
                    ("position_indices", position_indices, (Nb, L), torch.int32),
                    ("initial_state", initial_state, (Nb, H, dk, dv), torch.float32)])
    return (Nb, H, G, dk, dv, L), per_token, device


def delta_rule_fwd(q, k, v, beta, decay, position_indices, scale: float = 1.0, out_f32: bool = False,
                   initial_state=None, return_final: bool = False, workspace=None):
    """out (batch, heads, dv, seqlen), and with return_final the state after each row, (batch, heads,
    dk, dv) fp32.  q, k (batch, groups, dk, seqlen), v (batch, heads, dv, seqlen); beta (batch, heads, seqlen)
    fp32; decay: log decays, fp32, (batch, heads, seqlen), (heads), or None; position_indices (batch, seqlen)
    int32; initial_state as the final one.  out_f32: for bf16 inputs, out before its last rounding."""
    torch = _torch()
    shape, per_token, device = _inputs(q, k, v, beta, decay, position_indices, initial_state)
    Nb, H, G, dk, dv, L = shape
    code = _code(q, out_f32)
    out = _empty_out(v, out_f32)
    fin = torch.empty((Nb, H, dk, dv), dtype=torch.float32, device=device) if return_final else None
    ws = _workspace(workspace, _size(load(), "packmamba_delta_rule_fwd_workspace_size", *shape), device)
    _call(device, "packmamba_delta_rule_fwd", _p(q), _p(k), _p(v), _p(beta), _p(decay), _p(position_indices), _p(initial_state),
          float(scale), _p(out), _p(fin), _p(ws), _bytes(ws), *shape, int(per_token), code, _stream(q))
    return (out, fin) if return_final else out


def delta_rule_bwd(q, k, v, beta, decay, position_indices, dout, scale: float = 1.0, out_f32: bool = False,
                   initial_state=None, dfinal_state=None, decay_grad: bool = True,
                   workspace=None) -> Dict[str, object]:
    """The gradients of delta_rule_fwd: dq, dk, dv (in the inputs' type, or fp32), dbeta (fp32), ddecay (decay's
    shape, fp32; None without a decay or decay_grad) and dinitial_state (None without an initial state).
    dout as v; dfinal_state: the gradient of the final state, or None."""
    torch = _torch()
    shape, per_token, device = _inputs(q, k, v, beta, decay, position_indices, initial_state)
    Nb, H, G, dk, dv, L = shape
    _check(device, [("dout", dout, (Nb, H, dv, L), q.dtype),
                    ("dfinal_state", dfinal_state, (Nb, H, dk, dv), torch.float32)])
    code = _code(q, out_f32)
    g = {"dq": _empty_out(q, out_f32), "dk": _empty_out(k, out_f32), "dv": _empty_out(v, out_f32),
         "dbeta": torch.empty_like(beta),
         "ddecay": torch.empty_like(decay) if decay is not None and decay_grad else None,
         "dinitial_state": torch.empty_like(initial_state) if initial_state is not None else None}
    ws = _workspace(workspace, _size(load(), "packmamba_delta_rule_bwd_workspace_size", *shape, code), device)
    _call(device, "packmamba_delta_rule_bwd", _p(q), _p(k), _p(v), _p(beta), _p(decay), _p(position_indices), _p(initial_state),
          float(scale), _p(dout), _p(dfinal_state), _p(g["dq"]), _p(g["dk"]), _p(g["dv"]), _p(g["dbeta"]), _p(g["ddecay"]),
          _p(g["dinitial_state"]), _p(ws), _bytes(ws), *shape, int(per_token), code, _stream(q))
    return g


def delta_rule_step(q, k, v, beta, decay, state, position_indices=None, scale: float = 1.0, out_f32: bool = False):
    """One token of each sequence: out (batch, heads, dv); state (batch, heads, dk, dv) fp32 is updated in
    place.  q, k (batch, groups, dk), v (batch, heads, dv), beta (batch, heads) fp32; decay (batch, heads) or
    (heads), or None; position_indices (batch) int32: 0 starts a sequence, a negative index marks an idle row (its
    state stays, its out is 0); None: every sequence goes on."""
    torch = _torch()
    Nb, H, G, dk, dv, _ = _dims(q, v, 3)
    device = _on_gpu("q", q)
    shape, per_token = _decay_shape(decay, Nb, H, None)
    _check(device, [("q", q, (Nb, G, dk), q.dtype), ("k", k, (Nb, G, dk), q.dtype), ("v", v, (Nb, H, dv), q.dtype),
                    ("beta", beta, (Nb, H), torch.float32), ("decay", decay, shape, torch.float32),
                    ("state", state, (Nb, H, dk, dv), torch.float32), ("position_indices", position_indices, (Nb,), torch.int32)])
    code = _code(q, out_f32)
    out = _empty_out(v, out_f32)
    _call(device, "packmamba_delta_rule_step", _p(q), _p(k), _p(v), _p(beta), _p(decay), _p(position_indices), _p(state),
          float(scale), _p(out), Nb, H, G, dk, dv, int(per_token), code, _stream(q))
    return out
