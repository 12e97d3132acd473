"""Torch wrappers of include/packmamba_linear.h: packed linear attention with a decay for each head (in
chunks, and token by token) and the gated RMSNorm after it.

    out, state = linear_attention_fwd(q, k, v, decay, position_indices, scale=s, return_final=True)
    grads = linear_attention_bwd(q, k, v, decay, position_indices, dout, scale=s)
    out = linear_attention_step(q, k, v, decay, state, scale=s)          # one token, state in place
    y, rstd = gated_rmsnorm_fwd(x, z, weight, groups=heads)
    dx, dz, dweight = gated_rmsnorm_bwd(x, z, weight, rstd, dy, groups=heads)

S_t = exp(decay_t) S_{t-1} + k_t v_t^T (nothing of S_{t-1} where position_indices is 0) and
out_t = scale S_t^T q_t, per batch row and head; q and k are shared by heads / groups heads.
Tensors are contiguous, on one GPU; what does not fit raises TypeError, ValueError or, from the
library's own checks (alignment, limits, the workspace's size), PackMambaError before anything is
launched.
"""
from __future__ import annotations

from typing import Dict

from . import _code, _empty_out, _lib, _p, _size, _stream, _torch, load

MAX_HEAD = 128


def _check(device, tensors):
    """Each (name, tensor or None, shape, dtype): contiguous, of that shape and type, on `device`."""
    for name, t, shape, dtype in tensors:
        if t is None:
            continue
        if t.dtype != dtype:
            raise TypeError(f"{name} is {t.dtype}, not {dtype}")
        if t.shape != shape:
            raise ValueError(f"{name} has shape {tuple(t.shape)}, not {shape}")
        if t.device != device:
            raise ValueError(f"{name} is on {t.device}, not on {device}")
        if not t.is_contiguous():
            raise ValueError(f"{name} is not contiguous")


def _on_gpu(name, t):
    if not t.is_cuda:
        raise ValueError(f"{name} is on {t.device}, not on a GPU")
    return t.device


def _call(device, name, *args):
    """The library's call, with `device` current; its status checked."""
    torch = _torch()
    fn = getattr(load(), name)
    if torch.cuda.current_device() == device.index:
        st = fn(*args)
    else:
        with torch.cuda.device(device):
            st = fn(*args)
    if st:
        _lib.check(name, st)


def _workspace(workspace, need, device):
    """The caller's workspace, or one of `need` bytes; None where nothing is needed."""
    torch = _torch()
    if workspace is None:
        return torch.empty(need, dtype=torch.uint8, device=device) if need else None
    if workspace.device != device or workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise ValueError("workspace is a contiguous uint8 tensor on the inputs' GPU")
    return workspace


def _bytes(ws):
    return 0 if ws is None else ws.numel()


def _dims(q, v, nd):
    if q.dim() != nd or v.dim() != nd:
        raise ValueError(f"q and v have {nd} dimensions, not {q.dim()} and {v.dim()}")
    (Nb, G, dk), (H, dv) = q.shape[:3], v.shape[1:3]
    L = q.shape[3] if nd == 4 else None
    if G < 1 or H % G:
        raise ValueError(f"{H} heads are no multiple of {G} groups")
    if not (1 <= dk <= MAX_HEAD and 1 <= dv <= MAX_HEAD):
        raise ValueError(f"head sizes {dk} and {dv} are not in 1 .. {MAX_HEAD}")
    if Nb < 1 or H < 1 or (nd == 4 and L < 1):
        raise ValueError("empty batch, heads or rows")
    return Nb, H, G, dk, dv, L


def _decay_shape(decay, Nb, H, L):
    """The decay's shape, and whether it is one for each token."""
    if decay is None or decay.dim() == 1:
        return (H,), False
    return ((Nb, H) if L is None else (Nb, H, L)), True


def _attention_inputs(q, k, v, decay, position_indices, initial_state, extra=()):
    torch = _torch()
    Nb, H, G, dk, dv, L = _dims(q, v, 4)
    device = _on_gpu("q", q)
    shape, per_token = _decay_shape(decay, Nb, H, L)
    _check(device, [("q", q, (Nb, G, dk, L), q.dtype), ("k", k, (Nb, G, dk, L), q.dtype), ("v", v, (Nb, H, dv, L), q.dtype),
                    ("decay", decay, shape, torch.float32), ("position_indices", position_indices, (Nb, L), torch.int32),
                    ("initial_state", initial_state, (Nb, H, dk, dv), torch.float32)])
    return (Nb, H, G, dk, dv, L), per_token, device


def linear_attention_fwd(q, k, v, decay, position_indices, scale: float = 1.0, out_f32: bool = False,
                         initial_state=None, return_final: bool = False, workspace=None):
    """out (batch, heads, dv, seqlen), and with return_final the state after each row, (batch, heads,
    dk, dv) fp32.  q, k (batch, groups, dk, seqlen), v (batch, heads, dv, seqlen); decay: log decays,
    fp32, (batch, heads, seqlen), (heads), or None; position_indices (batch, seqlen) int32;
    initial_state as the final one.  out_f32: for bf16 inputs, out before its last rounding."""
    torch = _torch()
    shape, per_token, device = _attention_inputs(q, k, v, decay, position_indices, initial_state)
    Nb, H, G, dk, dv, L = shape
    code = _code(q, out_f32)
    out = _empty_out(v, out_f32)
    fin = torch.empty((Nb, H, dk, dv), dtype=torch.float32, device=device) if return_final else None
    ws = _workspace(workspace, _size(load(), "packmamba_linear_attention_fwd_workspace_size", *shape), device)
    _call(device, "packmamba_linear_attention_fwd", _p(q), _p(k), _p(v), _p(decay), _p(position_indices), _p(initial_state),
          float(scale), _p(out), _p(fin), _p(ws), _bytes(ws), *shape, int(per_token), code, _stream(q))
    return (out, fin) if return_final else out


def linear_attention_bwd(q, k, v, decay, position_indices, dout, scale: float = 1.0, out_f32: bool = False,
                         initial_state=None, dfinal_state=None, decay_grad: bool = True,
                         workspace=None) -> Dict[str, object]:
    """The gradients of linear_attention_fwd: dq, dk, dv (in the inputs' type, or fp32), ddecay (decay's
    shape, fp32; None without a decay or decay_grad) and dinitial_state (None without an initial state).
    dout as v; dfinal_state: the gradient of the final state, or None."""
    torch = _torch()
    shape, per_token, device = _attention_inputs(q, k, v, decay, position_indices, initial_state)
    Nb, H, G, dk, dv, L = shape
    _check(device, [("dout", dout, (Nb, H, dv, L), q.dtype),
                    ("dfinal_state", dfinal_state, (Nb, H, dk, dv), torch.float32)])
    code = _code(q, out_f32)
    g = {"dq": _empty_out(q, out_f32), "dk": _empty_out(k, out_f32), "dv": _empty_out(v, out_f32),
         "ddecay": torch.empty_like(decay) if decay is not None and decay_grad else None,
         "dinitial_state": torch.empty_like(initial_state) if initial_state is not None else None}
    ws = _workspace(workspace, _size(load(), "packmamba_linear_attention_bwd_workspace_size", *shape), device)
    _call(device, "packmamba_linear_attention_bwd", _p(q), _p(k), _p(v), _p(decay), _p(position_indices), _p(initial_state),
          float(scale), _p(dout), _p(dfinal_state), _p(g["dq"]), _p(g["dk"]), _p(g["dv"]), _p(g["ddecay"]),
          _p(g["dinitial_state"]), _p(ws), _bytes(ws), *shape, int(per_token), code, _stream(q))
    return g


def linear_attention_step(q, k, v, decay, state, position_indices=None, scale: float = 1.0, out_f32: bool = False):
    """One token of each sequence: out (batch, heads, dv); state (batch, heads, dk, dv) fp32 is updated in
    place.  q, k (batch, groups, dk), v (batch, heads, dv); decay (batch, heads) or (heads), or None;
    position_indices (batch) int32: 0 starts a sequence, a negative index marks an idle row (its state
    stays, its out is 0); None: every sequence goes on."""
    torch = _torch()
    Nb, H, G, dk, dv, _ = _dims(q, v, 3)
    device = _on_gpu("q", q)
    shape, per_token = _decay_shape(decay, Nb, H, None)
    _check(device, [("q", q, (Nb, G, dk), q.dtype), ("k", k, (Nb, G, dk), q.dtype), ("v", v, (Nb, H, dv), q.dtype),
                    ("decay", decay, shape, torch.float32), ("state", state, (Nb, H, dk, dv), torch.float32),
                    ("position_indices", position_indices, (Nb,), torch.int32)])
    code = _code(q, out_f32)
    out = _empty_out(v, out_f32)
    _call(device, "packmamba_linear_attention_step", _p(q), _p(k), _p(v), _p(decay), _p(position_indices), _p(state),
          float(scale), _p(out), Nb, H, G, dk, dv, int(per_token), code, _stream(q))
    return out


def _norm_inputs(x, z, weight, groups):
    torch = _torch()
    if x.dim() != 3:
        raise ValueError(f"x has 3 dimensions, not {x.dim()}")
    Nb, Dn, L = x.shape
    if groups < 1 or Dn % groups:
        raise ValueError(f"{Dn} features are no multiple of {groups} groups")
    if Nb < 1 or Dn < 1 or L < 1:
        raise ValueError("empty batch, features or rows")
    device = _on_gpu("x", x)
    _check(device, [("x", x, (Nb, Dn, L), x.dtype), ("z", z, (Nb, Dn, L), x.dtype), ("weight", weight, (Dn,), torch.float32)])
    return Nb, Dn, L, device


def gated_rmsnorm_fwd(x, z, weight, groups: int = 1, eps: float = 1e-5, gate_first: bool = True, out_f32: bool = False):
    """(out, rstd): with gate = z sigmoid(z), the RMSNorm over each of `groups` groups of x's features of
    x gate (gate_first), or of x, multiplied with gate afterwards; weight (dim) fp32, rstd (batch, groups,
    seqlen) fp32 for the backward."""
    torch = _torch()
    Nb, Dn, L, device = _norm_inputs(x, z, weight, groups)
    code = _code(x, out_f32)
    out = _empty_out(x, out_f32)
    rstd = torch.empty((Nb, groups, L), dtype=torch.float32, device=device)
    _call(device, "packmamba_gated_rmsnorm_fwd", _p(x), _p(z), _p(weight), float(eps), _p(out), _p(rstd), Nb, Dn, L, groups,
          int(gate_first), code, _stream(x))
    return out, rstd


def gated_rmsnorm_bwd(x, z, weight, rstd, dout, groups: int = 1, gate_first: bool = True, workspace=None,
                      out_f32: bool = False):
    """(dx, dz, dweight) of gated_rmsnorm_fwd, from its inputs and its rstd."""
    torch = _torch()
    Nb, Dn, L, device = _norm_inputs(x, z, weight, groups)
    _check(device, [("rstd", rstd, (Nb, groups, L), torch.float32), ("dout", dout, (Nb, Dn, L), x.dtype)])
    code = _code(x, out_f32)
    dx, dz, dw = _empty_out(x, out_f32), _empty_out(z, out_f32), torch.empty_like(weight)
    ws = _workspace(workspace, _size(load(), "packmamba_gated_rmsnorm_bwd_workspace_size", Nb, Dn, L, groups), device)
    _call(device, "packmamba_gated_rmsnorm_bwd", _p(x), _p(z), _p(weight), _p(rstd), _p(dout), _p(dx), _p(dz), _p(dw),
          _p(ws), _bytes(ws), Nb, Dn, L, groups, int(gate_first), code, _stream(x))
    return dx, dz, dw
