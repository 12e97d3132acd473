"""Torch wrappers of the norms in include/packmamba_delta.h: each head's features divided by their length, and the layer
norm over all features, of (batch, dim, seqlen) activations at every token.

    y, rnorm = head_l2norm_fwd(x, groups=heads)
    dx = head_l2norm_bwd(x, rnorm, dy, groups=heads)
    y, mean, rstd = layernorm_fwd(x, weight, bias)
    dx, dweight, dbias = layernorm_bwd(x, weight, mean, rstd, dy)

Tensors are contiguous, on one GPU; what does not fit raises TypeError, ValueError or, from the library's own checks
(alignment, limits, the workspace's size), PackMambaError before anything is launched.
"""
from __future__ import annotations

from . import _code, _empty_out, _p, _size, _stream, _torch, load
from .linear import _bytes, _call, _check, _on_gpu, _workspace


def _inputs(x, groups):
    if x.dim() != 3:
        raise ValueError(f"x has 3 dimensions, not {x.dim()}")
    Nb, Dn, L = x.shape
    if groups < 1 or Dn % groups:
        raise ValueError(f"{Dn} features are no multiple of {groups} groups")
    if Nb < 1 or Dn < 1 or L < 1:
        raise ValueError("empty batch, features or rows")
    device = _on_gpu("x", x)
    _check(device, [("x", x, (Nb, Dn, L), x.dtype)])
    return Nb, Dn, L, device


def head_l2norm_fwd(x, groups: int = 1, eps: float = 1e-6, out_f32: bool = False):
    """(out, rnorm): x divided by the length of each of `groups` groups of its features, rnorm = 1 / sqrt(sum of
    squares + eps), (batch, groups, seqlen) fp32 for the backward."""
    torch = _torch()
    Nb, Dn, L, device = _inputs(x, groups)
    code = _code(x, out_f32)
    out = _empty_out(x, out_f32)
    rnorm = torch.empty((Nb, groups, L), dtype=torch.float32, device=device)
    _call(device, "packmamba_head_l2norm_fwd", _p(x), float(eps), _p(out), _p(rnorm), Nb, Dn, L, groups, code, _stream(x))
    return out, rnorm


def head_l2norm_bwd(x, rnorm, dout, groups: int = 1, out_f32: bool = False):
    """dx of head_l2norm_fwd, from its input and its rnorm."""
    torch = _torch()
    Nb, Dn, L, device = _inputs(x, groups)
    _check(device, [("rnorm", rnorm, (Nb, groups, L), torch.float32), ("dout", dout, (Nb, Dn, L), x.dtype)])
    code = _code(x, out_f32)
    dx = _empty_out(x, out_f32)
    _call(device, "packmamba_head_l2norm_bwd", _p(x), _p(rnorm), _p(dout), _p(dx), Nb, Dn, L, groups, code, _stream(x))
    return dx


def layernorm_fwd(x, weight, bias=None, eps: float = 1e-5, out_f32: bool = False):
    """(out, mean, rstd): the layer norm over the feature axis of x (batch, dim, seqlen); weight, bias (dim) fp32,
    mean, rstd (batch, seqlen) fp32 for the backward."""
    torch = _torch()
    Nb, Dn, L, device = _inputs(x, 1)
    _check(device, [("weight", weight, (Dn,), torch.float32), ("bias", bias, (Dn,), torch.float32)])
    code = _code(x, out_f32)
    out = _empty_out(x, out_f32)
    mean = torch.empty((Nb, L), dtype=torch.float32, device=device)
    rstd = torch.empty_like(mean)
    _call(device, "packmamba_layernorm_fwd", _p(x), _p(weight), _p(bias), float(eps), _p(out), _p(mean), _p(rstd), Nb, Dn, L,
          code, _stream(x))
    return out, mean, rstd


def layernorm_bwd(x, weight, mean, rstd, dout, dresidual=None, workspace=None, out_f32: bool = False, bias_grad: bool = True):
    """(dx, dweight, dbias) of layernorm_fwd, from its inputs, its mean and its rstd; dresidual, if given, is added to dx (a
    residual connection); dbias is None without bias_grad."""
    torch = _torch()
    Nb, Dn, L, device = _inputs(x, 1)
    _check(device, [("weight", weight, (Dn,), torch.float32), ("mean", mean, (Nb, L), torch.float32),
                    ("rstd", rstd, (Nb, L), torch.float32), ("dout", dout, (Nb, Dn, L), x.dtype),
                    ("dresidual", dresidual, (Nb, Dn, L), x.dtype)])
    code = _code(x, out_f32)
    dx, dw, db = _empty_out(x, out_f32), torch.empty_like(weight), torch.empty_like(weight) if bias_grad else None
    ws = _workspace(workspace, _size(load(), "packmamba_layernorm_bwd_workspace_size", Nb, Dn, L, code), device)
    _call(device, "packmamba_layernorm_bwd", _p(x), _p(weight), _p(mean), _p(rstd), _p(dout), _p(dresidual), _p(dx), _p(dw),
          _p(db), _p(ws), _bytes(ws), Nb, Dn, L, code, _stream(x))
    return dx, dw, db
