"""The C ABI of packmamba_delta.h on the CPU: its symbols, sizes and argument errors before anything is
enqueued, and the wrappers' refusals."""
import os
import re

import pytest

from test_abi import _gpu_visible, _lib
from test_linear_abi import C_TYPES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "packmamba_delta.h")


def test_header_and_binding_agree():
    from paper_2408_03865_amd import _lib as L
    text = re.sub(r"/\*.*?\*/", " ", open(HEADER).read(), flags=re.S)
    decls = {m.group(2): (m.group(1), [p.strip() for p in m.group(3).split(",")])
             for m in re.finditer(r"\b(int|size_t) (packmamba_\w+)\s*\(([^;{]*?)\)\s*;", text)}
    assert set(decls) == set(L.DELTA_EXPORTS)
    lib = _lib()
    for name, (ret, params) in decls.items():
        args, size = L.DELTA_EXPORTS[name]
        assert hasattr(lib, name) and (ret == "size_t") == size
        assert len(args) == len(params), name
        for code, p in zip(args, params):
            assert ("*" in p) == (code == "p") and re.search(C_TYPES[code], p), (name, p)


def test_sizes():
    lib = _lib()
    fwd, bwd = lib.packmamba_delta_rule_fwd_workspace_size, lib.packmamba_delta_rule_bwd_workspace_size
    two = 2 * 10 * 64 * 4 * 4                                   # a chunk's two products: 10 tiles of 64 x 4 values
    assert fwd(8, 64, 8, 128, 64, 4096) >= 8 * 64 * 64 * (two + 448 * 4)
    assert fwd(1, 4, 4, 64, 64, 64 * 64) >= 4 * 64 * (two + 448 * 4) + 4 * 3 * (2 * 64 * 64 + 1) * 4        # segments
    assert bwd(2, 6, 2, 128, 64, 300, 0) >= 2 * 6 * 5 * (two + 2 * 128 * 64 * 4) + 2 * 6 * 64 * 300 * 4
    assert bwd(2, 6, 2, 128, 64, 300, 1) < bwd(2, 6, 2, 128, 64, 300, 2) < bwd(2, 6, 2, 128, 64, 300, 0)
    assert bwd(2, 6, 2, 128, 64, 300, 3) == 0
    bad = [(0, 8, 8, 64, 64, 64), (1, 8, 3, 64, 64, 64), (1, 8, 8, 129, 64, 64), (1, 8, 8, 64, 0, 64), (1, 8, 8, 64, 64, -1),
           (1, 0, 8, 64, 64, 64), (1, 8, 0, 64, 64, 64), (1, 8, 8, 64, 129, 64), (1 << 20, 2, 2, 64, 64, 64), (1, 1, 1, 64, 64, (1 << 22) + 1),
           (1, 8, 8, 64, 64, 1 << 40), (16, 16, 16, 128, 128, (1 << 18) + 1), (1 << 62, 4, 4, 8, 8, 8), (4, 1 << 62, 1, 8, 8, 8)]
    for shape in bad:
        assert fwd(*shape) == 0 and bwd(*shape, 1) == 0, shape
    assert fwd(1, 16, 16, 8, 8, 1 << 22) > 0 and fwd(1 << 20, 1, 1, 8, 8, 64) > 0       # the limits themselves
    # linear in the chunks, whatever the split: products 22 KB, two states 128, errors 32, pieces of two gradients 64, a boundary 64,
    # a segment of two chunks or more 128
    for shape in ((1, 1, 1, 128, 128, 1 << 22), (1, 16, 2, 128, 128, 1 << 22), (1 << 10, 64, 64, 128, 128, 1024), (3, 5, 5, 128, 128, 100)):
        units = shape[0] * shape[1] * -(-shape[5] // 64)
        assert 0 < bwd(*shape, 0) <= units * 400 * 1024 + (1 << 20), shape
    norm = lib.packmamba_layernorm_bwd_workspace_size
    up = lambda n: (n + 255) // 256 * 256  # noqa: E731
    assert norm(1, 48, 1, 1) == up(2 * 48 * 4) and norm(4, 48, 130, 1) == up(4 * 17 * 2 * 48 * 4)       # tiles of 8 tokens
    assert norm(8, 2048, 4096, 1) == up(8 * 64 * 2 * 2048 * 4) and norm(8, 2048, 4096, 0) == up(8 * 128 * 2 * 2048 * 4)
    for b, d, n in [(0, 48, 8), (1, 0, 8), (1, 48, 0), (1, (1 << 26) - 31, 1), ((1 << 20) + 1, 4, 1), (1 << 10, 4, 1 << 16), (1, 4, 1 << 31),
                    (1, 1 << 20, 1 << 14), (1 << 62, 4, 4), (4, 1 << 62, 4)]:
        assert norm(b, d, n, 1) == 0, (b, d, n)
    assert norm(1, 48, 8, 5) == 0


def _call(fn, good):
    def call(**at):
        a = list(good)
        for i, v in at.items():
            a[int(i[1:])] = v
        return fn(*a)
    return call


@pytest.mark.skipif(_gpu_visible(), reason="fake pointers are only passed where no GPU exists")
def test_argument_errors_before_launch():
    lib = _lib()
    P, U = 0x10000, 0x10008         # fake, aligned and not; every case must fail validation first
    # q, k, v, beta, decay, pos, initial, scale, out, final, ws, bytes, batch, heads, groups, dk, dv, seqlen, per_token, dtype, stream
    fwd = _call(lib.packmamba_delta_rule_fwd, [P, P, P, P, P, P, None, 1.0, P, None, P, 1 << 40, 2, 4, 2, 64, 64, 100, 1, 1, None])
    for i in (0, 1, 2, 3, 5, 8):
        assert fwd(**{f"_{i}": None}) == 1, i
    for i in (0, 1, 2, 3, 4, 5, 6, 8, 9, 10):
        assert fwd(**{f"_{i}": U}) == 4, i
    for i in (12, 13, 14, 15, 16, 17):
        assert fwd(**{f"_{i}": 0}) == 2 and fwd(**{f"_{i}": -1}) == 2, i
    assert fwd(_14=3) == 2 and fwd(_15=129) == 3 and fwd(_16=129) == 3 and fwd(_19=3) == 3 and fwd(_19=-1) == 3
    assert fwd(_12=1 << 62) == 2 and fwd(_17=1 << 31) == 2 and fwd(_12=1 << 17, _17=1 << 10) == 2
    need = lib.packmamba_delta_rule_fwd_workspace_size(2, 4, 2, 64, 64, 100)
    assert fwd(_10=None) == 5 and fwd(_11=need - 1) == 5
    # q, k, v, beta, decay, pos, initial, scale, dout, dfinal, dq, dk, dv, dbeta, ddecay, dinitial, ws, bytes, batch, heads, groups,
    # dk, dv, seqlen, per_token, dtype, stream
    bwd = _call(lib.packmamba_delta_rule_bwd, [P, P, P, P, P, P, P, 1.0, P, P, P, P, P, P, P, P, P, 1 << 40, 2, 4, 2, 64, 64, 100, 1, 1, None])
    for i in (0, 1, 2, 3, 5, 8, 10, 11, 12, 13):
        assert bwd(**{f"_{i}": None}) == 1, i
    assert bwd(_4=None) == 1 and bwd(_6=None) == 1 and bwd(_15=None) == 1      # ddecay without a decay, states without gradients
    for i in (0, 1, 2, 3, 4, 5, 6, 8, 9, 10, 11, 12, 13, 14, 15, 16):
        assert bwd(**{f"_{i}": U}) == 4, i
    for dtype in (0, 1, 2):
        need = lib.packmamba_delta_rule_bwd_workspace_size(2, 4, 2, 64, 64, 100, dtype)
        assert bwd(_17=need - 1, _25=dtype) == 5
    assert bwd(_16=None) == 5 and bwd(_20=3) == 2 and bwd(_21=200) == 3 and bwd(_25=9) == 3 and bwd(_23=0) == 2
    # q, k, v, beta, decay, pos, state, scale, out, batch, heads, groups, dk, dv, per_token, dtype, stream
    step = _call(lib.packmamba_delta_rule_step, [P, P, P, P, P, None, P, 1.0, P, 2, 4, 2, 64, 64, 1, 1, None])
    for i in (0, 1, 2, 3, 6, 8):
        assert step(**{f"_{i}": None}) == 1, i
    for i in (0, 1, 2, 3, 4, 5, 6, 8):
        assert step(**{f"_{i}": U}) == 4, i
    assert step(_11=3) == 2 and step(_13=129) == 3 and step(_12=129) == 3 and step(_15=7) == 3 and step(_9=(1 << 20) + 1) == 2
    # x, eps, out, rnorm, batch, dim, seqlen, groups, dtype, stream
    lf = _call(lib.packmamba_head_l2norm_fwd, [P, 1e-6, P, P, 2, 8, 10, 2, 1, None])
    lb = _call(lib.packmamba_head_l2norm_bwd, [P, P, P, P, 2, 8, 10, 2, 1, None])
    for i in (0, 2, 3):
        assert lf(**{f"_{i}": None}) == 1 and lf(**{f"_{i}": U}) == 4
    for i in (0, 1, 2, 3):
        assert lb(**{f"_{i}": None}) == 1 and lb(**{f"_{i}": U}) == 4
    for call in (lf, lb):
        for i in (4, 5, 6, 7):
            assert call(**{f"_{i}": 0}) == 2 and call(**{f"_{i}": -1}) == 2
        assert call(_7=3) == 2 and call(_8=3) == 3 and call(_4=1 << 62) == 2 and call(_6=1 << 31) == 2
    assert lf(_1=-1.0) == 2 and lf(_1=float("nan")) == 2
    # x, weight, bias, eps, out, mean, rstd, batch, dim, seqlen, dtype, stream
    nf = _call(lib.packmamba_layernorm_fwd, [P, P, None, 1e-5, P, P, P, 2, 8, 10, 1, None])
    for i in (0, 1, 4, 5, 6):
        assert nf(**{f"_{i}": None}) == 1
    for i in (0, 1, 2, 4, 5, 6):
        assert nf(**{f"_{i}": U}) == 4
    assert nf(_3=-1.0) == 2 and nf(_3=float("nan")) == 2 and nf(_8=0) == 2 and nf(_10=4) == 3 and nf(_8=1 << 26) == 2
    # x, weight, mean, rstd, dout, dresidual, dx, dweight, dbias, ws, bytes, batch, dim, seqlen, dtype, stream
    nb = _call(lib.packmamba_layernorm_bwd, [P, P, P, P, P, None, P, P, None, P, 1 << 40, 2, 8, 10, 1, None])
    for i in (0, 1, 2, 3, 4, 6, 7):
        assert nb(**{f"_{i}": None}) == 1
    for i in (0, 1, 2, 3, 4, 5, 6, 7, 8, 9):
        assert nb(**{f"_{i}": U}) == 4
    need = lib.packmamba_layernorm_bwd_workspace_size(2, 8, 10, 1)
    assert nb(_9=None) == 5 and nb(_10=need - 1) == 5 and nb(_11=-1) == 2 and nb(_14=3) == 3


def test_wrappers_refuse():
    """Shapes, types, places and layouts that do not fit raise before the library is called (on the CPU every
    call ends at the device's check at the latest)."""
    import torch
    import paper_2408_03865_amd as P
    q, v, beta, pos = torch.zeros(2, 2, 8, 5), torch.zeros(2, 4, 6, 5), torch.zeros(2, 4, 5), torch.zeros(2, 5, dtype=torch.int32)
    with pytest.raises(ValueError, match="not on a GPU"):
        P.delta_rule_fwd(q, q, v, beta, None, pos)
    with pytest.raises(ValueError, match="not on a GPU"):
        P.delta_rule_bwd(q, q, v, beta, None, pos, v)
    with pytest.raises(ValueError, match="multiple"):
        P.delta_rule_fwd(torch.zeros(2, 3, 8, 5), q, v, beta, None, pos)
    with pytest.raises(ValueError, match="head sizes"):
        P.delta_rule_fwd(torch.zeros(2, 2, 130, 5), q, v, beta, None, pos)
    with pytest.raises(ValueError, match="empty"):
        P.delta_rule_fwd(q[..., :0], q, v[..., :0], beta, None, pos)
    with pytest.raises(ValueError, match="dimensions"):
        P.delta_rule_step(q, q, v, beta, None, torch.zeros(2, 4, 8, 6))
    with pytest.raises(ValueError, match="not on a GPU"):
        P.delta_rule_step(q[..., 0], q[..., 0], v[..., 0], beta[..., 0], None, torch.zeros(2, 4, 8, 6))
    x = torch.zeros(2, 6, 5)
    for fwd in (lambda x, **o: P.head_l2norm_fwd(x, **o), lambda x, **o: P.head_l2norm_bwd(x, torch.ones(2, 1, 5), x, **o)):
        with pytest.raises(ValueError, match="groups"):
            fwd(x, groups=4)
        with pytest.raises(ValueError, match="groups"):
            fwd(x, groups=0)
        with pytest.raises(ValueError, match="not on a GPU"):
            fwd(x, groups=2)
    for norm in (lambda x: P.layernorm_fwd(x, torch.ones(6)), lambda x: P.layernorm_bwd(x, torch.ones(6), torch.ones(2, 5), torch.ones(2, 5), x)):
        with pytest.raises(ValueError, match="3 dimensions"):
            norm(x[0])
        with pytest.raises(ValueError, match="empty"):
            norm(x[..., :0])
        with pytest.raises(ValueError, match="not on a GPU"):
            norm(x)
