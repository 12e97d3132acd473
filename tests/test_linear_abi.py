"""The C ABI of packmamba_linear.h on the CPU: its symbols, sizes and argument errors before anything is
enqueued, and the wrappers' refusals."""
import os
import re

import pytest

from test_abi import _gpu_visible, _lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "packmamba_linear.h")
C_TYPES = {"p": r"\*", "s": r"\bsize_t\b", "l": r"\bint64_t\b", "i": r"\bint32_t\b", "f": r"\bfloat\b"}


def test_header_and_binding_agree():
    from paper_2408_03865_amd import _lib as L
    text = re.sub(r"/\*.*?\*/", " ", open(HEADER).read(), flags=re.S)
    decls = {m.group(2): (m.group(1), [p.strip() for p in m.group(3).split(",")])
             for m in re.finditer(r"\b(int|size_t) (packmamba_\w+)\s*\(([^;{]*?)\)\s*;", text)}
    assert set(decls) == set(L.LINEAR_EXPORTS)
    lib = _lib()
    for name, (ret, params) in decls.items():
        args, size = L.LINEAR_EXPORTS[name]
        assert hasattr(lib, name) and (ret == "size_t") == size
        assert len(args) == len(params), name
        for code, p in zip(args, params):
            assert ("*" in p) == (code == "p") and re.search(C_TYPES[code], p), (name, p)


def test_sizes():
    lib = _lib()
    fwd, bwd = lib.packmamba_linear_attention_fwd_workspace_size, lib.packmamba_linear_attention_bwd_workspace_size
    assert fwd(8, 64, 8, 128, 64, 4096) == 0                    # rows and heads enough
    assert fwd(1, 8, 8, 64, 64, 3 * 64) == 0                    # few chunks
    assert fwd(1, 8, 8, 64, 64, 4 * 64) >= 8 * 2 * 64 * 64 * 4      # segments
    assert bwd(2, 6, 2, 128, 64, 300) >= 2 * 6 * 300 * 4 * (128 + 2)
    for bad in [(0, 8, 8, 64, 64, 64), (1, 8, 3, 64, 64, 64), (1, 8, 8, 129, 64, 64), (1, 8, 8, 64, 0, 64), (1, 8, 8, 64, 64, -1),
                (1 << 21, 2, 2, 64, 64, 64), (1, 1, 1, 64, 64, (1 << 22) + 1), (1, 8, 8, 64, 64, 1 << 40), (64, 64, 64, 128, 128, 1 << 17), (1 << 62, 4, 4, 8, 8, 8)]:
        assert fwd(*bad) == 0 and bwd(*bad) == 0, bad
    assert bwd(1024, 64, 64, 64, 64, 64) <= 4 * 65536 * (64 * 64 + 2 + 2 * 64 + 1) + 8 * 256       # one state a row
    norm = lib.packmamba_gated_rmsnorm_bwd_workspace_size
    up = lambda n: (n + 255) // 256 * 256  # noqa: E731
    assert norm(4, 48, 130, 6) == up(4 * 3 * 48 * 4)           # 72 tiles of 64 tokens
    assert norm(2, 48, 130, 3) == up(2 * 9 * 48 * 4)           # 18 of them: tiles of 16
    assert norm(2, 48, 8, 3) == up(2 * 48 * 4)                 # one of 8
    assert norm(2, 48, 130, 5) == 0 and norm(0, 48, 130, 3) == 0 and norm(1 << 20, 48, 1, 3) == 0 and norm(1 << 10, 8, 1 << 14, 8) == 0


@pytest.mark.skipif(_gpu_visible(), reason="fake pointers are only passed where no GPU exists")
def test_argument_errors_before_launch():
    lib = _lib()
    P, U = 0x10000, 0x10008         # fake, aligned and not; every case must fail validation first
    # q, k, v, decay, pos, initial, scale, out, final, ws, bytes, batch, heads, groups, dk, dv, seqlen, per_token, dtype, stream
    good = [P, P, P, P, P, None, 1.0, P, None, P, 1 << 40, 2, 4, 2, 64, 64, 100, 1, 1, None]

    def fwd(**at):
        a = list(good)
        for i, v in at.items():
            a[int(i[1:])] = v
        return lib.packmamba_linear_attention_fwd(*a)

    for i in (0, 1, 2, 4, 7):
        assert fwd(**{f"_{i}": None}) == 1, i
    for i in (0, 1, 2, 3, 4, 5, 7, 8, 9):
        assert fwd(**{f"_{i}": U}) == 4, i
    for i in (11, 12, 13, 14, 15, 16):
        assert fwd(**{f"_{i}": 0}) == 2 and fwd(**{f"_{i}": -1}) == 2, i
    assert fwd(_13=3) == 2 and fwd(_14=129) == 3 and fwd(_15=129) == 3 and fwd(_18=3) == 3
    assert fwd(_11=1 << 62) == 2 and fwd(_16=1 << 31) == 2 and fwd(_16=900, _9=None) == 5 and fwd(_16=900, _10=100) == 5
    # q, k, v, decay, pos, initial, scale, dout, dfinal, dq, dk, dv, ddecay, dinitial, ws, bytes, batch, ...
    good_b = [P, P, P, P, P, None, 1.0, P, None, P, P, P, P, None, P, 1 << 40, 2, 4, 2, 64, 64, 100, 1, 1, None]

    def bwd(**at):
        a = list(good_b)
        for i, v in at.items():
            a[int(i[1:])] = v
        return lib.packmamba_linear_attention_bwd(*a)

    for i in (0, 1, 2, 4, 7, 9, 10, 11):
        assert bwd(**{f"_{i}": None}) == 1, i
    assert bwd(_3=None) == 1 and bwd(_5=P) == 1 and bwd(_13=P) == 1     # ddecay without a decay, states without gradients
    for i in (0, 1, 2, 3, 4, 7, 8, 9, 10, 11, 12, 14):
        assert bwd(**{f"_{i}": U}) == 4, i
    need = lib.packmamba_linear_attention_bwd_workspace_size(2, 4, 2, 64, 64, 100)
    assert bwd(_15=need - 1) == 5 and bwd(_14=None) == 5 and bwd(_18=3) == 2 and bwd(_19=200) == 3 and bwd(_23=9) == 3
    # q, k, v, decay, pos, state, scale, out, batch, heads, groups, dk, dv, per_token, dtype, stream
    step = lib.packmamba_linear_attention_step
    assert step(P, P, P, P, None, None, 1.0, P, 2, 4, 2, 64, 64, 1, 1, None) == 1
    assert step(P, P, P, P, None, P, 1.0, P, 2, 4, 3, 64, 64, 1, 1, None) == 2
    assert step(P, P, P, P, None, P, 1.0, P, 2, 4, 2, 64, 129, 1, 1, None) == 3
    assert step(P, P, P, P, None, P, 1.0, P, 2, 4, 2, 64, 64, 1, 7, None) == 3
    assert step(P, P, P, P, U, P, 1.0, P, 2, 4, 2, 64, 64, 1, 1, None) == 4
    # x, z, w, eps, out, rstd, batch, dim, seqlen, groups, gate_first, dtype, stream
    nf, nb = lib.packmamba_gated_rmsnorm_fwd, lib.packmamba_gated_rmsnorm_bwd
    assert nf(P, None, P, 1e-5, P, P, 1, 4, 8, 2, 1, 0, None) == 1
    assert nf(P, P, P, 1e-5, P, P, 1, 4, 8, 3, 1, 0, None) == 2 and nf(P, P, P, 1e-5, P, P, 1, 4, 0, 2, 1, 0, None) == 2
    assert nf(P, P, P, -1.0, P, P, 1, 4, 8, 2, 1, 0, None) == 2 and nf(P, P, P, float("nan"), P, P, 1, 4, 8, 2, 1, 0, None) == 2
    assert nf(P, P, P, 1e-5, P, P, 1, 4, 8, 2, 1, 5, None) == 3 and nf(P, P, P, 1e-5, P, U, 1, 4, 8, 2, 1, 0, None) == 4
    ws = lib.packmamba_gated_rmsnorm_bwd_workspace_size(1, 4, 8, 2)
    assert nb(P, P, P, P, P, P, P, None, P, ws, 1, 4, 8, 2, 1, 0, None) == 1
    assert nb(P, P, P, P, P, P, P, P, P, ws - 1, 1, 4, 8, 2, 1, 0, None) == 5
    assert nb(P, P, P, P, P, P, U, P, P, ws, 1, 4, 8, 2, 1, 0, None) == 4


def test_wrappers_refuse():
    """Shapes, types, places and layouts that do not fit raise before the library is called (on the CPU every
    call ends at the device's check at the latest)."""
    import torch
    import paper_2408_03865_amd as P
    q, v, pos = torch.zeros(2, 2, 8, 5), torch.zeros(2, 4, 6, 5), torch.zeros(2, 5, dtype=torch.int32)
    with pytest.raises(ValueError, match="not on a GPU"):
        P.linear_attention_fwd(q, q, v, None, pos)
    with pytest.raises(ValueError, match="multiple"):
        P.linear_attention_fwd(torch.zeros(2, 3, 8, 5), q, v, None, pos)
    with pytest.raises(ValueError, match="head sizes"):
        P.linear_attention_fwd(torch.zeros(2, 2, 130, 5), q, v, None, pos)
    with pytest.raises(ValueError, match="empty"):
        P.linear_attention_fwd(q[..., :0], q, v[..., :0], None, pos)
    with pytest.raises(ValueError, match="dimensions"):
        P.linear_attention_step(q, q, v, None, torch.zeros(2, 4, 8, 6))
    with pytest.raises(ValueError, match="not on a GPU"):
        P.linear_attention_step(q[..., 0], q[..., 0], v[..., 0], None, torch.zeros(2, 4, 8, 6))
    x = torch.zeros(2, 6, 5)
    with pytest.raises(ValueError, match="groups"):
        P.gated_rmsnorm_fwd(x, x, torch.ones(6), groups=4)
    with pytest.raises(ValueError, match="not on a GPU"):
        P.gated_rmsnorm_bwd(x, x, torch.ones(6), torch.ones(2, 1, 5), x)
    from paper_2408_03865_amd.linear import _check
    cpu = torch.device("cpu")
    for t, err in ((x.double(), TypeError), (x[:, :5], ValueError), (x.transpose(0, 1).contiguous().transpose(0, 1), ValueError),
                   (torch.empty(2, 6, 5, device="meta"), ValueError)):
        with pytest.raises(err):
            _check(cpu, [("x", t, (2, 6, 5), torch.float32)])
    _check(cpu, [("x", x, (2, 6, 5), torch.float32), ("none", None, (1,), torch.float32)])
