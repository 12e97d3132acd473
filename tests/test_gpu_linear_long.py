"""GPU: linear attention of the longest rows, 2^22 tokens, and a backward whose gradients and heads' parts have more than
2^32 elements.  The reference is the recurrence in 64 bits over whole sequences of such a row: its first ones, some in
its middle and its last.  Tolerances as in test_gpu_linear, with the sequence for a row."""
import pytest

import linear_reference as R
from gpu_common import note
from test_gpu_linear import check

pytestmark = pytest.mark.gpu


def inputs(B, H, G, dk, dv, L, dtype, seed, starts):
    """Rows with sequences at `starts`; values on the GPU, of which only the last row need be random."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]

    def rnd(*s):
        x = torch.empty(s, dtype=t, device="cuda")
        for h in range(s[1]):
            x[-1, h] = torch.randn(s[2:], generator=gen, device="cuda", dtype=torch.float32).to(t)
        if B > 1:
            x[:-1].fill_(0.5)
        return x

    token = torch.arange(L, device="cuda", dtype=torch.int32)
    pos = token.clone()
    for s in starts:
        pos[s:] = token[:L - s]
    return dict(q=rnd(B, G, dk, L), k=rnd(B, G, dk, L), v=rnd(B, H, dv, L), dout=rnd(B, H, dv, L),
                decay=-0.01 - 0.2 * torch.rand((B, H, L), generator=gen, device="cuda"), pos=pos.expand(B, L).contiguous(),
                scale=dk ** -0.5)


def compare(d, got, starts, shape, rounded):
    """The last row's sequences from each of starts to the next, whole."""
    B, H, G, dk, dv, L = shape
    for a, b in starts:
        note(f"  tokens {a} to {b}")
        part = {n: d[n][-1:, ..., a:b].contiguous().cpu() for n in ("q", "k", "v", "dout", "decay", "pos")}
        ref, mag = (R.reference(part["q"], part["k"], part["v"], part["decay"], part["pos"], d["scale"], None, part["dout"],
                                absolute=m) for m in (False, True))
        for name, t in got.items():
            if name == "final_state":
                if b == L:
                    check(t[-1:], ref[name], mag[name], (1, H, G, dk, dv, b - a), name, False)
            else:
                check(t[-1:, ..., a:b], ref[name], mag[name], (1, H, G, dk, dv, b - a), name, rounded and name != "ddecay")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads", [(2, 2, 16, 24), (2, 1, 128, 128)], ids=lambda s: "x".join(map(str, s)))
def test_longest_rows(heads, dtype):
    import paper_2408_03865_amd as P
    L = 1 << 22
    H, G, dk, dv = heads
    shape = (1, H, G, dk, dv, L)
    note(f"linear attention {shape} {dtype}")
    middle = 32768 * 61 + 5
    d = inputs(*shape, dtype, 3, [130, middle, middle + 200, L - 333])
    g = (d["q"], d["k"], d["v"], d["decay"], d["pos"])
    out, fin = P.linear_attention_fwd(*g, scale=d["scale"], return_final=True)
    got = P.linear_attention_bwd(*g, d["dout"], scale=d["scale"])
    got = {"out": out, "final_state": fin, **{n: got[n] for n in ("dq", "dk", "dv", "ddecay")}}
    compare(d, got, [(0, 130), (middle, middle + 200), (L - 333, L)], shape, dtype == "bf16")


def test_backward_beyond_32_bit_offsets():
    """v, dout, dv and the heads' parts of dq and dk have 4.8e9 elements."""
    import paper_2408_03865_amd as P
    B, H, G, dk, dv, L = shape = (9, 64, 1, 128, 128, 65536)
    note(f"linear attention backward {shape}")
    d = inputs(*shape, "bf16", 4, [90, 30000, 30140, L - 150])
    got = P.linear_attention_bwd(d["q"], d["k"], d["v"], d["decay"], d["pos"], d["dout"], scale=d["scale"])
    compare(d, {n: got[n] for n in ("dq", "dk", "dv", "ddecay")}, [(0, 90), (30000, 30140), (L - 150, L)], shape, True)
