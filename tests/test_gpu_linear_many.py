"""GPU: linear attention of so many rows and heads that a walk takes its form for them, against the
recurrence in 64 bits; the tolerances are those of the other forms."""
import pytest

import linear_reference as R
from gpu_common import note
from test_gpu_linear import backward, check, cuda, forward, make
from test_gpu_linear_edges import test_nonfinite_stays as nonfinite_stays

pytestmark = pytest.mark.gpu


# 767 and 768 rows, above with odd sizes, and heads of one feature; starts in and between chunks
@pytest.mark.parametrize("states", [True, False])
@pytest.mark.parametrize("shape", [(13, 59, 1, 16, 24, 70), (96, 8, 2, 64, 64, 131), (33, 25, 5, 37, 61, 200), (70, 12, 12, 1, 1, 65)],
                         ids=lambda s: "x".join(map(str, s)))
def test_many_rows(shape, states):
    d = make(shape, "bf16", "token", states, 31 + sum(shape))
    note(f"linear attention {shape} states={states}")
    args = (d["q"], d["k"], d["v"], d["decay"], d["pos"], d["scale"], d["initial"], d["dout"], d["dfinal"])
    ref, mag = (R.reference(*args, absolute=m) for m in (False, True))
    g = cuda(d)
    out, fin = forward(g)
    check(out, ref["out"], mag["out"], shape, "out", True)
    check(fin, ref["final_state"], mag["final_state"], shape, "final_state", False)
    import paper_2408_03865_amd as P
    short = P.linear_attention_fwd(g["q"], g["k"], g["v"], g["decay"], g["pos"], scale=g["scale"], initial_state=g["initial"])
    check(short, ref["out"], mag["out"], shape, "out", True)
    got = backward(g)
    for name in ("dq", "dk", "dv", "ddecay", "dinitial_state"):
        if got[name] is not None:
            check(got[name], ref[name], mag[name], shape, name, name in ("dq", "dk", "dv"))


def test_nonfinite_stays_in_many_rows():
    nonfinite_stays((97, 8, 1, 16, 20, 130), "bf16")
