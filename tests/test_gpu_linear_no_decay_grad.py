"""GPU: the backward of linear attention without the decay's gradient, whose walks are other ones, against the
recurrence in 64 bits; the tolerances are those of test_gpu_linear."""
import pytest

import linear_reference as R
from gpu_common import note
from test_gpu_linear import SHAPES, backward, check, cuda, make

pytestmark = pytest.mark.gpu

# 767 rows and 768, and above with odd sizes: from 768 on bf16 walks of heads of up to 64 features take one part
MANY = [(13, 59, 1, 16, 24, 70), (96, 8, 2, 64, 64, 131), (33, 25, 5, 37, 61, 200), (70, 12, 12, 1, 1, 65)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind,states", [("token", True), ("head", False), ("token", False), ("head", True)])
@pytest.mark.parametrize("shape", SHAPES + MANY, ids=lambda s: "x".join(map(str, s)))
def test_without_the_decays_gradient(shape, kind, states, dtype):
    d = make(shape, dtype, kind, states, 13 + sum(shape))
    note(f"linear attention backward without ddecay {shape} {kind} states={states} {dtype}")
    args = (d["q"], d["k"], d["v"], d["decay"], d["pos"], d["scale"], d["initial"], d["dout"], d["dfinal"])
    ref, mag = (R.reference(*args, absolute=m) for m in (False, True))
    got = backward(cuda(d), decay_grad=False)
    assert got["ddecay"] is None and (got["dinitial_state"] is None) == (not states)
    for name in ("dq", "dk", "dv", "dinitial_state"):
        if got[name] is not None:
            w = check(got[name], ref[name], mag[name], shape, name, dtype == "bf16" and name != "dinitial_state")
            note(f"  {name} {w[0]:.2g} of its bound, {w[1]:.2g} off")
