"""GPU: the calls that the package's documentation shows, as it shows them."""
import re

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("text,names", [("linear_attention_fwd", "q k v decay"), ("layernorm_fwd", "q v beta decay")])
def test_documented_calls_run(text, names):
    import torch
    import paper_2408_03865_amd as P
    block = next(b for b in P.__doc__.split("\n\n") if text in b)
    code = "\n".join(line.strip() for line in block.split("\n") if re.match(r"    \S", line))
    assert code.count("\n") >= 2
    B, H, G, dk, dv, L = 2, 4, 2, 16, 24, 70
    gen = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    have = dict(vars(P), heads=H, groups=G, x=r(B, 40, L), z=r(B, H * dv, L), bias=r(40), weight=r(H * dv), q=r(B, G, dk, L), v=r(B, H, dv, L),
                k=r(B, G, dk, L), beta=torch.rand((B, H, L), generator=gen, device="cuda"), decay=-r(B, H, L).abs(),
                position_indices=torch.arange(L, device="cuda", dtype=torch.int32).expand(B, L).contiguous())
    if "layernorm" in code:
        have.update(weight=r(40), k=r(B, G * dk, L))
    have.update({n + "1": have[n][..., 0].contiguous() for n in ("q", "v", "beta", "decay")}, k1=r(B, G, dk))
    exec(code, have)
    assert have["state"].shape == (B, H, dk, dv) and have["out"].shape == (B, H, dv) and bool(have["out"].isfinite().all())
