"""bfloat16 rows of the decay attention are as exact as their own rounding.

Scores, states and weighted values are operands in two or three bfloat16 parts (2^-16 relative and less), sums are float32: a
value differs from the exact one by half a step of bfloat16 (2^-8 of it) and by (2^-14 + (d + N + 64) u) of the sum of
absolute values that form it (three parts of 2^-16 each, and u = 2^-24 for each addition).  One part for any of them is off by up
to 2^-8 of that sum, which the cancelling sums of random rows show in many values."""
import pytest
import torch

import decay_definition as D
import paper_2607_20214_amd as E
from gpu_util import say

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


# one and several segments and chunks, both head widths, all columns a workgroup and half of them
@pytest.mark.parametrize("B,H,N,d", [(1, 2, 40, 64), (2, 3, 700, 64), (1, 2, 700, 128), (8, 41, 130, 128), (5, 17, 1100, 128)])
def test_rows_are_rounded_once(B, H, N, d):
    say(f"[decay] precision {B}x{H}x{N}x{d}")
    g = torch.Generator(device="cuda").manual_seed(1)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")          # noqa: E731
    q, k, v, do = (rn(B, H, N, d).bfloat16() for _ in range(4))
    s0, ds = rn(B, H, d, d), rn(B, H, d, d)
    ld = torch.tensor([-0.02, -0.3, -0.002, 0.0], device="cuda").repeat(-(-H // 4))[:H]
    cfg = E.DecayConfig(B, H, N, d)
    o, _ = E.decay_fwd(cfg, q, k, v, ld, state=s0)
    grads = E.decay_bwd(cfg, q, k, v, ld, do, state=s0, dstate_out=ds)[:3]
    tau, tol = d ** -0.5, 2.0 ** -14 + (d + N + 64) * U
    for b in range(B):
        for i in (0, 1, H - 1):
            a = [t[b, i] for t in (q, k, v)]
            ref = D.head(*a, ld[i], tau, do[b, i], s0[b, i], ds[b, i])
            big = D.head(*(t.abs() for t in a), ld[i], tau, do[b, i].abs(), s0[b, i].abs(), ds[b, i].abs())
            for name, got, j in zip(("o", "dq", "dk", "dv"), (o, *grads), (0, 2, 3, 4)):
                err = (got[b, i].double() - ref[j]).abs()
                bound = 2.0 ** -8 * ref[j].abs() + tol * (1 + 2.0 ** -8) * big[j]
                assert bool((err <= bound).all()), f"{name}: worst {float((err / bound).max()):.3g} x"
