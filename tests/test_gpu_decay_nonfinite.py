"""Infinities and NaN among the rows of the decay attention reach what the recurrence says and nothing
else: in the forward a token's value reaches the outputs of that token and later ones (a query only its own),
in the backward dQ likewise, dK and dV those of that token and earlier ones.

The float64 recurrence (oracle/operators.py) is run on the same inputs: where it is finite, the result
is finite and within the bounds of test_gpu_decay.py (the same recurrence over absolute values is finite
there too); where it is not, neither is the result."""
import numpy as np
import pytest
import torch

import paper_2607_20214_amd as E
from gpu_util import say
from oracle import operators as P

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "f32": U}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
INF, NAN = float("inf"), float("nan")
# tensor, sequence, head, token, column, value
SPECIALS = {
    "value": [("v", 0, 0, 200, 3, INF), ("v", 1, 1, 64, 5, NAN)],
    "key": [("k", 0, 1, 70, 3, INF), ("k", 1, 0, 255, 63, NAN)],
    "query": [("q", 0, 0, 130, 7, -INF), ("q", 1, 1, 63, 0, NAN)],
    "upstream": [("do", 0, 0, 65, 7, INF), ("do", 0, 1, 191, 1, NAN)],
    "first and last": [("v", 0, 0, 0, 2, NAN), ("v", 0, 1, 259, 2, INF), ("k", 1, 0, 0, 9, NAN), ("q", 1, 1, 259, 9, -INF)],
    "several": [("v", 1, 0, 60, 3, INF), ("v", 1, 0, 61, 3, -INF), ("v", 1, 0, 100, 40, NAN), ("k", 1, 1, 192, 1, INF),
                ("do", 0, 1, 10, 3, INF), ("q", 0, 1, 11, 3, INF)],
}
# B, H, N, d, lengths, heads to look at: one and several segments, ragged, and (d 128, bfloat16) workgroups of all 128 columns
CASES = [(2, 2, 260, 64, None, None), (2, 2, 260, 128, None, None), (2, 2, 260, 64, [260, 256], None), (4, 70, 260, 128, None, (0, 1, 69))]


def _np(t):
    return t.double().cpu().numpy()


def _same(name, got, ref, scale, h, N, d):
    fin = np.isfinite(ref)
    assert np.array_equal(np.isfinite(got), fin), f"{name}: finite where the definition is not, or the other way round"
    err = np.abs(got[fin] - ref[fin])
    tol = (3 * h + (d + N + 64) * U) * scale[fin] + 1e-30
    assert (err <= tol).all(), f"{name}: worst {np.max(err / tol):.3g} x"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("what", list(SPECIALS))
@pytest.mark.parametrize("c", CASES, ids=["plain64", "plain128", "ragged", "wide"])
def test_specials_reach_what_the_recurrence_says(c, what, dtype):
    B, H, N, d, lengths, heads = c
    say(f"[decay] {what} {c} {dtype}")
    g = torch.Generator(device="cuda").manual_seed(1)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")          # noqa: E731
    t = {n: rn(B, H, N, d).to(DT[dtype]) for n in ("q", "k", "v", "do")}
    s0, ds = rn(B, H, d, d), rn(B, H, d, d)
    ld = torch.tensor([-0.02, -0.5, 0.0, -4.0, -0.1], device="cuda").repeat(-(-H // 5))[:H]
    for name, b, h, tok, col, x in SPECIALS[what]:
        t[name][b, h, tok, col] = x
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    cfg = E.DecayConfig(B, H, N, d, dtype)
    o, s = E.decay_fwd(cfg, t["q"], t["k"], t["v"], ld, state=s0, lengths=ln)
    res = E.decay_bwd(cfg, t["q"], t["k"], t["v"], ld, t["do"], state=s0, dstate_out=ds, lengths=ln, want_dstate=True)
    keep = slice(None) if heads is None else list(heads)
    pick = lambda x: _np(x[:2, keep])                                     # noqa: E731
    lens = None if lengths is None else lengths[:2]
    a = [pick(t[n]) for n in ("q", "k", "v")]
    up, st, dst, lg, tau, hs = pick(t["do"]), pick(s0), pick(ds), _np(ld[keep]), d ** -0.5, HALF[dtype]
    ab = np.abs
    with np.errstate(all="ignore"):
        f, fa = P.decay_forward(*a, lg, tau, st, lens), P.decay_forward(*map(ab, a), lg, tau, ab(st), lens)
        r = P.decay_backward(*a, lg, tau, up, st, dst, lens)
        ra = P.decay_backward(*map(ab, a), lg, tau, ab(up), ab(st), ab(dst), lens)
    for b in range(2):
        n = N if lengths is None else lengths[b]
        _same("o", pick(o)[b, :, :n], f[0][b, :, :n], fa[0][b, :, :n], hs, N, d)
        for name, got, ref, sc in zip(("dq", "dk", "dv"), res, r, ra):
            _same(name, pick(got)[b, :, :n], ref[b, :, :n], sc[b, :, :n], hs, N, d)
    sh = 2.0 ** -18 if dtype == "bf16" else 0                             # (states: 2^-16 of the sums, 3 hs here)
    _same("state", pick(s), f[1], f[2], sh, N, d)
    _same("dstate", pick(res[3]), r[3], r[4], sh, N, d)


def test_rows_before_the_token_are_the_same_bits_where_the_segment_is_walked():
    # the chunks before the token's are read out as without it
    B, H, N, d = 1, 3, 1000, 64
    g = torch.Generator(device="cuda").manual_seed(2)
    q, k, v = (torch.randn(B, H, N, d, generator=g, device="cuda").bfloat16() for _ in range(3))
    ld = torch.tensor([-0.01, -0.2, 0.0], device="cuda")
    cfg = E.DecayConfig(B, H, N, d)
    ref, _ = E.decay_fwd(cfg, q, k, v, ld)
    v[0, 1, 500, 6] = INF
    o, _ = E.decay_fwd(cfg, q, k, v, ld)
    assert torch.equal(o[0, 0], ref[0, 0]) and torch.equal(o[0, 2], ref[0, 2])
    assert torch.equal(o[0, 1, :448], ref[0, 1, :448])
    others = [c for c in range(d) if c != 6]
    assert bool(torch.isfinite(o[0, 1][:, others]).all()) and bool(torch.isfinite(o[0, 1, :500]).all())
    assert not bool(torch.isfinite(o[0, 1, 500:, 6]).any())
