"""The decay attention by the kernels that large calls take, against the float64 definition
(decay_definition.py): workgroups of all 128 columns or half of them in the state pass and in the
readout, one segment and several, several chunks a segment, long sequences.  Each case states which kernels it means
and reads from the launch record that they ran.

Tolerances as in test_gpu_decay.py: a value within (3 h + (d + N + 64) u) of the sum of absolute
values that form it, a bfloat16 head's relative l2 norm within 1.5 h, states within 2^-16 (bfloat16 storage) + (N +
16) u of theirs; h the storage type's half step, u = 2^-24."""
import pytest
import torch

import decay_definition as D
import paper_2607_20214_amd as E
from gpu_util import say

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "f32": U}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
DECAYS = [-0.02, 0.0, -0.5, -1e-3, -float("inf"), -0.1, -4.0]

# B, H, N, d, type, lengths, with states, (kernels of the forward, of the backward)
WIDE, HALVES = ("decay_state", "decay_out"), ("decay_state_half", "decay_out_half")
CASES = [
    # one segment of three chunks, the last one short
    ((8, 41, 130, 128, "bf16", None, True), WIDE, WIDE),
    ((8, 41, 130, 128, "bf16", [130, 0, 1, 64, 65, 129, 128, 99], True), WIDE, WIDE),
    # forward in two segments of nine chunks
    ((8, 25, 1100, 128, "bf16", None, True), WIDE, WIDE),
    ((8, 25, 1100, 128, "bf16", [1100, 576, 577, 575, 0, 1, 1099, 64], True), WIDE, WIDE),
    # backward in two segments of nine chunks, forward in three of six, the two passes by different kernels
    ((5, 17, 1100, 128, "bf16", None, True), HALVES, WIDE),
    ((5, 17, 1100, 128, "bf16", [1100, 577, 1099, 1, 0], True), HALVES, WIDE),
    # long sequences: 32 segments of eight chunks forward, ten backward
    ((1, 16, 16384, 128, "bf16", None, True), WIDE, ("decay_state_half", "decay_out")),
    ((1, 16, 16384, 128, "bf16", None, False), WIDE, ("decay_state_half", "decay_out")),
    # half the columns, several chunks a segment
    ((1, 3, 4099, 128, "bf16", None, True), HALVES, ("decay_state_half", "decay_out")),
    ((1, 2, 4099, 128, "bf16", None, True), HALVES, HALVES),
    ((2, 16, 5000, 64, "bf16", [5000, 3001], True), WIDE, WIDE),
    ((2, 4, 4099, 64, "f32", [4099, 2050], True), WIDE, WIDE),
    ((2, 3, 2500, 128, "f32", [1900, 2500], True), WIDE, WIDE),
]
IDS = ["{}x{}x{}x{}{}{}".format(*c[0][:4], c[0][4], "r" if c[0][5] else "") + ("" if c[0][6] else "n") for c in CASES]


def _launched(fn):
    E.profile_enable(True)
    try:
        out = fn()
        torch.cuda.synchronize()
        names = set(E.profile_read())
    finally:
        E.profile_enable(False)
    return out, {n for n in names if n.startswith(("decay_state", "decay_out"))}


def _check(name, got, ref, scale, tol, norm=None):
    got = got.double()
    err = (got - ref).abs()
    assert bool((err <= tol * scale + 1e-30).all()), f"{name}: worst {float((err / (tol * scale + 1e-30)).max()):.3g} x"
    if norm:
        e = float(err.norm() / (ref.norm() + 1e-30))
        assert e <= norm, f"{name}: relative norm {e:.3e}"


@pytest.mark.parametrize("c,fwd,bwd", CASES, ids=IDS)
def test_against_the_definition(c, fwd, bwd):
    B, H, N, d, dtype, lengths, states = c
    say(f"[decay] {c}")
    g = torch.Generator(device="cuda").manual_seed(1)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")          # noqa: E731
    q, k, v, do = (rn(B, H, N, d).to(DT[dtype]) for _ in range(4))
    ld = torch.tensor(DECAYS, device="cuda").repeat(-(-H // len(DECAYS)))[:H]
    s0, ds = (rn(B, H, d, d), rn(B, H, d, d)) if states else (None, None)
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    lens = [N] * B if lengths is None else lengths
    for b in range(B):
        for t in (q, k, v, do):
            t[b, :, lens[b]:] = float("nan")
    cfg = E.DecayConfig(B, H, N, d, dtype)
    (o, s), names = _launched(lambda: E.decay_fwd(cfg, q, k, v, ld, state=s0, lengths=ln, zero_tail=True))
    assert names == set(fwd), f"forward by {names}"
    res, names = _launched(lambda: E.decay_bwd(cfg, q, k, v, ld, do, state=s0, dstate_out=ds, lengths=ln, want_dstate=True))
    assert names == set(bwd), f"backward by {names}"
    h, tau = HALF[dtype], d ** -0.5
    tol, ts = 3 * h + (d + N + 64) * U, (2.0 ** -16 if dtype == "bf16" else 0) + (N + 16) * U
    heads = range(H) if N < 2000 else (0, 1, H - 1)
    for b in range(B):
        n = lens[b]
        for i in heads:
            a = [t[b, i, :n] for t in (q, k, v)]
            st = [None, None] if s0 is None else [s0[b, i], ds[b, i]]
            ref = D.head(*a, ld[i], tau, do[b, i, :n], *st)
            big = D.head(*(t.abs() for t in a), ld[i], tau, do[b, i, :n].abs(), *(t if t is None else t.abs() for t in st))
            rows = (o, None, *res[:3])
            for j, name in ((0, "o"), (2, "dq"), (3, "dk"), (4, "dv")):
                what = f"{name} of sequence {b}, head {i}"
                if n:
                    _check(what, rows[j][b, i, :n], ref[j], big[j], tol, 1.5 * h if dtype == "bf16" else None)
                assert bool((rows[j][b, i, n:] == 0).all()), what + ": rows behind it"
            _check(f"state of sequence {b}, head {i}", s[b, i], ref[1], big[1], ts)
            _check(f"dstate of sequence {b}, head {i}", res[3][b, i], ref[5], big[5], ts)
    # the same bits without the states' outputs (another launch sequence where there is one segment)
    o2, _ = E.decay_fwd(cfg, q, k, v, ld, state=s0, lengths=ln, zero_tail=True, want_state=False)
    assert torch.equal(o2, o)
    again = E.decay_bwd(cfg, q, k, v, ld, do, state=s0, dstate_out=ds, lengths=ln)
    assert all(torch.equal(x, y) for x, y in zip(again[:3], res[:3]))
