"""Linear attention with a decay for each head as masked products of whole sequences, one head at a time, float64
torch on any device (test infrastructure: the recurrence of oracle/operators.py takes too long past a thousand tokens)."""
from __future__ import annotations

import torch

ROWS = 2048


def _powers(lg, e):
    """exp(lg e), 1 at e = 0 whatever lg."""
    return torch.where(e == 0, torch.ones_like(e), torch.exp(lg * e.clamp(min=1)))


def head(q, k, v, lg, tau, do=None, s0=None, ds=None):
    """One head, [n, d] inputs and [d, d] states: o, state and, with do, dq, dk, dv, dstate (None and zero: no state)."""
    q, k, v = q.double(), k.double(), v.double()
    n, d = q.shape
    lg = lg.double()
    t = torch.arange(n, device=q.device, dtype=torch.float64)
    zero = torch.zeros(d, d, dtype=torch.float64, device=q.device)
    s0 = zero if s0 is None else s0.double()
    ds = zero if ds is None else ds.double()
    first, last = tau * _powers(lg, t + 1)[:, None], _powers(lg, n - 1 - t)[:, None]
    whole = _powers(lg, torch.tensor(float(n), dtype=torch.float64, device=q.device))
    state = (k * last).t() @ v + whole * s0
    o = first * (q @ s0)
    if do is not None:
        do = do.double()
        dq, dk, dv = first * (do @ s0.t()), last * (v @ ds.t()), last * (k @ ds)
        dstate = (q * first).t() @ do + whole * ds
    for i in range(0, n, ROWS):
        j = min(n, i + ROWS)
        gap = t[i:j, None] - t[None, :j]
        w = torch.where(gap < 0, torch.zeros_like(gap), tau * _powers(lg, gap.clamp(min=0)))
        a = (q[i:j] @ k[:j].t()) * w
        o[i:j] += a @ v[:j]
        if do is not None:
            da = (do[i:j] @ v[:j].t()) * w
            dq[i:j] += da @ k[:j]
            dk[:j] += da.t() @ q[i:j]
            dv[:j] += a.t() @ do[i:j]
    return (o, state) if do is None else (o, state, dq, dk, dv, dstate)
