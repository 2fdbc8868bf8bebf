"""The masked products of decay_definition.py against the recurrence of oracle/operators.py."""
import numpy as np
import pytest
import torch

import decay_definition as D
from oracle import operators as P


@pytest.mark.parametrize("n", [1, 2, 65, 150])
@pytest.mark.parametrize("lg", [0.0, -0.03, -3.0, -float("inf")])
def test_against_the_recurrence(n, lg, monkeypatch):
    monkeypatch.setattr(D, "ROWS", 40)                 # (several pieces of rows)
    g = torch.Generator().manual_seed(1)
    q, k, v, do = (torch.randn(n, 8, generator=g, dtype=torch.float64) for _ in range(4))
    s0, ds = (torch.randn(8, 8, generator=g, dtype=torch.float64) for _ in range(2))
    a = [t.numpy()[None, None] for t in (q, k, v)]
    gl = np.array([lg])
    o, s, _ = P.decay_forward(*a, gl, 0.3, s0.numpy()[None, None])
    want = [o, s, *P.decay_backward(*a, gl, 0.3, do.numpy()[None, None], s0.numpy()[None, None], ds.numpy()[None, None])[:4]]
    got = D.head(q, k, v, torch.tensor(lg, dtype=torch.float64), 0.3, do, s0, ds)
    for x, y in zip(got, want):
        np.testing.assert_allclose(x.numpy(), y[0, 0], rtol=1e-11, atol=1e-11)
    for x, y in zip(D.head(q, k, v, torch.tensor(lg, dtype=torch.float64), 0.3), P.decay_forward(*a, gl, 0.3)):
        np.testing.assert_allclose(x.numpy(), y[0, 0], rtol=1e-11, atol=1e-11)
