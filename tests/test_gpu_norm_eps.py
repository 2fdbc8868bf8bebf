"""The norm at the smallest and largest eps, with rows of zeros and rows far below sqrt(eps)."""
import numpy as np
import pytest
import torch

import paper_2607_20214_amd as E
from oracle import operators as P

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("eps", [2.0 ** -140, 1e-38, 1e-30, 1e-12, 1.0, 1e30])
@pytest.mark.parametrize("cols", [64, 1001])
def test_rows_of_zeros_and_small_rows(cols, eps):
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randn(4, cols, generator=g, device="cuda") for _ in range(2))
    w = torch.randn(cols, generator=g, device="cuda")
    x[0] = 0
    x[1] *= eps ** 0.5 * 1e-3
    x[2] *= eps ** 0.5
    if eps < 1e-36:
        x[1] = 0                                      # (squares below float32's range count as 0)
        x[2] *= 1e20
    np64 = lambda t: t.double().cpu().numpy()         # noqa: E731
    eps32 = float(np.float32(eps))
    y64, _ = P.rms_norm(np64(x), np64(w), eps=eps32)
    dx64, dw64, xs, ws = P.rms_norm_backward(np64(x), np64(w), np64(dy), eps=eps32)
    y, _ = E.rms_norm_fwd(x, w, eps=eps)
    dx, dw = E.rms_norm_bwd(x, w, dy, eps=eps)
    # as in test_gpu_norm.py: 96 half steps of float32, and of the terms' sizes
    assert (np.abs(np64(y) - y64) <= 97 * U * np.abs(y64) + 1e-37).all()
    assert (np.abs(np64(dx) - dx64) <= 97 * U * xs).all()
    assert (np.abs(np64(dw) - dw64) <= 250 * U * ws + 1e-37).all()
