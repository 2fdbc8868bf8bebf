"""The operators around attention at sizes that one launch of their usual kernels does not hold
(2^32 threads in a dimension)."""
import pytest
import torch

import paper_2607_20214_amd as E
from gpu_util import say

pytestmark = pytest.mark.gpu


def test_few_tokens_with_2_28_channels():
    M, N, K = 2, (1 << 28) + 37, 16
    say(f"[limits] gemm_i8 {M}x{N}x{K}")
    g = torch.Generator(device="cuda").manual_seed(1)
    a = torch.randint(-128, 128, (M, K), generator=g, device="cuda", dtype=torch.int8)
    b = torch.randint(-128, 128, (N, K), generator=g, device="cuda", dtype=torch.int8)
    sa, sb = torch.rand(M, generator=g, device="cuda"), torch.rand(N, generator=g, device="cuda")
    c = E.gemm_i8(a, sa, b, sb)
    step = 1 << 26
    for n in range(0, N, step):                        # (exact sums: float32 holds 2^14 K)
        m = min(N, n + step)
        ref = (a.float() @ b[n:m].float().t()) * sa[:, None] * sb[n:m]
        # float32 scaling on both sides (2 u each) and the output's half step
        assert bool(((c[:, n:m].float() - ref).abs() <= (2.0 ** -8 + 2.0 ** -20) * ref.abs()).all())
