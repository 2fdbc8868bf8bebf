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


def _state_of_one_token(B, H, d, check):
    """One token for each of B * H heads: the state behind it is k v' + lambda S, o = tau q' S."""
    say(f"[limits] decay {B}x{H} states of {d}")
    g = torch.Generator(device="cuda").manual_seed(2)
    q, k, v = (torch.randn(B, H, 1, d, generator=g, device="cuda").bfloat16() for _ in range(3))
    ld = torch.linspace(-0.5, 0.0, H, device="cuda")
    o, s = E.decay_fwd(E.DecayConfig(B, H, 1, d), q, k, v, ld)
    for i in check:
        want = k[i].transpose(1, 2).float() * v[i].float()
        assert torch.equal(s[i], want), f"state of sequence {i}"      # (a product of two bfloat16 values is exact)
        # scores, state and output are each rounded to bfloat16, the sums of d terms in float32
        big = (q[i].float().abs() @ want.abs()) * d ** -0.5
        assert bool(((o[i].float() - (q[i].float() @ want) * d ** -0.5).abs() <= (3 * 2.0 ** -8 + d * 2.0 ** -24) * big).all())


@pytest.mark.parametrize("B,H,d", [(4100, 1, 128), (1025, 17, 64)])
def test_more_states_than_the_scan_has_workgroups(B, H, d):
    _state_of_one_token(B, H, d, range(B))


def test_2_20_states_of_128():
    """64 GB of states and twice that of slots: more workgroups of the scan than a launch holds."""
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 215 << 30:
        pytest.skip("needs 200 GiB of free memory")
    n = 1 << 13
    _state_of_one_token(n, 128, 128, (0, 1, n // 2 - 1, n // 2, n - 2, n - 1))
    torch.cuda.empty_cache()
