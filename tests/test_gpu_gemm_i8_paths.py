"""The 8-bit product by each of its kernels, read from the launch record: the three large tiles over one
and many K-tiles, with and without a split K, with K ranges that begin with a short K-tile, plain and head-major outputs whose
tiles lie in one sequence or cross several, outputs that take no vector stores.

Tolerances as in test_gpu_gemm_i8.py: exact sums, scaled and rounded in float32 (3.1 half steps, 2^-24 each) and once to
the output's type."""
import pytest
import torch

import paper_2607_20214_amd as E
from gpu_util import say

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TOL = {torch.float32: 3.1 * U, torch.bfloat16: 3.1 * U + 2.0 ** -8}
# M, N, K, kernel, split
CASES = [
    (3318, 4398, 496, "gemm_i8_256x256", False),       # K 3 x 128 + 112
    (8002, 2048, 2048, "gemm_i8_256x256", False),
    (8000, 2048, 256, "gemm_i8_256x256", False),
    (1188, 3449, 6864, "gemm_i8_256x256", True),       # 53 x 128 + 80 in three ranges
    (1834, 4831, 4736, "gemm_i8_256x192", False),      # 37 K-tiles
    (7000, 1280, 656, "gemm_i8_256x192", False),       # 5 x 128 + 16
    (8000, 1024, 384, "gemm_i8_256x128", False),
    (182, 5907, 4144, "gemm_i8_256x128", True),        # 32 x 128 + 48
    (200, 300, 8192, None, True),
    (1000, 2048, 2049, "gemm_i8", False),              # no multiple of 16: small tiles whatever the size
    (4097, 4100, 1001, "gemm_i8", False),
    (40, 4099, 4100, "gemm_i8_rows", False),
    (64, 4080, 2048, "gemm_i8_rows", False),           # 16 waves: fewer than 256 groups of 16 channels
]
KERNELS = {"gemm_i8_256x256", "gemm_i8_256x192", "gemm_i8_256x128", "gemm_i8", "gemm_i8_rows"}


def _rows(n, k, seed):
    """8-bit rows whose stride is a multiple of 16, with other bytes behind them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.randint(-128, 128, (n, -(-k // 16) * 16 + 16), generator=g, device="cuda", dtype=torch.int8)
    return t[:, :k], torch.rand(n, generator=g, device="cuda") + 0.01


def _run(fn):
    E.profile_enable(True)
    try:
        out = fn()
        torch.cuda.synchronize()
        return out, set(E.profile_read())
    finally:
        E.profile_enable(False)


def _check(got, a, sa, b, sb):
    ref = (a.double() @ b.double().t()) * sa.double()[:, None] * sb.double()[None]     # (|sums| < 2^31: exact)
    bad = ~((got.double() - ref).abs() <= TOL[got.dtype] * ref.abs())
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} values off, first at {bad.nonzero()[0].tolist()}"


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("M,N,K,kernel,split", CASES)
def test_kernels(M, N, K, kernel, split, out):
    say(f"[gemm_i8] {M}x{N}x{K} {kernel} {out}")
    (a, sa), (b, sb) = _rows(M, K, 1), _rows(N, K, 2)
    c, names = _run(lambda: E.gemm_i8(a, sa, b, sb, out_dtype=out))
    assert ("gemm_i8_reduce" in names) == split, names
    assert kernel is None or names & KERNELS == {kernel}, names
    _check(c, a, sa, b, sb)


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
# sequences of several tiles, of one and a bit, of less than one; a row of C in 8 columns a head; K no multiple of 128
@pytest.mark.parametrize("B,H,S,d,K,kernel", [
    (1, 16, 8192, 128, 512, "gemm_i8_256x256"), (2, 16, 4001, 128, 272, "gemm_i8_256x256"), (25, 32, 320, 64, 256, "gemm_i8_256x256"),
    (100, 16, 80, 128, 400, "gemm_i8_256x256"), (4, 6, 2000, 256, 400, "gemm_i8_256x192"), (3, 192, 2048, 8, 1024, "gemm_i8_256x192"),
    (8, 8, 1000, 128, 384, "gemm_i8_256x128"), (8000, 8, 1, 128, 384, "gemm_i8_256x128"), (7, 128, 1024, 8, 384, "gemm_i8_256x128"),
])
def test_head_major_outputs_of_large_tiles(B, H, S, d, K, kernel, out):
    say(f"[gemm_i8] head-major {B}x{H}x{S}x{d} K {K} {out}")
    (a, sa), (b, sb) = _rows(B * S, K, 3), _rows(H * d, K, 4)
    c = torch.empty(B, H, S, d, dtype=out, device="cuda")
    _, names = _run(lambda: E.gemm_i8(a, sa, b, sb, out=c))
    assert names == {kernel}, names
    plain = c.transpose(1, 2).reshape(B * S, H * d)
    _check(plain, a, sa, b, sb)
    assert torch.equal(plain, E.gemm_i8(a, sa, b, sb, out_dtype=out))


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("M,N,K,kernel", [(8000, 2048, 256, "gemm_i8_256x256"), (7000, 1280, 640, "gemm_i8_256x192"),
                                          (8000, 1024, 384, "gemm_i8_256x128")])
def test_outputs_of_large_tiles_without_vector_stores(M, N, K, kernel, out):
    (a, sa), (b, sb) = _rows(M, K, 5), _rows(N, K, 6)
    ref = E.gemm_i8(a, sa, b, sb, out_dtype=out)
    for width, off in ((N + 3, 0), (N + 8, 3), (N + 8, 8)):
        c = torch.full((M, width), 9, dtype=out, device="cuda")
        _, names = _run(lambda: E.gemm_i8(a, sa, b, sb, out=c[:, off:off + N]))
        assert names == {kernel}, names
        assert torch.equal(c[:, off:off + N], ref)
        assert bool((c[:, :off] == 9).all()) and bool((c[:, off + N:] == 9).all())
