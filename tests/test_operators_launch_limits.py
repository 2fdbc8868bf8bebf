"""Sizes at the border of what one launch holds (2^32 threads in a dimension): refused on the host, before any
launch, or planned with a kernel that fits (no GPU needed)."""
import ctypes as C

import pytest

import paper_2607_20214_amd as E

OK_PTR = C.c_void_p(4096)          # never dereferenced
UNSUPPORTED = -2


def _i8(M, N, K):
    ld = -(-K // 16) * 16
    return E._GemmI8Desc(M, N, K, ld, ld, N, 0, 0, E.BF16)


# 2^24 tiles of 128 x 128 (K no multiple of 16, or short), of 256 x 256, and far more
@pytest.mark.parametrize("M,N,K", [(129, 1 << 30, 16), (1 << 30, 129, 1000), (1 << 19, 1 << 19, 16), (257, 1 << 30, 128 * 5 + 1),
                                   (1 << 20, 1 << 20, 128), (1 << 30, 1 << 30, 2048)])
def test_products_of_too_many_tiles_are_refused(M, N, K):
    d, n, p = _i8(M, N, K), C.c_size_t(), OK_PTR
    assert E.load().elsaa_gemm_i8_workspace_bytes(C.byref(d), C.byref(n)) == UNSUPPORTED
    assert "too large" in E.load().elsaa_last_error().decode()
    assert E.load().elsaa_gemm_i8(C.byref(d), p, p, p, p, p, p, 1 << 40, None) == UNSUPPORTED


@pytest.mark.parametrize("M,N,K", [(64, 1 << 30, 16), (128, 1 << 30, 1000), (1 << 30, 128, 7), (256, 1 << 30, 128),
                                   (1 << 30, 257, 2048), (1 << 19, 1 << 19, 2048)])
def test_products_below_that_are_planned_without_splits(M, N, K):
    assert E.gemm_i8_workspace_bytes(M, N, K) == 0
