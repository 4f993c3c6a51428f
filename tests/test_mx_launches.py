"""Launches of the sqllm_mx_* entry points at the ends of their documented sizes (no GPU: they are taken down, none runs)."""
import pytest

from host_launches import is_possible, launches

A = 1 << 40         # an aligned address that nothing follows
LARGEST = 0x7FFFFF80
GEMM = "iiiipppppllp".replace("ll", "li")


def gemm(T, M, N, type=0):
    return "sqllm_mx_gemm", GEMM, [T, M, N, type, A, A, A, A, A, M, 0, 0]


@pytest.mark.parametrize("N", [128, 4096, 1 << 24, LARGEST - 256, LARGEST - 128, LARGEST - 127, LARGEST])
def test_products_of_wide_rows(N):
    for status, limits, launched in launches([gemm(1, 1, N), gemm(1, 40, N, 1), gemm(300, 200, N, 2)]):
        assert status == 0 and len(launched) == 1
        assert is_possible(launched[0], max([v for _, v in limits], default=0)), launched


def quantize(M, N, type, rows, columns):
    r, c = A if rows else 0, A if columns else 0
    return "sqllm_mx_quantize", "iiiplppppp", [M, N, type, A, N, r, r, c, c, 0]


@pytest.mark.parametrize("rows", [False, True])
@pytest.mark.parametrize("M,N,tiles", [(1, 1, 1), (1999, 5120, 640), (LARGEST, 1, (1 << 24) - 1), (1, LARGEST, (1 << 24) - 1), (LARGEST - 2047, 64, (1 << 24) - 17), (1 << 27, 129, 1 << 21)])
def test_quantisation_along_the_columns(M, N, tiles, rows):
    """every tile has a workgroup: an eighth of them, rounded up, for each XCD over the launches together"""
    for status, limits, launched in launches([quantize(M, N, type, rows, True) for type in range(3)]):
        assert status == 0 and launched
        assert all(is_possible(l, max([v for _, v in limits], default=0)) for l in launched), launched
        assert all(grid[0] % 8 == 0 for _, grid, _, _ in launched)
        assert sum(grid[0] for _, grid, _, _ in launched) == -(-tiles // 8) * 8
