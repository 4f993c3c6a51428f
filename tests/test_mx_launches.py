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
