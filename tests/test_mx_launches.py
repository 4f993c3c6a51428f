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


def gemv(M, N, B):
    return "sqllm_mx_gemv", "iiippppip", [M, N, B, A, A, A, A, 0, 0]


def test_the_limit_of_lds_of_a_kernel_is_one_number():
    """the limit belongs to the kernel, and a thread may set it between another's setting and that other's launch: whatever the sizes, every call sets the same"""
    calls = [gemv(M, N, B) for B in (3, 7, 12, 16) for N in (2176, 5120, 8192, 28672) for M in (100, 4097, 12289, 16000, 20480, 32768, 100000)]
    calls += [gemm(T, M, N, type) for type in range(3) for T in (1, 20, 33, 40, 64) for M in (40, 500, 1000) for N in (1500, 1664, 1792, 2048, 4096)]
    calls += [quantize(200, 300, type, rows, True) for type in range(3) for rows in (False, True)]
    limit, largest = {}, {}
    for status, limits, launched in launches(calls):
        assert status == 0
        for kernel, size in limits:
            limit.setdefault(kernel, set()).add(size)
        for kernel, _, _, size in launched:
            largest[kernel] = max(size, largest.get(kernel, 0))
    assert len(limit) == 4 * 3 + 3 + 2, limit                            # column counts x shares of the gemv, types of the product of few rows, forms of the tile in fp32
    assert all(len(sizes) == 1 for sizes in limit.values()), limit
    assert all(largest[kernel] <= min(sizes) <= 160 * 1024 for kernel, sizes in limit.items())


def test_tiles_take_the_rows_they_are_made_for():
    """below 512 columns a row has fewer scales than the other form of the tiles reads at once; above 2^24 its offsets leave 32 bits"""
    calls = [gemm(T, M, N, type) for type in range(3) for T in (1, 33, 300, 4096, 20000) for M in (1, 64, 1000, 22016) for N in (1, 128, 129, 384, 385, 512, 640, 8192, 1 << 24, (1 << 24) + 1, 1 << 28)]
    short, plain, few = 0, 0, 0
    for (_, _, args), (status, _, launched) in zip(calls, launches(calls)):
        K = -(-args[2] // 128) * 128
        assert status == 0 and len(launched) == 1
        kernel = launched[0][0]
        if "tile" in kernel:
            assert ("ELb1E" in kernel) == (K < 512) and ("ELb0E" in kernel) == (K >= 512) and K <= 1 << 24, (args, kernel)
        short, plain, few = short + ("ELb1E" in kernel), plain + ("ELb0E" in kernel), few + ("few" in kernel)
    assert short and plain and few


@pytest.mark.parametrize("T,M,N,kernel", [(20, 70, 4100, "few_kernelILi{}ELi1E"), (300, 270, 1152, "few_kernelILi{}ELi2E"), (1030, 2050, 300, "ELb1E"), (2100, 4100, 640, "Li2ELNS"), (4090, 4000, 4900, "Li4ELNS")])
def test_the_sizes_of_the_range_tests_take_every_kernel(T, M, N, kernel):
    for type in range(3):
        assert kernel.format(type) in launches([gemm(T, M, N, type)])[0][2][0][0]
