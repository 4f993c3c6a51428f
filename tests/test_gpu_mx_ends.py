"""The packed 4-bit format on the GPU at the ends of its ranges: the longest rows and the most rows that the entry points take."""
import numpy as np
import pytest

from oracle import mx_oracle as mx

pytestmark = pytest.mark.gpu
LARGEST = 0x7FFFFF80


def numbers(codes, scales):
    """what a run of columns holds: uint8 [R, n / 2], uint8 [R, n / 32] on the GPU"""
    return mx.expand(codes.cpu().numpy(), scales.cpu().numpy(), 2 * codes.shape[1])


@pytest.mark.parametrize("N", [LARGEST, LARGEST - 127, LARGEST - 128])
def test_product_of_the_widest_rows(N):
    """x is zero but for three runs of columns, the last one at the rows' end; sums of multiples of 1/16 below 2^20 are exact in fp32"""
    import torch
    import paper_2306_07629_amd as sq
    print(f"mx gemm 2x3x{N}", flush=True)
    T, M, P = 2, 3, mx.padded(N)
    g = torch.Generator(device="cuda").manual_seed(N % 1000)
    wc = torch.randint(0, 256, (M, P // 2), dtype=torch.uint8, device="cuda", generator=g)
    ws = torch.randint(126, 129, (M, P // 32), dtype=torch.uint8, device="cuda", generator=g)
    xc, xs = torch.zeros((T, P // 2), dtype=torch.uint8, device="cuda"), torch.zeros((T, P // 32), dtype=torch.uint8, device="cuda")
    want = np.zeros((T, M))
    for first in (0, 1 << 30, P - 1024):
        codes, scales = slice(first // 2, first // 2 + 512), slice(first // 32, first // 32 + 32)
        xc[:, codes] = torch.randint(0, 256, (T, 512), dtype=torch.uint8, device="cuda", generator=g)
        xs[:, scales] = torch.randint(126, 129, (T, 32), dtype=torch.uint8, device="cuda", generator=g)
        if first and N % 128:                                            # columns of the padding hold zeros
            xc[:, (N + 1) // 2:] = 0
            xc[:, N // 2] &= 15 if N % 2 else 0
        want += numbers(xc[:, codes], xs[:, scales]) @ numbers(wc[:, codes], ws[:, scales]).T
    if N % 128:
        wc[:, (N + 1) // 2:] = 0
        wc[:, N // 2] &= 15 if N % 2 else 0
    y = sq.mx_gemm(sq.MxMatrix(T, N, xc, xs), sq.MxMatrix(M, N, wc, ws), torch.float32)
    assert np.array_equal(y.cpu().numpy().astype(np.float64), want)


def same_as_by_rows(packed, w, step=1 << 26):
    """a packed matrix of w's rows, compared in pieces with the quantisation of those rows alone"""
    import torch
    import paper_2306_07629_amd as sq
    return all(torch.equal(piece.codes, packed.codes[i:i + step]) and torch.equal(piece.scales, packed.scales[i:i + step])
               for i in range(0, w.shape[0], step) for piece in (sq.mx_quantize(w[i:i + step]),))


def test_quantisation_of_the_most_tiles():
    """a column of 2^31 - 128 numbers in both directions, and the same numbers as a row along the columns: 2^24 - 1 tiles each, in more than one launch"""
    import torch
    import paper_2306_07629_amd as sq
    w = torch.randn((LARGEST, 1), dtype=torch.float16, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    row = w.view(1, LARGEST)
    by_rows = sq.mx_quantize(row)
    for i in (0, 1 << 27, 1 << 30, LARGEST - 4096):                      # what the others are compared with, against the definition
        code, scale = mx.quantize(row[:, i:i + 4096].cpu().numpy().astype(np.float64))
        assert np.array_equal(by_rows.codes[:, i // 2:i // 2 + 2048].cpu().numpy(), mx.pack(code)) and np.array_equal(by_rows.scales[:, i // 32:i // 32 + 128].cpu().numpy(), scale)
    print("a column in both directions", flush=True)
    rows, columns = sq.mx_quantize(w, "both")
    assert torch.equal(columns.codes, by_rows.codes) and torch.equal(columns.scales, by_rows.scales)
    assert same_as_by_rows(rows, w)
    del rows, columns
    torch.cuda.empty_cache()
    print("a row along the columns", flush=True)
    columns = sq.mx_quantize(row, "columns")
    assert same_as_by_rows(columns, w)
    del columns, by_rows, w, row
    torch.cuda.empty_cache()


def test_calls_from_two_threads():
    """the same kernels with different needs of LDS, called by two host threads at once on streams of their own"""
    import threading
    import torch
    import paper_2306_07629_amd as sq
    rng = np.random.default_rng(3)
    work = []
    for M, T in ((20480, 40), (32768, 64)):
        w = sq.mx_quantize(torch.from_numpy(rng.normal(size=(M, 2048)).astype(np.float16)).cuda())
        few = sq.MxMatrix(M // 40, 2048, w.codes[:M // 40], w.scales[:M // 40])
        x = torch.from_numpy(rng.normal(size=(2048, 16)).astype(np.float16)).cuda()
        tokens = sq.mx_quantize(torch.from_numpy(rng.normal(size=(T, 2048)).astype(np.float16)).cuda())
        work.append((w, x, tokens, few))
    step = lambda w, x, tokens, few: (sq.mx_gemv(w, x), sq.mx_gemm(tokens, few, torch.float32))
    want = [step(*k) for k in work]
    torch.cuda.synchronize()
    got, errors = [None, None], []

    def run(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(200):
                    got[i] = step(*work[i])
                torch.cuda.current_stream().synchronize()
        except Exception as e:
            errors.append(e)
    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    assert all(torch.equal(a, b) for i in range(2) for a, b in zip(got[i], want[i]))
