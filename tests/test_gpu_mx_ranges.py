"""Packed 4-bit products on the GPU with scales at the ends of their range and NaN blocks, in every kernel and every place of its loops, against 64 bits.

Tolerances as in test_gpu_mx_products.py; where products may lie below 2^-149, the smallest fp32 number, each of the 64 + K / 64 roundings may also be off by that."""
import numpy as np
import pytest

from oracle import mx_oracle as mx
from test_gpu_mx_products import HALF_STEP, SMALLEST, close, dtype_of, host

pytestmark = pytest.mark.gpu
OUTSIDE = np.array([61, 75, 90, 105, 113, 141, 143, 146, 148], np.uint8)     # scale bytes that leave fp16 weights, and below them
NOTHING = np.array([0, 1, 30, 59, 60], np.uint8)                             # those whose blocks count as zeros beside fp16 results


def made(code, scales, N):
    import torch
    import paper_2306_07629_amd as sq
    codes = mx.pack(code)
    return sq.MxMatrix(len(code), N, torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()), mx.expand(codes, scales, N)


def gemv_weights(M, N, rng):
    """groups of 16 rows in turn with: scales of fp16 weights; the same with some blocks outside; blocks that count as nothing among them; all three"""
    code = rng.integers(0, 16, (M, N), dtype=np.uint8)
    scales = (121 + rng.integers(-6, 7, (M, N // 32))).astype(np.uint8)
    kind = (np.arange(M) // 16 % 4)[:, None]
    u = rng.random(scales.shape)
    scales = np.where((kind % 2 == 1) & (u < 0.03), rng.choice(OUTSIDE, scales.shape), scales)
    scales = np.where((kind >= 2) & (u > 0.6), rng.choice(NOTHING, scales.shape), scales)
    return code, scales.astype(np.uint8)


# columns: shares of 4, 5 and 8 steps to a wave, 65 steps in two rounds of 5, 224 in four of 7; rows: one group to a workgroup, and two with the last one short
@pytest.mark.parametrize("M,N", [(70, 4096), (70, 5120), (4500, 5120), (70, 8192), (4500, 8192), (70, 8320), (70, 28672)])
@pytest.mark.parametrize("B", [1, 2, 3, 4, 6, 8, 13, 16])
def test_gemv_with_blocks_outside_fp16(M, N, B):
    import torch
    import paper_2306_07629_amd as sq
    print(f"mx gemv ranges {M}x{N} batch {B}", flush=True)
    rng = np.random.default_rng(N + B)
    w, v = made(*gemv_weights(M, N, rng), N)
    x = (rng.normal(size=(N, B)) * 2.0 ** -12).astype(np.float16)
    x64 = x.astype(np.float64)
    want, S = v @ x64, np.abs(v) @ np.abs(x64)
    fits = np.abs(want) + (64 + N / 64) * 2.0 ** -23 * S < 65000
    assert fits.mean() > 0.9
    xd = torch.from_numpy(x).cuda()
    y = sq.mx_gemv(w, xd)
    close(host(y)[fits], want[fits], S[fits], N)
    first = host(y)
    sq.mx_gemv(w, xd, y, accumulate=True)
    fits &= np.abs(first + want) + (64 + N / 64) * 2.0 ** -23 * S < 65000
    close(host(y)[fits], (first + want)[fits], S[fits], N)


@pytest.mark.parametrize("N", [4096, 5120, 8192, 8320, 28672])
@pytest.mark.parametrize("B", [1, 2, 3, 4, 11, 16])
def test_gemv_of_blocks_that_count_as_nothing(N, B):
    """all scale bytes 60 or less: below half the smallest fp16 number, whatever x; beside an accumulated y nothing"""
    import torch
    import paper_2306_07629_amd as sq
    M = 40
    rng = np.random.default_rng(B)
    code = rng.integers(0, 16, (M, N), dtype=np.uint8)
    w, v = made(code, rng.integers(0, 61, (M, N // 32), dtype=np.uint8), N)
    x = torch.from_numpy((rng.choice([-1, 1], (N, B)) * 65504.0).astype(np.float16)).cuda()
    assert (np.abs(v) @ np.abs(host(x))).max() < 2.0 ** -25
    assert not bool(sq.mx_gemv(w, x).any())
    y = torch.from_numpy(rng.normal(size=(M, B)).astype(np.float16)).cuda()
    before = y.clone()
    assert torch.equal(sq.mx_gemv(w, x, y, accumulate=True), before)


@pytest.mark.parametrize("M,N", [(70, 4096), (70, 5120), (4500, 5120), (70, 8192), (4500, 8192), (70, 8320), (70, 28672)])
@pytest.mark.parametrize("B", [1, 3, 4, 13, 16])
def test_gemv_nan_blocks_everywhere(M, N, B):
    """every second row has one NaN block, at every step of a wave's share and in every round; an infinite activation in one column reaches no other"""
    import torch
    import paper_2306_07629_amd as sq
    rng = np.random.default_rng(M + N + B)
    code, scales = gemv_weights(M, N, rng)
    nan = np.arange(M) % 2 == 1
    _, v = made(code, scales, N)
    scales[nan, (np.arange(M)[nan] // 2 * 37 + 4 * 4 + 1) % (N // 32)] = 255   # 37 and the number of blocks share no factor
    w, _ = made(code, scales, N)
    x = (rng.normal(size=(N, B)) * 2.0 ** -12).astype(np.float16)
    x64 = x.astype(np.float64)
    want, S = v @ x64, np.abs(v) @ np.abs(x64)
    xd = torch.from_numpy(x).cuda()
    got = host(sq.mx_gemv(w, xd))
    assert np.isnan(got[nan]).all()
    fits = (np.abs(want) + (64 + N / 64) * 2.0 ** -23 * S < 65000) & ~nan[:, None]
    close(got[fits], want[fits], S[fits], N)
    xd[N - 1, B - 1] = float("inf")
    with_inf = host(sq.mx_gemv(w, xd))
    assert not np.isfinite(with_inf[:, B - 1]).any()
    assert np.array_equal(with_inf[:, :B - 1], got[:, :B - 1], equal_nan=True)


# one size each for the two forms of the kernel of few rows, the tiles of 128 rows in both forms, and those of 256; ends inside a tile and inside a stage
SIZES = [(20, 70, 4100), (300, 270, 1152), (1030, 2050, 300), (2100, 4100, 640), (4090, 4000, 4900)]


def exact(xv, wv):
    import torch
    x, w = torch.from_numpy(xv).cuda(), torch.from_numpy(wv).cuda()
    return torch.mm(x, w.t().contiguous()), torch.mm(x.abs(), w.abs().t().contiguous())


def near(got, want, S, K, kind, where=None):
    import torch
    tol = HALF_STEP[kind] * want.abs() * (1 + 2.0 ** -10) + SMALLEST[kind] + (64 + K / 64) * (2.0 ** -23 * S * (1 + HALF_STEP[kind]) + 2.0 ** -149)
    bad = (got.double() - want).abs() > tol
    if where is not None:
        bad &= where
    assert not bool(bad.any()), (int(bad.sum()), float((got.double() - want).abs().max()))


def random(M, N, rng, scales):
    P = mx.padded(N)
    code = rng.integers(0, 16, (M, P), dtype=np.uint8)
    code[:, N:] = 0
    return made(code, scales((M, P // 32)).astype(np.uint8), N)


@pytest.mark.parametrize("kind", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("T,M,N", SIZES)
def test_gemm_of_scales_far_apart(T, M, N, kind):
    """blocks 2^100 apart in a row, on either side: what is large decides, and what is small counts where nothing large is"""
    import paper_2306_07629_amd as sq
    print(f"mx gemm ranges {T}x{M}x{N} {kind}", flush=True)
    rng = np.random.default_rng(T + N)
    x, xv = random(T, N, rng, lambda s: 127 + rng.integers(-3, 4, s) - 100 * (rng.random(s) < 0.5))
    w, wv = random(M, N, rng, lambda s: 122 + rng.integers(-3, 4, s) - 100 * (rng.random(s) < 0.5))
    want, S = exact(xv, wv)
    y = sq.mx_gemm(x, w, dtype_of(kind))
    near(y, want, S, N, kind)
    first = y.clone()
    near(sq.mx_gemm(x, w, y=y, accumulate=True), first.double() + want, S + first.double().abs(), N, kind)


@pytest.mark.parametrize("T,M,N", SIZES)
@pytest.mark.parametrize("bx,bw", [(60, 60), (30, 97), (1, 116), (0, 0), (8, 98), (90, 33), (254, 0), (200, 160)])
def test_gemm_near_the_ends_of_fp32(T, M, N, bx, bw):
    """products among the subnormal numbers of fp32, below them (which round away), and near its largest"""
    import torch
    import paper_2306_07629_amd as sq
    rng = np.random.default_rng(bx)
    x, xv = random(T, N, rng, lambda s: np.full(s, bx))
    w, wv = random(M, N, rng, lambda s: np.full(s, bw))
    want, S = exact(xv, wv)
    near(sq.mx_gemm(x, w, torch.float32), want, S, N, "f32")


@pytest.mark.parametrize("kind", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("T,M,N", SIZES)
def test_gemm_nan_blocks_everywhere(T, M, N, kind):
    """rows of both operands with one NaN block, at every place of a stage and of a group of scales: their rows and columns of y are NaN, the rest has the same bits"""
    import torch
    import paper_2306_07629_amd as sq
    rng = np.random.default_rng(N)
    P = mx.padded(N)
    x, _ = random(T, N, rng, lambda s: 124 + rng.integers(-4, 5, s))
    w, _ = random(M, N, rng, lambda s: 119 + rng.integers(-6, 7, s))
    base = sq.mx_gemm(x, w, dtype_of(kind))
    nan = torch.zeros((T, M), dtype=torch.bool, device="cuda")
    blocks = -(-N // 32)
    for m, rows, step in ((x, T, 7), (w, M, 9)):
        at = torch.arange(step // 2, rows, step, device="cuda")
        m.scales[at, torch.arange(len(at), device="cuda") * 5 % blocks] = 255
        if m is x:
            nan[at] = True
        else:
            nan[:, at] = True
    y = sq.mx_gemm(x, w, dtype_of(kind))
    assert torch.equal(torch.isnan(y), nan) and torch.equal(y[~nan], base[~nan])
    y = torch.zeros_like(y)
    sq.mx_gemm(x, w, y=y, accumulate=True)
    assert torch.equal(torch.isnan(y), nan) and torch.equal(y[~nan], base[~nan])


@pytest.mark.parametrize("T,M,N", SIZES)
def test_gemm_beyond_fp16(T, M, N):
    import torch
    import paper_2306_07629_amd as sq
    rng = np.random.default_rng(T)
    x, xv = random(T, N, rng, lambda s: 127 + 30 + rng.integers(-2, 3, s))
    w, wv = random(M, N, rng, lambda s: 127 - 20 + rng.integers(-2, 3, s))
    want, S = exact(xv, wv)
    near(sq.mx_gemm(x, w, torch.float32), want, S, N, "f32")
    got = sq.mx_gemm(x, w, torch.float16).double()
    sure = want.abs() > 65520 * (1 + 2.0 ** -10) + (64 + N / 64) * 2.0 ** -23 * S
    assert bool(sure.any()) and bool(torch.isinf(got[sure]).all()) and torch.equal(torch.sign(got[sure]), torch.sign(want[sure]))
    near(got.to(torch.float16), want, S, N, "f16", want.abs() + (64 + N / 64) * 2.0 ** -23 * S < 65000)
