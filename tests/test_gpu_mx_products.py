"""Products of packed 4-bit matrices on the GPU against 64 bits: a few fp16 columns, two packed matrices, the three products of a training step.

Tolerance of a sum of K exact products, |error| <= half a step of the result's type + (64 + K / 64) 2^-23 S with S the sum of their magnitudes:
every path adds the K products in at most 64 + K / 64 roundings per result, one matrix instruction (64 products) or one block's chain at a time,
and a rounding that may cut instead of round is off by at most 2^-23 of what it rounds, which is at most S."""
import numpy as np
import pytest

from oracle import mx_oracle as mx

pytestmark = pytest.mark.gpu
HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}
SMALLEST = {"f16": 2.0 ** -25, "bf16": 2.0 ** -134, "f32": 2.0 ** -150}
UINT = {"f16": np.uint16, "bf16": np.uint16, "f32": np.uint32}


def dtype_of(kind):
    import torch
    return {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}[kind]


def packed(M, N, rng, spread=6, base=121):
    """random codes in every column but the padding, scales within +- spread of 2^(base - 127); returns (MxMatrix, its numbers)"""
    import torch
    import paper_2306_07629_amd as sq
    P = mx.padded(N)
    code = rng.integers(0, 16, (M, P), dtype=np.uint8)
    code[:, N:] = 0
    scales = np.clip(base + rng.integers(-spread, spread + 1, (M, P // 32)), 0, 254).astype(np.uint8)
    codes = mx.pack(code)
    m = sq.MxMatrix(M, N, torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda())
    return m, mx.expand(codes, scales, N)


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def close(got, want, S, K, kind="f16", extra=0.0):
    ok = np.abs(got - want) <= HALF_STEP[kind] * np.abs(want) * (1 + 2.0 ** -10) + SMALLEST[kind] + (64 + K / 64) * 2.0 ** -23 * S * (1 + HALF_STEP[kind]) + extra
    assert ok.all(), (int((~ok).sum()), float(np.abs(got - want).max()), float(S.max()))


@pytest.mark.parametrize("M,N", [(1, 128), (3, 256), (17, 384), (33, 2048), (16, 2176), (130, 4096), (5, 11008), (64, 8192), (31, 28672), (257, 640)])
@pytest.mark.parametrize("B", [1, 2, 3, 4, 5, 7, 8, 9, 12, 15, 16])
def test_gemv(M, N, B):
    import torch
    import paper_2306_07629_amd as sq
    print(f"mx gemv {M}x{N} batch {B}", flush=True)
    rng = np.random.default_rng(M + N + B)
    w, v = packed(M, N, rng)
    x = rng.normal(size=(N, B)).astype(np.float16)
    xd = torch.from_numpy(x).cuda()
    buf = torch.full((M * B + 256,), 7.0, dtype=torch.float16, device="cuda")
    y = buf[:M * B].view(M, B)
    sq.mx_gemv(w, xd, y)
    x64 = x.astype(np.float64)
    want, S = v @ x64, np.abs(v) @ np.abs(x64)
    close(host(y), want, S, N)
    assert bool((buf[M * B:] == 7.0).all())
    first = y.clone()
    sq.mx_gemv(w, xd, y, accumulate=True)
    close(host(y), host(first) + want, S, N)
    assert torch.equal(sq.mx_gemv(w, xd), first)                        # the same call gives the same bits


@pytest.mark.parametrize("B", [1, 2, 4, 7, 16])
@pytest.mark.parametrize("what", ["wide", "tiny", "huge", "zero scale", "subnormal x"])
def test_gemv_with_scales_and_activations_at_the_ends_of_their_ranges(what, B):
    """scales that no fp16 weight could carry: the result is that of the definition as long as it is an fp16 number"""
    import torch
    import paper_2306_07629_amd as sq
    M, N = 37, 2176
    rng = np.random.default_rng(B)
    if what == "wide":                               # neighbouring blocks 2^80 apart
        w, v = packed(M, N, rng, 40, 127 - 40)
    elif what == "tiny":
        w, v = packed(M, N, rng, 3, 127 - 20)
    elif what == "huge":                             # weights beyond fp16 on small activations
        w, v = packed(M, N, rng, 2, 127 + 18)
    elif what == "subnormal x":
        w, v = packed(M, N, rng, 4, 127 + 10)
    else:                                            # every scale byte but 255; one activation, so that sums stay within fp16 in some rows
        w, v = packed(M, N, rng, 127, 100)
    x = rng.normal(size=(N, B))
    x = (x * {"huge": 2.0 ** -20, "subnormal x": 2.0 ** -22}.get(what, 1.0)).astype(np.float16)
    if what == "zero scale":
        x *= 0
        x[3] = 60000.0
    x64 = x.astype(np.float64)
    want, S = v @ x64, np.abs(v) @ np.abs(x64)
    got = host(sq.mx_gemv(w, torch.from_numpy(x).cuda()))
    fits = np.abs(want) + (64 + N / 64) * 2.0 ** -23 * S < 65000
    assert fits.any()
    close(got[fits], want[fits], S[fits], N)


@pytest.mark.parametrize("B", [1, 3, 16])
def test_gemv_nan_blocks_and_non_finite_activations(B):
    import torch
    import paper_2306_07629_amd as sq
    M, N = 40, 512
    rng = np.random.default_rng(9)
    w, v = packed(M, N, rng)
    x = torch.from_numpy(rng.normal(size=(N, B)).astype(np.float16)).cuda()
    base = host(sq.mx_gemv(w, x))
    w.scales[7, 3] = 255
    w.scales[39, 15] = 255
    got = host(sq.mx_gemv(w, x))
    others = [i for i in range(M) if i not in (7, 39)]
    assert np.isnan(got[[7, 39]]).all() and np.array_equal(got[others], base[others])
    # a non-finite activation reaches every row of its own column and no other column
    for bad in (float("inf"), float("nan")):
        xb = x.clone()
        xb[100, B - 1] = bad
        got = host(sq.mx_gemv(w, xb))
        assert not np.isfinite(got[:, B - 1]).any()
        assert np.array_equal(got[others][:, :B - 1], base[others][:, :B - 1])


SHAPES = [(1, 1, 1), (1, 5, 128), (3, 2, 130), (17, 33, 256), (31, 65, 384), (64, 64, 512), (65, 63, 640), (33, 300, 4096), (130, 257, 1000), (300, 129, 2049), (257, 513, 896), (512, 256, 11008),
          (1, 1000, 5120), (1000, 1, 300), (129, 130, 65), (16, 4096, 2048), (260, 1030, 1152)]


@pytest.mark.parametrize("kind", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("T,M,N", SHAPES)
def test_gemm(T, M, N, kind):
    import torch
    import paper_2306_07629_amd as sq
    print(f"mx gemm {T}x{M}x{N} {kind}", flush=True)
    rng = np.random.default_rng(T + M + N)
    x, xv = packed(T, N, rng, 4, 124)
    w, wv = packed(M, N, rng, 6, 119)
    want, S = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
    y = sq.mx_gemm(x, w, dtype_of(kind))
    close(host(y), want, S, N, kind)
    assert torch.equal(sq.mx_gemm(x, w, dtype_of(kind)), y)
    # into rows of a larger matrix, with and without adding to what is there
    for ld, off in ((M + 3, 1), (M + 8 - M % 8, 0)):
        big = torch.full((T, ld + 8), 3.0, dtype=dtype_of(kind), device="cuda")
        part = big[:, off:off + M]
        sq.mx_gemm(x, w, y=part)
        assert torch.equal(part, y) and bool((big[:, :off] == 3.0).all()) and bool((big[:, off + M:] == 3.0).all())
        sq.mx_gemm(x, w, y=part, accumulate=True)
        close(host(part), host(y) + want, S, N, kind)
        assert bool((big[:, :off] == 3.0).all()) and bool((big[:, off + M:] == 3.0).all())


@pytest.mark.parametrize("T,M,N,kind", [(4101, 2050, 130, "f16"), (2048, 4096, 128, "bf16"), (2305, 3900, 1152, "bf16"), (4096, 2300, 640, "f32"), (1800, 5121, 2049, "f16"), (8200, 1030, 384, "f32"), (1, 40000, 256, "f16"),
                                        (40000, 3, 130, "f32"), (260, 33000, 300, "bf16"), (2040, 8190, 4100, "f32"), (2048, 8192, 4096, "bf16")])
def test_gemm_of_many_rows(T, M, N, kind):
    """enough rows on both sides, or on one, for the kernels that large products take; ragged ends in every direction"""
    import torch
    import paper_2306_07629_amd as sq
    print(f"mx gemm {T}x{M}x{N} {kind}", flush=True)
    rng = np.random.default_rng(T + M + N)
    x, xv = packed(T, N, rng, 4, 124)
    w, wv = packed(M, N, rng, 6, 119)
    want, S = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
    ld = M + 5
    big = torch.full((T + 1, ld), 3.0, dtype=dtype_of(kind), device="cuda")
    part = big[:T, :M]
    sq.mx_gemm(x, w, y=part)
    close(host(part), want, S, N, kind)
    first = part.clone()
    assert torch.equal(sq.mx_gemm(x, w, dtype_of(kind)), first)
    sq.mx_gemm(x, w, y=part, accumulate=True)
    close(host(part), host(first) + want, S, N, kind)
    assert bool((big[:, M:] == 3.0).all()) and bool((big[T] == 3.0).all())


@pytest.mark.parametrize("kind", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("T,M,N", [(1030, 2056, 1500), (2300, 4104, 5000), (1027, 5000, 100), (4099, 2064, 260), (513, 4095, 1024)])
def test_gemm_of_many_rows_aligned(T, M, N, kind):
    """rows of y that start at 16 bytes, written and added to, with ends inside a tile; a tail of the rows is left as it was"""
    import torch
    import paper_2306_07629_amd as sq
    print(f"mx gemm aligned {T}x{M}x{N} {kind}", flush=True)
    rng = np.random.default_rng(T + M + N)
    x, xv = packed(T, N, rng, 4, 124)
    w, wv = packed(M, N, rng, 6, 119)
    want, S = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
    big = torch.full((T + 1, M + 16 - M % 8), 3.0, dtype=dtype_of(kind), device="cuda")
    part = big[:T, :M]
    sq.mx_gemm(x, w, y=part)
    first = host(part)
    close(first, want, S, N, kind)
    assert torch.equal(sq.mx_gemm(x, w, dtype_of(kind)), part)
    sq.mx_gemm(x, w, y=part, accumulate=True)
    close(host(part), first + want, S, N, kind)
    assert bool((big[:, M:] == 3.0).all()) and bool((big[T] == 3.0).all())


@pytest.mark.parametrize("kind", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("T,M,N", [(1030, 2050, 300), (1030, 2050, 600), (2300, 4098, 5000)])
def test_gemm_into_rows_at_every_alignment(T, M, N, kind):
    """row lengths and starts at every place of sixteen bytes, for every kernel of many rows"""
    import torch
    import paper_2306_07629_amd as sq
    print(f"mx gemm alignments {T}x{M}x{N} {kind}", flush=True)
    rng = np.random.default_rng(T + M + N)
    x, xv = packed(T, N, rng, 4, 124)
    w, wv = packed(M, N, rng, 6, 119)
    want, S = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
    first = None
    for less in range(8):
        m = M - less
        part = sq.MxMatrix(m, N, w.codes[:m], w.scales[:m])
        big = torch.full((T, m + less % 3 + 8), 3.0, dtype=dtype_of(kind), device="cuda")
        y = big[:, less:less + m]
        sq.mx_gemm(x, part, y=y)
        if first is None:
            first = y.clone()
            close(host(first), want, S, N, kind)
        assert torch.equal(y, first[:, :m]), less
        assert bool((big[:, :less] == 3.0).all()) and bool((big[:, less + m:] == 3.0).all()), less


@pytest.mark.parametrize("T,M,N", [(33, 65, 300), (300, 270, 1152), (2100, 4100, 640)])
def test_gemm_ends_of_the_ranges(T, M, N):
    """NaN blocks reach their rows only; scales whose products leave fp16 or fp32 give infinities where the definition does"""
    import torch
    import paper_2306_07629_amd as sq
    rng = np.random.default_rng(4)
    x, xv = packed(T, N, rng)
    w, wv = packed(M, N, rng)
    base = sq.mx_gemm(x, w, torch.float32)
    x.scales[5, 2] = 255
    w.scales[M - 1, 0] = 255
    got = sq.mx_gemm(x, w, torch.float32)
    nan = torch.zeros((T, M), dtype=torch.bool, device="cuda")
    nan[5] = True
    nan[:, M - 1] = True
    assert torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], base[~nan])
    x, xv = packed(T, N, rng, 2, 127 + 30)
    w, wv = packed(M, N, rng, 2, 127 - 20)
    want, S = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
    close(host(sq.mx_gemm(x, w, torch.float32)), want, S, N, "f32")
    got = host(sq.mx_gemm(x, w, torch.float16))
    sure = np.abs(want) > 65520 * (1 + 2.0 ** -10) + (64 + N / 64) * 2.0 ** -23 * S
    assert sure.any() and np.isinf(got[sure]).all() and (np.sign(got[sure]) == np.sign(want[sure])).all()


@pytest.mark.parametrize("T,M,N,kind", [(1, 3, 5, "f32"), (33, 130, 257, "bf16"), (200, 96, 640, "f16"), (517, 300, 260, "f32")])
def test_training_step(T, M, N, kind):
    """forward and both gradients against the formulas in 64 bits on what the operands were rounded to"""
    import torch
    import paper_2306_07629_amd as sq
    rng = np.random.default_rng(T)
    bits = {n: mx.from_double(rng.normal(size=s) * f, kind) for n, s, f in (("x", (T, N), 1.0), ("w", (M, N), 0.02), ("dy", (T, M), 1e-3))}
    v = {n: mx.to_double(b, kind) for n, b in bits.items()}
    d = {n: torch.from_numpy(b.view({2: np.int16, 4: np.int32}[b.itemsize])).cuda().view(dtype_of(kind)) for n, b in bits.items()}
    def q(a):
        c, s = mx.quantize(a)
        return mx.expand(mx.pack(c), s, a.shape[1])
    x, x_t = sq.mx_quantize(d["x"], "both")
    w, w_t = sq.mx_quantize(d["w"], "both")
    y = sq.mx_linear(d["x"], w)
    assert torch.equal(y, sq.mx_gemm(x, w, dtype_of(kind)))
    dx, dw = sq.mx_linear_backward(d["dy"], x_t, w_t)
    for got, a, b, k in ((y, q(v["x"]), q(v["w"]), kind), (dx, q(v["dy"]), q(v["w"].T), kind), (dw, q(v["dy"].T), q(v["x"].T), "f32")):
        close(host(got), a @ b.T, np.abs(a) @ np.abs(b).T, a.shape[1], k)
    dx2, dw2 = sq.mx_linear_backward(d["dy"], x_t, w_t, torch.float32, dw.clone())
    a, b = q(v["dy"].T), q(v["x"].T)
    close(host(dw2), host(dw) + a @ b.T, np.abs(a) @ np.abs(b).T, T, "f32")
    assert dx2.dtype == torch.float32


def test_gradients_against_differences():
    """operands that the format holds exactly, so the loss sum(y g) is linear in each of them and differences of it are exact: the gradient's entry is
    the loss's change when that entry of x or w changes by one representable step"""
    import torch
    import paper_2306_07629_amd as sq
    rng = np.random.default_rng(2)
    T, M, N = 40, 36, 70
    def grid(shape):                                  # every block of 32 in either direction has 4 or 6 as its largest entry: scale 1
        a = rng.choice([0.0, 0.5, 1.0, 1.5, 2.0, 3.0], shape) * rng.choice([-1.0, 1.0], shape)
        a[::5, :] = np.where(np.arange(shape[1]) % 5 == 0, 4.0, a[::5, :])
        for o in range(5):
            a[o::5, o::5] = 6.0
        return a
    x, w, g = grid((T, N)), grid((M, N)), grid((T, M))
    up = lambda a: torch.from_numpy(a).float().cuda()
    _, x_t = sq.mx_quantize(up(x), "both")
    qw, w_t = sq.mx_quantize(up(w), "both")
    dx, dw = sq.mx_linear_backward(up(g), x_t, w_t)
    loss = lambda xx, ww: float((host(sq.mx_linear(up(xx), sq.mx_quantize(up(ww)))) * g).sum())
    base = loss(x, w)
    for t, j in [(0, 0), (7, 69), (39, 33), (21, 31)]:
        x2 = x.copy()
        x2[t, j] = 3.0 if x[t, j] != 3.0 else 2.0
        assert loss(x2, w) - base == float(dx[t, j]) * (x2[t, j] - x[t, j])
    for i, j in [(0, 1), (35, 69), (32, 32), (5, 64)]:
        w2 = w.copy()
        w2[i, j] = -1.0 if w[i, j] != -1.0 else 2.0
        assert loss(x, w2) - base == float(dw[i, j]) * (w2[i, j] - w[i, j])


@pytest.mark.parametrize("B", [1, 5])
def test_dense_and_sparse_layer(B):
    """the operators as they are used together: the offline pass takes the outliers out, the rest is packed, gemv and the sparse term share y"""
    import gen
    import torch
    import paper_2306_07629_amd as sq
    M, N = 96, 1024
    w16, sens = gen.make_weights(M, N, 3), gen.make_sens(M, N, 3)
    wd = torch.from_numpy(w16.view(np.int16)).cuda()
    n_lo, n_hi, n_sens = sq.sqllm_extraction_counts(M, N, 0.004, 0.0005)
    q = sq.quantize_layer(wd, torch.from_numpy(sens.view(np.int16)).cuda(), 4, n_lo, n_hi, n_sens)
    nnz = q.nnz()
    rows = torch.repeat_interleave(torch.arange(M, device="cuda"), (q.rowptr[1:] - q.rowptr[:-1]).long())
    dense = wd.view(torch.float16).clone()
    dense[rows, q.cols[:nnz].long()] = 0.0
    packed_rest = sq.mx_quantize(dense)
    x = torch.from_numpy(gen.make_x(N, B, 3).view(np.float16).reshape(N, B)).cuda()
    y = sq.mx_gemv(packed_rest, x)
    sq.sqllm_csr_spmv(M, N, nnz, B, q.rowptr, q.cols, q.vals, x, y, accumulate=1)
    code, scale = mx.quantize(host(dense))
    W = mx.expand(mx.pack(code), scale, N)
    S64 = np.zeros((M, N))
    S64[rows.cpu().numpy(), q.cols[:nnz].cpu().numpy()] = q.vals[:nnz].view(torch.float16).float().cpu().numpy()
    x64 = host(x)
    want, S = (W + S64) @ x64, np.abs(W + S64) @ np.abs(x64)
    # y is rounded to fp16 twice: once per term
    close(host(y), want, S, N, extra=2.0 ** -11 * (np.abs(W @ x64) + (64 + N / 64) * 2.0 ** -23 * S) + 2.0 ** -25)
    assert torch.equal(packed_rest.dequantize(torch.float16).float() != 0, torch.from_numpy(W != 0).cuda())


@pytest.mark.parametrize("B", [1, 3])
def test_gemv_of_more_rows_than_a_launch(B):
    """2^28 + 37 rows: the last 64 hold numbers, the others zeros"""
    import torch
    import paper_2306_07629_amd as sq
    M, N = (1 << 28) + 37, 128
    rng = np.random.default_rng(B)
    tail, v = packed(64, N, rng)
    w = sq.MxMatrix(M, N, torch.zeros((M, 64), dtype=torch.uint8, device="cuda"), torch.full((M, 4), 120, dtype=torch.uint8, device="cuda"))
    w.codes[-64:], w.scales[-64:] = tail.codes, tail.scales
    x = torch.from_numpy(rng.normal(size=(N, B)).astype(np.float16)).cuda()
    y = sq.mx_gemv(w, x)
    xh = host(x)
    close(host(y[-64:]), v @ xh, np.abs(v) @ np.abs(xh), N)
    assert not bool(y[:-64].any())


@pytest.mark.parametrize("T,M,N,kind", [(33100, 33001, 100, "f32"), (46400, 46408, 130, "bf16")])
def test_gemm_with_a_result_beyond_four_gigabytes(T, M, N, kind):
    import torch
    import paper_2306_07629_amd as sq
    rng = np.random.default_rng(T)
    x, xv = packed(T, N, rng, 4, 124)
    w, wv = packed(M, N, rng, 6, 119)
    y = sq.mx_gemm(x, w, dtype_of(kind))
    for rows, cols in ((slice(0, 70), slice(0, 300)), (slice(T - 70, T), slice(M - 300, M)), (slice(T // 2, T // 2 + 70), slice(0, 300))):
        close(host(y[rows, cols]), xv[rows] @ wv[cols].T, np.abs(xv[rows]) @ np.abs(wv[cols]).T, N, kind)


@pytest.mark.parametrize("M,N", [(40, 300), (700, 1152), (2200, 640)])
def test_gemm_of_a_matrix_with_itself(M, N):
    import torch
    import paper_2306_07629_amd as sq
    w, v = packed(M, N, np.random.default_rng(M))
    got = sq.mx_gemm(w, w, torch.float32)
    close(host(got), v @ v.T, np.abs(v) @ np.abs(v).T, N, "f32")
    other = sq.MxMatrix(M, N, w.codes.clone(), w.scales.clone())
    assert torch.equal(sq.mx_gemm(w, other, torch.float32), got)


def test_no_rows_and_no_tokens():
    import torch
    import paper_2306_07629_amd as sq
    half = dict(dtype=torch.float16, device="cuda")
    none = sq.mx_quantize(torch.zeros((0, 256), **half))
    assert none.codes.shape == (0, 128) and none.dequantize(torch.float32).shape == (0, 256)
    assert sq.mx_gemv(none, torch.zeros((256, 3), **half)).shape == (0, 3)
    w = sq.mx_quantize(torch.ones((5, 256), **half))
    assert sq.mx_linear(torch.zeros((0, 256), **half), w).shape == (0, 5) and sq.mx_gemm(w, none).shape == (5, 0)
    torch.cuda.synchronize()


def test_two_streams_at_once():
    """calls of every operator that run side by side on two streams, sharing their weights"""
    import torch
    import paper_2306_07629_amd as sq
    rng = np.random.default_rng(12)
    w, _ = packed(1200, 2048, rng)
    xs = [torch.from_numpy(rng.normal(size=(T, 2048)).astype(np.float16)).cuda() for T in (40, 600)]
    cols = [torch.from_numpy(rng.normal(size=(2048, B)).astype(np.float16)).cuda() for B in (1, 7)]
    def step(i):
        q, q_t = sq.mx_quantize(xs[i], "both")
        return [q.codes, q_t.codes, sq.mx_gemm(q, w), sq.mx_gemv(w, cols[i]), q.dequantize(torch.float32), sq.mx_gemm(q_t, q_t, torch.float32)]
    want = [step(i) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [None, None]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = step(i)
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(a, b) for a, b in zip(got[i], want[i])), i


def test_streams_graphs_and_repeated_calls():
    """every operator on another stream than the current one's and in a replayed graph, with eager work between the replays"""
    import torch
    import paper_2306_07629_amd as sq
    rng = np.random.default_rng(6)
    w, _ = packed(300, 1152, rng)
    x = torch.from_numpy(rng.normal(size=(270, 1152)).astype(np.float16)).cuda()
    col = torch.from_numpy(rng.normal(size=(1152, 5)).astype(np.float16)).cuda()
    dy = torch.from_numpy(rng.normal(size=(270, 300)).astype(np.float16)).cuda()
    _, x_t = sq.mx_quantize(x, "both")
    _, w_t = sq.mx_quantize(w.dequantize(), "both")
    def step():
        return [sq.mx_gemv(w, col), sq.mx_gemv(w, col[:, :1].contiguous()), sq.mx_linear(x, w), *sq.mx_linear_backward(dy, x_t, w_t), w.dequantize(torch.float32)]
    want = [t.clone() for t in step()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(20):
            got = step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            out = step()
    for rep in range(4):
        for t in out:
            t.fill_(5.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), f"replay {rep}"
